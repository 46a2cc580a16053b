// Attention over shared prefixes: which kernels a call takes, and the kernel of both parts in one
// launch, for few query rows.
//
// For calls that do not fill the chip: the parts run side by side, in workgroups of their own, and
// leave their sums where they have them; a second launch joins every row's, four threads sharing its
// sums (one after another they were 7.7 us of five requests' 18.4 after 5332 common keys).  Bound by
// latencies: lengths, pages, keys, the sums; 12.6 + 4.3 us for these five requests, 8 heads of 5
// queries, 15.6 a call in a stream, where the 11 MB of codes would take 2.4.
#include "kvx_prefix8.h"

#include "kvx_attend8_split.h"

namespace kvx {
namespace {

template <int DT, int D, int W, int NB>
__global__ void __launch_bounds__(64 * W, (W == 4 ? kOcc<DT, D, NB> : W / 4)) prefix8_split_kernel(CommonPart c, OwnLater o, int grid) {
  __shared__ union Lds {
    SplitLds<D, W, NB> c;
    SplitLds<D, W, 1> o;
    __device__ Lds() {}
  } lds;
  const int block = blockIdx.x;
  if (block < grid)
    attend8_split<DT, D, W, NB>(c, const_cast<float*>(c.partial), nullptr, lds.c, Group{block, grid});
  else
    attend8_split<DT, D, W, 1>(o, const_cast<float*>(o.partial), nullptr, lds.o, Group{block - grid, (int)gridDim.x - grid});
}

// A row's sums of both parts, by kShares times D / 4 threads.
constexpr int kShares = 4;
template <int DT, int D>
__global__ void __launch_bounds__(256) prefix8_join_kernel(PrefixArgs c, PrefixArgs o) {
  constexpr int Q = D / 4, ROWS = 256 / (kShares * Q);
  __shared__ f32x4_t sums[256];
  __shared__ float2 stats[256];
  const int share = (int)threadIdx.x / (ROWS * Q), place = (int)threadIdx.x - share * ROWS * Q;
  const int64_t row = (int64_t)blockIdx.x * ROWS + place / Q, rows = (int64_t)o.T * o.H * o.G, to = row < rows ? row : rows - 1;
  const int t = (int)(to / (o.H * o.G)), at[1] = {place % Q * 4};
  const uint64_t own = o.parts[to], common = c.parts[to];      // (anything, for rows of no request)
  auto start = [&](int b) { return clamp_to(o.cu[clamp_to(b, o.requests)], o.T); };
  const bool live = row < rows && t >= start(0) && t < start(o.requests);
  const bool joined = live && t >= start(o.shares[0]) && t < start(o.shares[o.prefixes]);
  float top = -INFINITY, den = 0.0f;
  f32x4_t sum = {0, 0, 0, 0};
  auto add = [&](const f32x4_t (&v)[1], float2 ml) {
    const FinishOwn::Both x = FinishOwn::both(top, den, ml);
    sum = x.own * sum + x.other * v[0];
  };
  if (live) FinishOwn::each_sum<D, 8, kShares>(o, to, own, at, add, share);
  if (joined) FinishOwn::each_sum<D, 16, kShares>(c, to, common, at, add, share);
  sums[threadIdx.x] = sum;
  stats[threadIdx.x] = make_float2(top, den);
  __syncthreads();
  if (share != 0 || !live) return;
#pragma unroll
  for (int x = 1; x < kShares; ++x) {
    const f32x4_t v[1] = {sums[x * ROWS * Q + place]};
    add(v, stats[x * ROWS * Q + place]);
  }
  Finish().row<DT, D>(o, to, at[0], top, den, sum);
}

template <int DT, int D>
struct Both {
  static constexpr int W = 4, NB = 1;
  static_assert(2 * kPrefixRows * (1 + kStart) >= (int64_t)16 * NB * kLeast<W> * (256 * kOcc<DT, D, NB> - 2),
                "calls that fit have room for both parts' sums");
  static bool fits(const PrefixArgs& c, const PrefixArgs& o) {
    return split_want<W, NB>(c) + split_want<W, NB>(o) <= 256 * kOcc<DT, D, NB>;
  }
  static hipError_t launch(const PrefixArgs& c, const PrefixArgs& o, hipStream_t stream) {
    CommonPart common{c};
    OwnLater own{o};
    common.slot_rows = own.slot_rows = 16 * NB;
    const unsigned first = split_grid<DT, D, W, NB>(c), second = split_grid<DT, D, W, NB>(o);
    const size_t lds = split_lds(c) > split_lds(o) ? split_lds(c) : split_lds(o);
    hipLaunchKernelGGL((prefix8_split_kernel<DT, D, W, NB>), dim3(first + second), dim3(64 * W), lds, stream, common, own, (int)first);
    const int64_t rows = (int64_t)o.T * o.H * o.G;
    hipLaunchKernelGGL((prefix8_join_kernel<DT, D>), dim3((unsigned)((rows * (D / 4) * kShares + 255) / 256)), dim3(256), 0, stream,
                       static_cast<const PrefixArgs&>(common), static_cast<const PrefixArgs&>(own));
    return hipGetLastError();
  }
  static void name(char* to, size_t n) { std::snprintf(to, n, "prefix8_split_kernel<%d, %d, %d, %d>", DT, D, W, NB); }
};

template <typename F>
auto with_both(int dtype, int d, F f) {
  if (dtype == 0) return d == 64 ? f(Both<0, 64>()) : f(Both<0, 128>());
  return d == 64 ? f(Both<1, 64>()) : f(Both<1, 128>());
}

// Both in one launch where neither has the rows for another kernel and both together do not fill
// the chip: five requests after 5332 common keys take 16.1 us instead of 21.5 in two launches, five
// fp32 ones of 4 queries after up to 251 keys 11.2 instead of 13.8.  Beyond that (up to four times
// as much) it pays or not by chance: two requests after 30000 keys 26.3 instead of 29.0, 16 requests
// of four prefixes 27.3 instead of 24.5.
bool together(const PrefixArgs& c, const PrefixArgs& o, int dtype, int d) {
  return (int64_t)o.T * o.H * o.G <= kPrefixRows && !prefix_by_rows(c, dtype, d) && !by_rows(o, dtype, d) && !two_tiles(o, dtype) &&
         !two_tiles(c, dtype) && with_both(dtype, d, [&](auto k) { return k.fits(c, o); });
}

}  // namespace

hipError_t launch_prefix(const PrefixArgs& common, const PrefixArgs& own, int dtype, int d, void* ws, hipStream_t stream) {
  PrefixArgs c = common, o = own;
  if (!together(c, o, dtype, d)) {
    o.slot_rows = prefix_slot_rows(c, dtype, d);      // the common part's, which the own one reads
    o.sums = c.sums;
    o.stats = c.stats;
    o.parts = c.parts;
    o.partial = c.partial;
    const hipError_t e = launch_prefix_common(c, dtype, d, stream);
    return e == hipSuccess ? launch_prefix_own(o, dtype, d, ws, stream) : e;
  }
  return with_both(dtype, d, [&](auto k) { return k.launch(c, o, stream); });
}

void prefix_kernel_names(const PrefixArgs& c, const PrefixArgs& o, int dtype, int d, const char** common, const char** own) {
  if (together(c, o, dtype, d)) {
    *common = *own = with_both(dtype, d, [](auto k) { return name_of(k); });
  } else {
    *common = prefix_common_kernel_name(c, dtype, d);
    *own = prefix_own_kernel_name(o, dtype, d);
  }
}

}  // namespace kvx
