// Attention over shared prefixes: the common part's kernels for few query rows.
#include "kvx_prefix8.h"

#include "kvx_attend8_split.h"

namespace kvx {
namespace {

template <int DT, int D, int W, int NB>
__global__ void __launch_bounds__(64 * W, (W == 4 ? kOcc<DT, D, NB> : W / 4)) prefix8_common_split_kernel(CommonPart a, float* partial, int* counters) {
  __shared__ SplitLds<D, W, NB> lds;
  attend8_split<DT, D, W, NB>(a, partial, counters, lds, Group{(int)blockIdx.x, (int)gridDim.x});
}

// Large workgroups of 32 rows: 8 waves, which have the registers for a step's keys ahead, also
// where three waves a SIMD would fit (d = 64; whole calls: 64 requests after 8000 common keys 41.4
// with 12 waves, 38.5 with 8, 40 requests of four prefixes 33.3 and 28.4, 16 after 8000 22.8 and 23.3).
template <int DT, int D, int W, int NB>
struct Split {
  static constexpr int kSlotRows = 16 * NB, kWaves = NB == 2 && W > 8 ? 8 : W;
  static hipError_t launch(const CommonPart& a, hipStream_t stream) {
    hipLaunchKernelGGL((prefix8_common_split_kernel<DT, D, kWaves, NB>), dim3(split_grid<DT, D, kWaves, NB>(a)), dim3(64 * kWaves),
                       split_lds(a), stream, a, const_cast<float*>(a.partial), nullptr);
    return hipGetLastError();
  }
  static void name(char* to, size_t n) { std::snprintf(to, n, "prefix8_common_split_kernel<%d, %d, %d, %d>", DT, D, kWaves, NB); }
};

template <int D>
struct Rows {
  static constexpr int kSlotRows = 256;
  static hipError_t launch(const CommonPart& a, hipStream_t stream) { return launch_prefix_common_rows(a, D, stream); }
  static void name(char* to, size_t n) { std::snprintf(to, n, "prefix8_common_rows_kernel<%d, 2>", D); }
};

}  // namespace

// By rows from twelve 2^30 of work on, whatever the units: its partial sums are long (130 KB a
// workgroup, written and read again by the own part), but nobody waits for their join.  Measured,
// whole calls, us, split / by rows, d = 128, 8 heads, G = 8:
//   64 requests after 8191 common keys (work 4 * 2^30) 60 / 68, 32 after 32000 (7.8) 84 / 92,
//   8 of 64 new tokens after 2000 (7.8) 103 / 98, 128 after 16000 (15.6) 152 / 144, 256 after 8191
//   (16) 155 / 149, 8 of 64 after 8191 (32) 276 / 245, 64 of 16 after 4 of 8191 (64) 528 / 458
//   d = 64: 64 after 32000 (7.8) 102 / 104, 8 of 64 after 8191 (16) 194 / 171
bool prefix_by_rows(const AttendArgs& a, int dtype, int d) {
  return may_go_by_rows(a.B, a.G, a.T, dtype) && (double)a.T * a.G * a.H * a.keys * d >= 12884901888.0;
}

hipError_t launch_prefix_common(const PrefixArgs& args, int dtype, int d, hipStream_t stream) {
  const CommonPart a{args};
  return with_kernel<Split, Rows>(a, dtype, d, prefix_by_rows(a, dtype, d), [&](auto k) { return k.launch(a, stream); });
}

const char* prefix_common_kernel_name(const AttendArgs& a, int dtype, int d) {
  return with_kernel<Split, Rows>(a, dtype, d, prefix_by_rows(a, dtype, d), [](auto k) { return name_of(k); });
}

int prefix_slot_rows(const AttendArgs& a, int dtype, int d) {
  return with_kernel<Split, Rows>(a, dtype, d, prefix_by_rows(a, dtype, d), [&](auto k) { return decltype(k)::kSlotRows; });
}

// Slots for the first and the last unit of each workgroup.
size_t prefix_partial_bytes(int S, int G, int T, int d, int dtype) {      // whichever kernel it will be
  size_t rows = 0;
  for (int n : {16, 32, may_go_by_rows(S, G, T, dtype) ? 256 : 32})
    rows = rows > (size_t)prefix_groups(n) * n ? rows : (size_t)prefix_groups(n) * n;
  return 2 * rows * (d + 2) * sizeof(float);
}

}  // namespace kvx
