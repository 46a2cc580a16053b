// Attention over shared prefixes: the own part's kernels for few query rows.
#include "kvx_prefix8.h"

#include "kvx_attend8_split.h"

namespace kvx {
namespace {

constexpr int kShortKeys = 64;       // of which units go to small workgroups

template <int DT, int D, int W, int NB>
__global__ void __launch_bounds__(64 * W, (W == 4 ? kOcc<DT, D, NB> : W / 4)) prefix8_own_split_kernel(OwnPart a, float* partial, int* counters) {
  __shared__ SplitLds<D, W, NB> lds;
  attend8_split<DT, D, W, NB>(a, partial, counters, lds, Group{(int)blockIdx.x, (int)gridDim.x});
}

template <int DT, int D, int W, int NB>
struct Split {
  static hipError_t launch(const OwnPart& a, void* ws, hipStream_t stream) {
    int* counters = static_cast<int*>(ws);
    hipLaunchKernelGGL((prefix8_own_split_kernel<DT, D, W, NB>), dim3(split_grid<DT, D, W, NB>(a)), dim3(64 * W),
                       split_lds(a), stream, a, reinterpret_cast<float*>(counters + kCounters), counters);
    return hipGetLastError();
  }
  static void name(char* to, size_t n) { std::snprintf(to, n, "prefix8_own_split_kernel<%d, %d, %d, %d>", DT, D, W, NB); }
};

template <int D>
struct Rows {
  static hipError_t launch(const OwnPart& a, void* ws, hipStream_t stream) { return launch_prefix_own_rows(a, D, ws, stream); }
  static void name(char* to, size_t n) { std::snprintf(to, n, "prefix8_own_rows_kernel<%d, 2>", D); }
};

// A unit a CU and more of 16 rows: small workgroups, whatever the tables hold.  Own tokens are
// ragged, and the parts of a call follow one another, so that starts count: 64 requests of 1 to 1023
// keys 23 us with large ones, 18 with small; whole calls of 48 requests of up to 2000 keys 39 and
// 36.7 us at d = 64, 54 and 50 at 128, 32 of 3000 to 4000 93 and 90; only 48 of equal length 44.9 and 45.5.
AttendArgs sizes(const AttendArgs& args, int dtype, int d) {
  AttendArgs a = args;
  if ((int64_t)a.B * a.H >= 256 && !two_tiles(args, dtype) && !by_rows(args, dtype, d) && a.keys > kShortKeys) a.keys = kShortKeys;
  return a;
}

}  // namespace

hipError_t launch_prefix_own(const PrefixArgs& args, int dtype, int d, void* ws, hipStream_t stream) {
  const AttendArgs s = sizes(args, dtype, d);
  const OwnPart a{args};
  return with_kernel<Split, Rows>(s, dtype, d, by_rows(s, dtype, d), [&](auto k) { return k.launch(a, ws, stream); });
}

const char* prefix_own_kernel_name(const AttendArgs& args, int dtype, int d) {
  const AttendArgs s = sizes(args, dtype, d);
  return with_kernel<Split, Rows>(s, dtype, d, by_rows(s, dtype, d), [](auto k) { return name_of(k); });
}

}  // namespace kvx
