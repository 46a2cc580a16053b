// Attention over shared prefixes: the own part's kernels for few query rows.
#include "kvx_prefix8.h"

#include "kvx_attend8_split.h"

namespace kvx {
namespace {

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

// Two units a CU and more: small workgroups, whatever the tables hold.  Own tokens are ragged, and
// the long workgroups' gain where all requests have 2000 keys and more is 3% (64 requests of 1 to
// 1023 keys 23 us with large ones, 18 with small).
AttendArgs sizes(const AttendArgs& args) {
  AttendArgs a = args;
  if ((int64_t)a.B * a.H >= 512 && a.keys > 1024) a.keys = 1024;
  return a;
}

}  // namespace

hipError_t launch_prefix_own(const PrefixArgs& args, int dtype, int d, void* ws, hipStream_t stream) {
  const AttendArgs s = sizes(args);
  OwnPart a{args};
  a.keys = s.keys;
  return with_kernel<Split, Rows>(s, dtype, d, by_rows(s, dtype, d), [&](auto k) { return k.launch(a, ws, stream); });
}

const char* prefix_own_kernel_name(const AttendArgs& args, int dtype, int d) {
  const AttendArgs s = sizes(args);
  return with_kernel<Split, Rows>(s, dtype, d, by_rows(s, dtype, d), [](auto k) { return name_of(k); });
}

}  // namespace kvx
