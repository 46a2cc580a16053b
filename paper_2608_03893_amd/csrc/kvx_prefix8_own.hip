// Attention over shared prefixes: the own part's kernels for few query rows.
#include "kvx_prefix8.h"

#include "kvx_attend8_split.h"

namespace kvx {
namespace {

template <int DT, int D, int W, int NB>
__global__ void __launch_bounds__(64 * W, (W == 4 ? kOcc<DT, D, NB> : W / 4)) prefix8_own_split_kernel(OwnPart a, float* partial, int* counters) {
  attend8_split<DT, D, W, NB>(a, partial, counters);
}

template <int DT, int D, int W, int NB>
struct Split {
  static hipError_t launch(const OwnPart& a, void* ws, hipStream_t stream) {
    int* counters = static_cast<int*>(ws);
    hipLaunchKernelGGL((prefix8_own_split_kernel<DT, D, W, NB>), dim3(split_grid<DT, D, W, NB>(a)), dim3(64 * W),
                       split_lds(a), stream, a, reinterpret_cast<float*>(counters + kCounters), counters);
    return hipGetLastError();
  }
};

template <int D>
struct Rows {
  static hipError_t launch(const OwnPart& a, void* ws, hipStream_t stream) { return launch_prefix_own_rows(a, D, ws, stream); }
};

}  // namespace

hipError_t launch_prefix_own(const PrefixArgs& args, int dtype, int d, void* ws, hipStream_t stream) {
  OwnPart a{args};
  // two units a CU and more: small workgroups, whatever the tables hold
  if ((int64_t)a.B * a.H >= 512 && a.keys > 1024) a.keys = 1024;
  return with_kernel<Split, Rows>(a, dtype, d, [&](auto k) { return k.launch(a, ws, stream); });
}

}  // namespace kvx
