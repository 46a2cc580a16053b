// Attention over shared prefixes: both parts' kernels for many query rows, bf16.
#include "kvx_prefix8.h"

#include "kvx_attend8_rows.h"

namespace kvx {
namespace {

template <int D, int NB>
__global__ void __launch_bounds__(kThreads, 2) prefix8_common_rows_kernel(CommonPart a, float* partial) {
  attend8_rows<D, NB>(a, partial, nullptr);
}
template <int D, int NB>
__global__ void __launch_bounds__(kThreads, 2) prefix8_own_rows_kernel(OwnPart a, float* partial, int* counters) {
  attend8_rows<D, NB>(a, partial, counters);
}

}  // namespace

hipError_t launch_prefix_common_rows(const PrefixArgs& args, int d, hipStream_t stream) {
  const CommonPart a{args};
  float* partial = const_cast<float*>(a.partial);
  if (d == 64)
    hipLaunchKernelGGL((prefix8_common_rows_kernel<64, kNb>), dim3(kGrid), dim3(kThreads), 0, stream, a, partial);
  else
    hipLaunchKernelGGL((prefix8_common_rows_kernel<128, kNb>), dim3(kGrid), dim3(kThreads), 0, stream, a, partial);
  return hipGetLastError();
}

hipError_t launch_prefix_own_rows(const PrefixArgs& args, int d, void* ws, hipStream_t stream) {
  const OwnPart a{args};
  int* counters = static_cast<int*>(ws);
  float* partial = reinterpret_cast<float*>(counters + kCounters);
  if (d == 64)
    hipLaunchKernelGGL((prefix8_own_rows_kernel<64, kNb>), dim3(kGrid), dim3(kThreads), 0, stream, a, partial, counters);
  else
    hipLaunchKernelGGL((prefix8_own_rows_kernel<128, kNb>), dim3(kGrid), dim3(kThreads), 0, stream, a, partial, counters);
  return hipGetLastError();
}

}  // namespace kvx
