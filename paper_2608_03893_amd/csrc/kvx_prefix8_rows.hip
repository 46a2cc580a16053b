// Attention over shared prefixes: both parts' kernels for many query rows, bf16.
#include "kvx_prefix8.h"

#include "kvx_attend8_rows.h"

namespace kvx {
namespace {

template <int D, int NB, typename A>
__global__ void __launch_bounds__(kThreads, 2) prefix8_rows_kernel(A a, float* partial, int* counters) {
  attend8_rows<D, NB>(a, partial, counters);
}

template <typename A>
hipError_t launch(const A& a, int d, float* partial, int* counters, hipStream_t stream) {
  if (d == 64)
    hipLaunchKernelGGL((prefix8_rows_kernel<64, kNb, A>), dim3(kGrid), dim3(kThreads), 0, stream, a, partial, counters);
  else
    hipLaunchKernelGGL((prefix8_rows_kernel<128, kNb, A>), dim3(kGrid), dim3(kThreads), 0, stream, a, partial, counters);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_prefix_common_rows(const PrefixArgs& a, int d, hipStream_t stream) {
  return launch(CommonPart{a}, d, const_cast<float*>(a.partial), nullptr, stream);
}
hipError_t launch_prefix_own_rows(const PrefixArgs& a, int d, void* ws, hipStream_t stream) {
  int* counters = static_cast<int*>(ws);
  return launch(OwnPart{a}, d, reinterpret_cast<float*>(counters + kCounters), counters, stream);
}

}  // namespace kvx
