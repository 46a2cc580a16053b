// Attention over the 8-bit pool: the kernel for chunks of new tokens, bf16.
#include "kvx_attend8_rows.h"

namespace kvx {
namespace {

template <int D, int NB>
__global__ void __launch_bounds__(kThreads, 2) attend8_rows_kernel(AttendArgs a, float* partial, int* counters) {
  // Where the instructions lie in memory decides up to 1%: the main loop's, the same in all, took 824
  // us for 2048 rows over 10240 keys as compiled, 816 behind two more instructions, 819 to 825 behind
  // one, or three to eight; 820 before the body was in a header.
  if (D == 128) asm volatile("s_nop 0\ns_nop 0");
  attend8_rows<D, NB>(a, partial, counters);
}

}  // namespace

// A counter pair and two partial sums for each share's first and last unit.
size_t attend_rows_ws_bytes(int d) {
  return kCounters * sizeof(int) + (size_t)kGrid * 2 * kWaves * kNb * (d / 4 + 2) * 64 * sizeof(float);
}

hipError_t launch_attend_rows(const AttendArgs& a, int d, void* ws, hipStream_t stream) {
  int* counters = static_cast<int*>(ws);
  float* partial = reinterpret_cast<float*>(counters + kCounters);
  if (d == 64)
    hipLaunchKernelGGL((attend8_rows_kernel<64, kNb>), dim3(kGrid), dim3(kThreads), 0, stream, a, partial, counters);
  else
    hipLaunchKernelGGL((attend8_rows_kernel<128, kNb>), dim3(kGrid), dim3(kThreads), 0, stream, a, partial, counters);
  return hipGetLastError();
}

}  // namespace kvx
