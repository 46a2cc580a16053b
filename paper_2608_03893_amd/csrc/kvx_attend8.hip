// Attention over the 8-bit pool: the kernels for few query rows a request, and which kernel a
// call takes.
#include "kvx_attend8_split.h"

namespace kvx {
namespace {

template <int DT, int D, int W, int NB>
__global__ void __launch_bounds__(64 * W, (W == 4 ? kOcc<DT, D, NB> : W / 4)) attend8_split_kernel(AttendArgs a, float* partial, int* counters) {
  __shared__ SplitLds<D, W, NB> lds;
  attend8_split<DT, D, W, NB>(a, partial, counters, lds, Group{(int)blockIdx.x, (int)gridDim.x});
}

}  // namespace

// Counters, and two partial sums for each workgroup's first and last unit: most rows with
// blocks of 32 rows and three workgroups a CU.
size_t attend_ws_bytes(int B, int G, int T, int d, int dtype) {
  const size_t split = kCounters * sizeof(int) + (size_t)256 * 3 * 2 * 32 * (d + 2) * sizeof(float);
  const size_t rows = may_go_by_rows(B, G, T, dtype) ? attend_rows_ws_bytes(d) : 0;
  return split > rows ? split : rows;
}

namespace {

template <int DT, int D, int W, int NB>
struct Split {
  static hipError_t launch(const AttendArgs& a, void* ws, hipStream_t stream) {
    int* counters = static_cast<int*>(ws);
    hipLaunchKernelGGL((attend8_split_kernel<DT, D, W, NB>), dim3(split_grid<DT, D, W, NB>(a)), dim3(64 * W),
                       split_lds(a), stream, a, reinterpret_cast<float*>(counters + kCounters), counters);
    return hipGetLastError();
  }
  static void name(char* to, size_t n) { std::snprintf(to, n, "attend8_split_kernel<%d, %d, %d, %d>", DT, D, W, NB); }
};

template <int D>
struct Rows {
  static hipError_t launch(const AttendArgs& a, void* ws, hipStream_t stream) { return launch_attend_rows(a, D, ws, stream); }
  static void name(char* to, size_t n) { std::snprintf(to, n, "attend8_rows_kernel<%d, 2>", D); }
};

}  // namespace

hipError_t launch_attend(const AttendArgs& a, int dtype, int d, void* ws, hipStream_t stream) {
  return with_kernel<Split, Rows>(a, dtype, d, by_rows(a, dtype, d), [&](auto k) { return k.launch(a, ws, stream); });
}

const char* attend_kernel_name(const AttendArgs& a, int dtype, int d) {
  return with_kernel<Split, Rows>(a, dtype, d, by_rows(a, dtype, d), [](auto k) { return name_of(k); });
}

}  // namespace kvx
