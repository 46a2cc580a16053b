// Attention over shared prefixes: the common part's kernels for few query rows.
#include "kvx_prefix8.h"

#include "kvx_attend8_split.h"

namespace kvx {
namespace {

template <int DT, int D, int W, int NB>
__global__ void __launch_bounds__(64 * W, (W == 4 ? kOcc<DT, D, NB> : W / 4)) prefix8_common_split_kernel(CommonPart a, float* partial, int* counters) {
  attend8_split<DT, D, W, NB>(a, partial, counters);
}

template <int DT, int D, int W, int NB>
struct Split {
  static constexpr int kSlotRows = 16 * NB;
  static hipError_t launch(const CommonPart& a, hipStream_t stream) {
    hipLaunchKernelGGL((prefix8_common_split_kernel<DT, D, W, NB>), dim3(split_grid<DT, D, W, NB>(a)), dim3(64 * W),
                       split_lds(a), stream, a, const_cast<float*>(a.partial), nullptr);
    return hipGetLastError();
  }
};

template <int D>
struct Rows {
  static constexpr int kSlotRows = 256;
  static hipError_t launch(const CommonPart& a, hipStream_t stream) { return launch_prefix_common_rows(a, D, stream); }
};

}  // namespace

hipError_t launch_prefix_common(const PrefixArgs& args, int dtype, int d, hipStream_t stream) {
  const CommonPart a{args};
  return with_kernel<Split, Rows>(a, dtype, d, [&](auto k) { return k.launch(a, stream); });
}

int prefix_slot_rows(const AttendArgs& a, int dtype, int d) {
  return with_kernel<Split, Rows>(a, dtype, d, [&](auto k) { return decltype(k)::kSlotRows; });
}

// Four a CU with blocks of 16 rows, three with 32, one with 256; slots for a first and a last unit.
int prefix_groups(int slot_rows) { return 256 * (slot_rows == 16 ? 4 : slot_rows == 32 ? 3 : 1); }
size_t prefix_partial_bytes(int S, int G, int T, int d, int dtype) {      // whichever kernel it will be
  size_t rows = 0;
  for (int n : {16, 32, may_go_by_rows(S, G, T, dtype) ? 256 : 32})
    rows = rows > (size_t)prefix_groups(n) * n ? rows : (size_t)prefix_groups(n) * n;
  return 2 * rows * (d + 2) * sizeof(float);
}

}  // namespace kvx
