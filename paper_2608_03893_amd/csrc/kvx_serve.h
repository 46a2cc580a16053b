// Internal interface of the serving operators: host checks (kvx_serve.hip), page
// plan (kvx_pages.hip), 8-bit store (kvx_store8.hip) and attention over the 8-bit
// pool (kvx_attend8.hip).
#pragma once

#include "kvx_internal.h"

namespace kvx {

struct PlanArgs {
  const int32_t* lens;      // [B]
  const int32_t* add;       // [B]
  int32_t* tables;          // [B, M]
  int32_t* ring;            // [N]
  const int32_t* free_in;   // [2] head, count
  int32_t* lens_out;        // [B]
  int32_t* cu;              // [B + 1]
  int32_t* positions;       // [T]
  int32_t* slots;           // [T]
  int32_t* free_out;        // [4] head, count, refused, rows
  int32_t B, T, M, N;
  int32_t log2p;            // page size = 1 << log2p
};
hipError_t launch_plan(const PlanArgs& a, hipStream_t stream);

struct StoreArgs {
  const void* x[2];         // K and V rows
  int64_t stride[2][3];     // elements: layer, head, token
  const int32_t* slots;     // [T]
  uint8_t* codes;           // [L, 2, H, N << log2p, d]
  float* scales;            // [L, 2, H, N]
  int32_t L, H, T, N, log2p;
};
// dtype: 0 = bf16, 1 = fp32; d: 64 or 128.
hipError_t launch_store(const StoreArgs& a, int dtype, int d, hipStream_t stream);

struct AttendArgs {
  const void* q;
  int64_t q_stride[2];      // elements: row, query head
  const uint8_t* codes;     // [2, H, N << log2p, d]
  const float* scales;      // [2, H, N]
  const int32_t* tables;    // [B, M]
  const int32_t* lens;      // [B]
  const int32_t* cu;        // [B + 1]
  void* out;                // [T, H * G, d]
  float* lse;               // [T, H * G] or nullptr
  float scale_log2;         // score factor times log2(e): softmax in powers of two
  int32_t B, H, G, T, M, N, log2p;
  int64_t keys;             // most a request has, as far as the host knows: for the choice of kernel
};
hipError_t launch_attend(const AttendArgs& a, int dtype, int d, void* ws, hipStream_t stream);
// The kernel it takes, as a trace shows it; a static string.
const char* attend_kernel_name(const AttendArgs& a, int dtype, int d);
size_t attend_ws_bytes(int B, int G, int T, int d, int dtype);
// Its kernel for many query rows a request (bf16).
hipError_t launch_attend_rows(const AttendArgs& a, int d, void* ws, hipStream_t stream);
size_t attend_rows_ws_bytes(int d);

}  // namespace kvx
