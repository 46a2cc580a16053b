// Internal interface of the serving operators: host checks (kvx_serve.hip), page
// plan (kvx_pages.hip), 8-bit store (kvx_store8.hip), attention over the 8-bit
// pool (kvx_attend8.hip) and over shared prefixes (kvx_prefix8_*.hip), norm and rotation (kvx_normrope.hip),
// token sampling (kvx_sample.hip).
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
  static constexpr bool kCausal = true;
  template <int NB>
  static constexpr bool kAhead = false;
  static constexpr bool kJoinLater = false;
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

// Attention over prefixes that requests share (kvx_prefix8_*.hip), in two parts: the common
// part's B, tables, lens, M and keys are the prefixes', the own part's the requests'.
// Most rows (T * H * G) of both parts in one launch, which fit the chip: of 16 rows and three
// quanta at least, two a workgroup.
constexpr int64_t kPrefixRows = 16 * 1024 / 3;
struct PrefixArgs : AttendArgs {
  const int32_t* shares;    // [prefixes + 1] requests of each prefix
  float* sums;              // [T, H * G, d] the part's weighted values
  float* stats;             // [T, H * G, 2] reference and sum of its exponentials
  uint64_t* parts;          // [T, H * G] 0: there, else in which partial sums of workgroups (parts_of)
  const float* partial;     // these, slots of slot_rows rows: values, then statistics
  int32_t prefixes, requests, slot_rows;
};
// Most workgroups of a part whose slots have so many rows, two slots each.
constexpr int prefix_groups(int slot_rows) { return slot_rows == 16 ? 1024 : slot_rows == 32 ? 768 : 256; }
hipError_t launch_prefix(const PrefixArgs& common, const PrefixArgs& own, int dtype, int d, void* ws, hipStream_t stream);
// The kernels of the two parts, as a trace shows them (the same where both go in one launch).
void prefix_kernel_names(const PrefixArgs& c, const PrefixArgs& o, int dtype, int d, const char** common, const char** own);
const char* prefix_common_kernel_name(const AttendArgs& a, int dtype, int d);
const char* prefix_own_kernel_name(const AttendArgs& a, int dtype, int d);
bool prefix_by_rows(const AttendArgs& a, int dtype, int d);      // the common part's kernel
// Rows of a slot of partial sums in the common part's kernel, and bytes of all slots.
int prefix_slot_rows(const AttendArgs& a, int dtype, int d);
size_t prefix_partial_bytes(int S, int G, int T, int d, int dtype);
// The parts in launches of their own; the own one reads the common one's sums.
hipError_t launch_prefix_common(const PrefixArgs& a, int dtype, int d, hipStream_t stream);
hipError_t launch_prefix_own(const PrefixArgs& a, int dtype, int d, void* ws, hipStream_t stream);
hipError_t launch_prefix_common_rows(const PrefixArgs& a, int d, hipStream_t stream);
hipError_t launch_prefix_own_rows(const PrefixArgs& a, int d, void* ws, hipStream_t stream);

struct NormRopeArgs {
  const void* x[2];         // queries, keys
  int64_t stride[2][2];     // elements: row, head
  const void* weight[2];    // [d] or nullptr: no norm
  void* out[2];             // [T, heads, d]
  const int32_t* positions; // [T]
  InvFreq turns;            // of each plane a position, 1 / (2 pi) times its frequency
  int64_t first;            // of a launch's waves
  float eps;
  int32_t T, heads[2];
};
hipError_t launch_norm_rope(const NormRopeArgs& a, int dtype, int d, int style, hipStream_t stream);

struct SampleArgs {
  const void* logits;
  int64_t stride;           // elements between rows
  const float* u;           // [B]
  const float *temperature, *top_p, *min_p;   // [B] or nullptr: off
  const int32_t* top_k;     // [B] or nullptr
  int32_t* tokens;          // [B]
  float* logprob;           // [B] or nullptr
  int32_t B, V;
};
hipError_t launch_sample(const SampleArgs& a, int dtype, void* ws, hipStream_t stream);
size_t sample_ws_bytes(int B);

// RoPE parameters: the map's checks and frequencies (kvx_api.hip).
kvx_status check_rope_params(const kvx_rope* r, const char* which);
void rope_frequencies(const kvx_rope& r, int d, InvFreq& out);

}  // namespace kvx
