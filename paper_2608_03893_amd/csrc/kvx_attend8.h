// Shared by the attention kernels over the 8-bit pool (device code only): codes as matrix
// operands, reductions over the lanes that share a query row, requests, partial sums that
// pass between workgroups.
#pragma once

#include "kvx_e4m3.h"
#include "kvx_serve.h"

namespace kvx {
namespace {

constexpr float kLazy = 8.0f;    // growth of a row's maximum (log2) that is let pass
constexpr int kXcds = 8;
// Share of workgroup `block` of `grid` (a multiple of the XCDs, which take workgroups in
// turn): neighbouring shares on one XCD, whose L2 then serves a head's keys to all of its
// blocks of rows.
__device__ __forceinline__ int xcd_order(int block, int grid) {
  return block % kXcds * (grid / kXcds) + block / kXcds;
}
// Arrival counters, first in the workspace (four for each workgroup of the largest grid):
// all kernels keep them there and leave them at zero, and partial sums behind.
constexpr int kCounters = 4 * 1024;
static_assert(kCounters * sizeof(int) == KVX_ATTEND_COUNTER_BYTES, "what a caller clears");

// Largest / sum of a value over the four lanes l, l ^ 16, l ^ 32, l ^ 48.
__device__ __forceinline__ float quad_max(float v) {
  auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ __forceinline__ float quad_sum(float v) {
  auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}

// Codes 2 HALF and 2 HALF + 1 of a word as bf16, exactly.
template <bool HALF>
__device__ __forceinline__ uint32_t bf16_pair(uint32_t w) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, HALF));
}
__device__ __forceinline__ bf16x8_t bf16_octet(uint32_t lo, uint32_t hi) {
  const u32x4_t r = {bf16_pair<false>(lo), bf16_pair<true>(lo), bf16_pair<false>(hi), bf16_pair<true>(hi)};
  return __builtin_bit_cast(bf16x8_t, r);
}

__device__ __forceinline__ f32x4_t mfma(bf16x8_t a, bf16x8_t b, f32x4_t c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// bf16 terms of a probability.  Three hold an fp32 number.  For bf16 queries two: their 16 bits
// leave the rounding of the output as the only one that counts.  With one, 8 bits as in the
// output, a fifth to a third of all outputs were not the bf16 number nearest to the exact one
// (relative error 0.0018 for 0.00167 over 64 ragged requests, 0.0021 for 0.00166 in a chunk of
// 2048 x 10240; with two 0.0002 to 0.0016 of them are not).  The second term costs 1% where the
// bytes bound the time (59.3 us for 58.7, mixed batch 22.6 for 21.8) and a third where the
// products do (818 us for 618).
template <int DT>
constexpr int kTerms = DT == 0 ? 2 : 3;

// x as TERMS bf16 terms: one is x itself where that is a bf16 number; the sum of two is x to
// 16 bits, of three to 24.
template <int TERMS>
__device__ __forceinline__ void split_terms(const float* x, bf16x8_t* out) {
  float rest[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) rest[i] = x[i];
#pragma unroll
  for (int t = 0; t < TERMS; ++t) {
    u32x4_t r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      r[i] = pack2(rest[2 * i], rest[2 * i + 1]);
      rest[2 * i] -= lo_bf16(r[i]);
      rest[2 * i + 1] -= hi_bf16(r[i]);
    }
    out[t] = __builtin_bit_cast(bf16x8_t, r);
  }
}

// A request's rows and keys, clamped to what the arrays hold.
struct Request {
  int32_t row0, tokens, rows;   // first query row, new tokens, rows of a KV head (tokens * G)
  int32_t len;                  // keys
};
__device__ __forceinline__ Request request(const AttendArgs& a, int b, int len) {
  Request r;
  int c0 = a.cu[b], c1 = a.cu[b + 1];
  c0 = c0 < 0 ? 0 : c0;
  c1 = c1 > a.T ? a.T : c1;
  r.row0 = c0;
  r.tokens = c1 > c0 ? c1 - c0 : 0;
  const int64_t cap = (int64_t)a.M << a.log2p;
  r.len = len < 0 ? 0 : len < cap ? len : (int)cap;
  r.rows = r.tokens * a.G;
  return r;
}
__device__ __forceinline__ Request request(const AttendArgs& a, int b) { return request(a, b, a.lens[b]); }

// Two floats written through to memory / read from there, past this XCD's L2.
__device__ __forceinline__ void put2(float* to, float x, float y) {
  const uint64_t v = (uint64_t)__float_as_uint(x) | (uint64_t)__float_as_uint(y) << 32;
  __hip_atomic_store(reinterpret_cast<uint64_t*>(to), v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 get2(const float* from) {
  const uint64_t v = __hip_atomic_load(reinterpret_cast<const uint64_t*>(from), __ATOMIC_RELAXED,
                                       __HIP_MEMORY_SCOPE_AGENT);
  return make_float2(__uint_as_float((uint32_t)v), __uint_as_float((uint32_t)(v >> 32)));
}

// A value that all lanes share, in scalar registers.
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ int64_t uniform(int64_t v) {
  return (int64_t)((uint64_t)(uint32_t)uniform((int)(uint32_t)v) | (uint64_t)(uint32_t)uniform((int)(v >> 32)) << 32);
}

// a / b for a >= 0, b > 0, by 32-bit division where that does.
__device__ __forceinline__ int64_t divide(int64_t a, int64_t b) {
  if ((uint64_t)(a | b) >> 32 == 0) return (uint32_t)a / (uint32_t)b;
  return a / b;
}

// Last key that the rows of a request's new token `token` see.
__device__ __forceinline__ int last_key(const AttendArgs&, const Request& r, int token) { return r.len - r.tokens + token; }

// What becomes of a unit's sums (request b's): of row `to` the reference `top` of its exponents,
// their sum `den`, and the weighted values.
struct Finish {
  // Four channels from jc on.
  template <int DT, int D>
  __device__ __forceinline__ void row(const AttendArgs& a, int64_t to, int jc, float top, float den, f32x4_t sum) const {
    const f32x4_t y = sum * (den == 0.0f ? 0.0f : 1.0f / den);    // no key: 0
    if (DT == 0)
      *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.out) + to * D + jc) = make_uint2(pack2(y[0], y[1]), pack2(y[2], y[3]));
    else
      *reinterpret_cast<f32x4_t*>(static_cast<float*>(a.out) + to * D + jc) = y;
    if (a.lse != nullptr && jc == 0)
      a.lse[to] = den == 0.0f ? -INFINITY : (top + __builtin_amdgcn_logf(den)) * 0.69314718055994530942f;
  }
  // bf16, channels (4 g4 + i) C + c, C = D / 16, of one of four lanes.
  template <int D>
  __device__ __forceinline__ void tile(const AttendArgs& a, int64_t to, int g4, float m, float l, const f32x4_t* o) const {
    constexpr int C = D / 16;
    const float f = l == 0.0f ? 0.0f : 1.0f / l;    // no key: 0
    u32x4_t* y = reinterpret_cast<u32x4_t*>(static_cast<uint16_t*>(a.out) + to * D + 4 * C * g4);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (C == 8) {
        u32x4_t w;
#pragma unroll
        for (int c = 0; c < 4; ++c) w[c] = pack2(o[(2 * c) % C][i] * f, o[(2 * c + 1) % C][i] * f);
        y[i] = w;
      } else if (i % 2 == 0) {
        y[i / 2] = (u32x4_t){pack2(o[0][i] * f, o[1][i] * f), pack2(o[2][i] * f, o[3][i] * f),
                             pack2(o[0][i + 1] * f, o[1][i + 1] * f), pack2(o[2][i + 1] * f, o[3][i + 1] * f)};
      }
    }
    if (a.lse != nullptr && g4 == 0)
      a.lse[to] = l == 0.0f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.69314718055994530942f;
  }
};
__device__ __forceinline__ Finish finisher(const AttendArgs&, int) { return Finish(); }

// pre[b] = sum of weight(request, number) over requests 0 .. b, by a workgroup of THREADS; part: an entry per wave.
template <int THREADS, typename A, typename W>
__device__ __forceinline__ void prefix_requests(const A& a, int64_t* pre, int64_t* part, W weight) {
  const int tid = threadIdx.x, lane = tid & 63;
  const int chunk = (a.B + THREADS - 1) / THREADS;
  const int b0 = tid * chunk < a.B ? tid * chunk : a.B, b1 = b0 + chunk < a.B ? b0 + chunk : a.B;
  int64_t sum = 0;
  for (int b = b0; b < b1; ++b) sum += weight(request(a, b), b);
  int64_t v = sum;
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) {
    const int64_t u = __shfl_up(v, s, 64);
    if (lane >= s) v += u;
  }
  if (lane == 63) part[tid >> 6] = v;
  __syncthreads();
  for (int w = 0; w < tid >> 6; ++w) v += part[w];
  v -= sum;
  for (int b = b0; b < b1; ++b) {
    v += weight(request(a, b), b);
    pre[b] = v;
  }
  __syncthreads();
}

// First b with pre[b] > x.
__device__ __forceinline__ int find_request(const int64_t* pre, int B, int64_t x) {
  int b = 0;
  for (int left = B; left > 0;) {
    const int half = left >> 1;
    if (pre[b + half] > x) left = half;
    else { b += half + 1; left -= half + 1; }
  }
  return b;
}

// Where a row's sums are that have yet to be joined: in the partial sums of workgroups g0 .. g1,
// row `row` of their slots.
__device__ __forceinline__ uint64_t parts_of(int g0, int g1, int row) {
  return (uint64_t)(uint32_t)(g1 - g0 + 1) << 32 | (uint32_t)g0 << 16 | (uint32_t)row;
}

// True in the workgroup that comes last of `count` at a counter, which is zero again then.
// What its threads wrote with put2 before is out; `last` is a word of LDS.  Relaxed
// operations at agent scope: the stores went past this XCD's L2 and have been waited for.
__device__ __forceinline__ bool arrive(int* counter, int count, int* last) {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (threadIdx.x == 0) {
    const int n = __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    *last = n == count - 1;
    if (*last) __hip_atomic_store(counter, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __syncthreads();
  return *last != 0;
}

}  // namespace
}  // namespace kvx
