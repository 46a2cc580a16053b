// Attention over shared prefixes (device code): what the two parts of a call change in the
// attention kernels.  The common part takes a prefix for a request, whose rows are those of all
// requests that share it and see all of its keys; it leaves every row's sums in fp32.  The own
// part goes over each request's own keys and joins the two.
#pragma once

#include "kvx_attend8.h"

namespace kvx {
namespace {

struct CommonPart : PrefixArgs {      // a.B, a.tables, a.lens, a.M: the prefixes'
  static constexpr bool kCausal = false;
};
struct OwnPart : PrefixArgs {
  static constexpr bool kCausal = true;
};

__device__ __forceinline__ int clamp_to(int v, int most) { return v < 0 ? 0 : v < most ? v : most; }

__device__ __forceinline__ Request request(const CommonPart& a, int s, int len) {
  Request r;
  const int c0 = clamp_to(a.cu[clamp_to(a.shares[s], a.requests)], a.T);
  const int c1 = clamp_to(a.cu[clamp_to(a.shares[s + 1], a.requests)], a.T);
  r.row0 = c0;
  r.tokens = c1 > c0 ? c1 - c0 : 0;
  const int64_t cap = (int64_t)a.M << a.log2p;
  r.len = len < 0 ? 0 : len < cap ? len : (int)cap;
  r.rows = r.tokens * a.G;
  return r;
}
__device__ __forceinline__ Request request(const CommonPart& a, int s) { return request(a, s, a.lens[s]); }
__device__ __forceinline__ int last_key(const CommonPart&, const Request& r, int) { return r.len - 1; }

struct FinishCommon {
  template <int DT, int D>
  __device__ __forceinline__ void row(const PrefixArgs& a, int64_t to, int jc, float top, float den, f32x4_t sum) const {
    *reinterpret_cast<f32x4_t*>(a.sums + to * D + jc) = sum;
    if (jc == 0) *reinterpret_cast<float2*>(a.stats + 2 * to) = make_float2(top, den);
  }
  template <int D>
  __device__ __forceinline__ void tile(const PrefixArgs& a, int64_t to, int g4, float m, float l, const f32x4_t* o) const {
    constexpr int C = D / 16;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int c = 0; c < C; c += 4)
        *reinterpret_cast<f32x4_t*>(a.sums + to * D + (4 * g4 + i) * C + c) = (f32x4_t){o[c][i], o[c + 1][i], o[c + 2][i], o[c + 3][i]};
    if (g4 == 0) *reinterpret_cast<float2*>(a.stats + 2 * to) = make_float2(m, l);
  }
};
__device__ __forceinline__ FinishCommon finisher(const CommonPart&, int) { return FinishCommon(); }

struct FinishOwn {
  int joined;        // the request has a prefix
  // Factors of the prefix's and the own sums, and the statistics of both.
  struct Both {
    float common, own, top, den;
  };
  __device__ __forceinline__ Both both(const PrefixArgs& a, int64_t to, float top, float den) const {
    const float2 ml = *reinterpret_cast<const float2*>(a.stats + 2 * to);
    Both x;
    x.top = fmaxf(top, ml.x);
    const float ref = x.top == -INFINITY ? 0.0f : x.top;
    x.common = __builtin_amdgcn_exp2f(ml.x - ref);
    x.own = __builtin_amdgcn_exp2f(top - ref);
    x.den = x.own * den + x.common * ml.y;
    return x;
  }
  template <int DT, int D>
  __device__ __forceinline__ void row(const PrefixArgs& a, int64_t to, int jc, float top, float den, f32x4_t sum) const {
    if (joined) {
      const Both x = both(a, to, top, den);
      sum = x.own * sum + x.common * *reinterpret_cast<const f32x4_t*>(a.sums + to * D + jc);
      top = x.top;
      den = x.den;
    }
    Finish().row<DT, D>(a, to, jc, top, den, sum);
  }
  template <int D>
  __device__ __forceinline__ void tile(const PrefixArgs& a, int64_t to, int g4, float m, float l, f32x4_t* o) const {
    constexpr int C = D / 16;
    if (joined) {
      const Both x = both(a, to, m, l);
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int c = 0; c < C; c += 4) {
          const f32x4_t y = *reinterpret_cast<const f32x4_t*>(a.sums + to * D + (4 * g4 + i) * C + c);
#pragma unroll
          for (int e = 0; e < 4; ++e) o[c + e][i] = x.own * o[c + e][i] + x.common * y[e];
        }
      m = x.top;
      l = x.den;
    }
    Finish().tile<D>(a, to, g4, m, l, o);
  }
};
__device__ __forceinline__ FinishOwn finisher(const OwnPart& a, int b) {
  return FinishOwn{b >= a.shares[0] && b < a.shares[a.prefixes] ? 1 : 0};
}

}  // namespace
}  // namespace kvx
