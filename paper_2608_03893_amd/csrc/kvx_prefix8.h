// Attention over shared prefixes (device code): what the two parts of a call change in the
// attention kernels.  The common part takes a prefix for a request, whose rows are those of all
// requests that share it and see all of its keys; it leaves every row's sums in fp32, as it has
// them: whole, or in the partial sums of the workgroups that have shared its keys out.  The own
// part goes over each request's own keys and joins all of these, every row by threads of its own:
// one workgroup at the end of the common part, as in attend_cache8, would take as long for one
// block of rows (29 partial sums of 16 rows 9 us) as all of them together take here.
#pragma once

#include "kvx_attend8.h"

namespace kvx {
namespace {

struct CommonPart : PrefixArgs {      // a.B, a.tables, a.lens, a.M: the prefixes'
  static constexpr bool kCausal = false;
  template <int NB>
  static constexpr bool kAhead = NB == 2;      // where a step has work to hide loads behind
  static constexpr bool kJoinLater = true;
};
struct OwnPart : PrefixArgs {        // joins its sums and the common part's
  static constexpr bool kCausal = true;
};
struct OwnLater : PrefixArgs {       // leaves its sums to a kernel that joins both parts'
  static constexpr bool kCausal = true;
  static constexpr bool kJoinLater = true;
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

struct FinishLater {
  template <int DT, int D>
  __device__ __forceinline__ void row(const PrefixArgs& a, int64_t to, int jc, float top, float den, f32x4_t sum) const {
    *reinterpret_cast<f32x4_t*>(a.sums + to * D + jc) = sum;
    if (jc != 0) return;
    *reinterpret_cast<float2*>(a.stats + 2 * to) = make_float2(top, den);
    a.parts[to] = 0;
  }
  template <int D>
  __device__ __forceinline__ void tile(const PrefixArgs& a, int64_t to, int g4, float m, float l, const f32x4_t* o) const {
    constexpr int C = D / 16;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int c = 0; c < C; c += 4)
        *reinterpret_cast<f32x4_t*>(a.sums + to * D + (4 * g4 + i) * C + c) = (f32x4_t){o[c][i], o[c + 1][i], o[c + 2][i], o[c + 3][i]};
    if (g4 != 0) return;
    *reinterpret_cast<float2*>(a.stats + 2 * to) = make_float2(m, l);
    a.parts[to] = 0;
  }
};
__device__ __forceinline__ FinishLater finisher(const CommonPart&, int) { return FinishLater(); }
__device__ __forceinline__ FinishLater finisher(const OwnLater&, int) { return FinishLater(); }

struct FinishOwn {
  int joined;        // the request has a prefix
  // f(values of the row, its statistics) for each of a part's sums of row `to`, which are where
  // `parts` says, FLY of them on the way at a time; at: where a thread's values stand.  Of several
  // threads that share them, thread `share` takes every SHARES-th one.
  template <int D, int FLY, int SHARES = 1, int N, typename F>
  __device__ __forceinline__ static void each_sum(const PrefixArgs& a, int64_t to, uint64_t parts, const int (&at)[N], F f,
                                                  int share = 0) {
    const int count = (int)(parts >> 32 & 0x7fffffff), g0 = (int)(parts >> 16 & 0xffff), row = (int)(parts & 0xffff);
    if (count == 0) {
      if (share != 0) return;
      f32x4_t v[N];
#pragma unroll
      for (int n = 0; n < N; ++n) v[n] = *reinterpret_cast<const f32x4_t*>(a.sums + to * D + at[n]);
      f(v, *reinterpret_cast<const float2*>(a.stats + 2 * to));
      return;
    }
    // (rows that no prefix has, of starts that do not rise, hold anything)
    if (count > prefix_groups(a.slot_rows) - g0 || row >= a.slot_rows) return;
    const int64_t slot = (int64_t)a.slot_rows * (D + 2);
    for (int i0 = share; i0 < count; i0 += FLY * SHARES) {
      f32x4_t v[FLY][N];
      float2 ml[FLY];
#pragma unroll
      for (int i = 0; i < FLY; ++i) {
        const int p = i0 + i * SHARES < count ? i0 + i * SHARES : count - 1;
        const float* from = a.partial + (2 * (g0 + p) + (p == 0 ? 1 : 0)) * slot;
#pragma unroll
        for (int n = 0; n < N; ++n) v[i][n] = *reinterpret_cast<const f32x4_t*>(from + row * D + at[n]);
        ml[i] = *reinterpret_cast<const float2*>(from + a.slot_rows * D + 2 * row);
      }
#pragma unroll
      for (int i = 0; i < FLY; ++i)
        if (i0 + i * SHARES < count) f(v[i], ml[i]);
    }
  }
  // Factors of the sums so far and of further ones, whose statistics are joined.
  struct Both {
    float own, other;
  };
  __device__ __forceinline__ static Both both(float& top, float& den, float2 ml) {
    const float now = fmaxf(top, ml.x), ref = now == -INFINITY ? 0.0f : now;
    const Both x = {__builtin_amdgcn_exp2f(top - ref), __builtin_amdgcn_exp2f(ml.x - ref)};
    den = x.own * den + x.other * ml.y;
    top = now;
    return x;
  }
  template <int DT, int D>
  __device__ __forceinline__ void row(const PrefixArgs& a, int64_t to, int jc, float top, float den, f32x4_t sum) const {
    if (joined) {
      const int at[1] = {jc};
      each_sum<D, 8>(a, to, a.parts[to], at, [&](const f32x4_t (&v)[1], float2 ml) {
        const Both x = both(top, den, ml);
        sum = x.own * sum + x.other * v[0];
      });
    }
    Finish().row<DT, D>(a, to, jc, top, den, sum);
  }
  template <int D>
  __device__ __forceinline__ void tile(const PrefixArgs& a, int64_t to, int g4, float m, float l, f32x4_t* o) const {
    constexpr int C = D / 16, N = C;       // four channels (4 g4 + i) C + c .. in each
    if (joined) {
      int at[N];
#pragma unroll
      for (int n = 0; n < N; ++n) at[n] = (4 * g4 + n / (C / 4)) * C + n % (C / 4) * 4;
      each_sum<D, 1>(a, to, a.parts[to], at, [&](const f32x4_t (&v)[N], float2 ml) {
        const Both x = both(m, l, ml);
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int c = n % (C / 4) * 4 + e, i = n / (C / 4);
            o[c][i] = x.own * o[c][i] + x.other * v[n][e];
          }
      });
    }
    Finish().tile<D>(a, to, g4, m, l, o);
  }
};
__device__ __forceinline__ FinishOwn finisher(const OwnPart& a, int b) {
  return FinishOwn{b >= a.shares[0] && b < a.shares[a.prefixes] ? 1 : 0};
}

}  // namespace
}  // namespace kvx
