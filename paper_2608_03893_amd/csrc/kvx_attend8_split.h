// Attention over the 8-bit pool, split over the keys: the kernel's body, for whole requests
// (kvx_attend8.hip) and for the parts of requests that share prefixes (kvx_prefix8_common.hip, _own.hip, _both.hip).
//
// For a block of 16 query rows (tokens times the G heads of a KV head) and a tile of
// 16 keys the scores are S^T = K Q^T on the matrix cores: a lane then holds one query
// row's scores for 4 keys, so the softmax needs no exchange but the maximum over four
// lanes, and P^T has the layout that O^T = V^T P^T takes as its second operand.  e4m3
// codes are bf16 numbers, so K and V enter exactly; a page's scales multiply the scores
// and the probabilities.  fp32 queries and their probabilities enter as three bf16 terms, which
// hold all 24 bits, the probabilities of bf16 queries as two.
//
// Bound by the bytes of K and V, which go from memory straight to registers, each once:
// a lane reads 16 bytes of one key's row, or 8 bytes of 8 value rows whose bytes it then
// pairs up for V^T.
//
// The grid fills the chip once and every workgroup takes an equal share of the weight of
// all units (request, head, row block), whatever the lengths: a quantum of 32 keys a wave
// weighs one and a unit's start two.  It finds its share from a prefix sum over the
// requests.  A unit whose keys span workgroups is joined by the workgroup that comes last,
// from partial sums in order of the keys, so results do not depend on timing.
//
// Measured, d = 128, G = 8, 8 KV heads, 16-token pages that no cache holds: 32 requests of
// 5000 keys 64 us (5.1 TB/s), 16 of 2178 24 us (3.0), 1 of 5000 14.1 us, 1 of 300 8.7 us:
// a launch, the lengths, pages, keys and joins, each of which waits for the one before, take
// 8 to 12 us, and the bytes come on top.
#pragma once

#include "kvx_attend8.h"

#include <cstdio>

namespace kvx {
namespace {

constexpr int kStep = 32;                  // keys of a wave's step
template <int W>
constexpr int kLeast = W > 4 ? 1 : 2;      // least quanta of a workgroup
constexpr int kStart = 2;                  // weight of a unit's start, in quanta
constexpr int kSmall = 10;                 // a unit is not split if it weighs no more than this
constexpr int kSplit = 5;                  // and than a share and what a join costs
constexpr int kJoin = 64;                  // most partial sums joined at a time
template <int D, int NB>
constexpr int kFlying = NB == 2 ? 8 : D == 64 ? 10 : 12;  // of which a thread has these in flight
// Waves a SIMD: as many as the registers hold.  More of them hide more of a unit's start
// (lengths, pages, scales, rows: loads that wait for one another) than prefetching
// within a wave: 64 ragged requests 86 us with two and the next step's loads in flight,
// 72 us with three and no prefetch; three and the next step's keys in flight, 124 -> 132 us
// at 64 requests of up to 8191 keys.  d = 64: 128 requests of 1000 keys 37 us with three,
// 32 with four.
template <int DT, int D, int NB>
constexpr int kOcc = D == 64 ? 5 - NB : DT == 1 ? 2 : 4 - NB;
template <int DT, int D, int NB>
constexpr int kLarge = kOcc<DT, D, NB> > 2 ? 12 : 8;   // waves of a large workgroup

// Blocks of rows, and quanta (of `quant` keys) of one block and head (rows without any key
// still have an output).
template <int R>
__device__ __forceinline__ int blocks_of(const Request& r) { return (r.rows + R - 1) / R; }
__device__ __forceinline__ int quanta_of(int len, int quant) {
  return len > quant ? (int)(((uint32_t)len + quant - 1) / quant) : 1;
}
__device__ __forceinline__ int quanta_of(const Request& r, int quant) { return quanta_of(r.len, quant); }

// A step's keys and values, as loaded.
template <int D>
struct Stage {
  static constexpr int U = D / 64, V = D / 64;
  uint4 k[2][U];            // tile t: row lane & 15, bytes 64 u + 16 (lane >> 4) ..
  uint32_t v[8][V];         // key (lane >> 4) * 4 + (j & 3) of tile j >> 2, bytes (lane & 15) * 4 V ..
};

template <int D, int W, int NB>
struct SplitLds {
  int64_t part[W];
  __attribute__((aligned(16))) float jo[W][16 * NB * (D + 4)];
  float jm[W][16 * NB], jl[W][16 * NB];
  int last;
};

// The workgroups of a call, or of a part of one.
struct Group {
  int block, grid;
};

// Request b's weight.
template <int W, int NB, typename A>
__device__ __forceinline__ int64_t weight_of(const A& a, const Request& r) {
  return (int64_t)blocks_of<16 * NB>(r) * (quanta_of(r, W * kStep) + kStart) * a.H;
}

// W waves: 4, and kOcc workgroups a CU; or kLarge, and one.
template <int DT, int D, int W, int NB, typename A>
__device__ __forceinline__ void attend8_split(const A& a, float* partial, int* counters, SplitLds<D, W, NB>& lds, Group group) {
  constexpr int kFly = kFlying<D, NB>;
  constexpr int kWaves = W, kThreads = 64 * W, kQuant = W * kStep, kRows = 16 * NB;
  constexpr int U = D / 64, TERMS = DT == 0 ? 1 : 3, PT = kTerms<DT>;    // terms of queries, probabilities
  constexpr int C = D / 16;                                        // channel tiles
  static_assert(kJoin % 16 == 0 && kJoin * kRows <= kRows * (D + 4), "weights of a join fit one wave's sums");
  constexpr int RS = D + 4;                                        // row stride in LDS
  constexpr int SLOT = kRows * (D + 2);                            // floats of a partial sum
  extern __shared__ int64_t pre[];                                 // [B] quanta of requests 0 .. b
  auto& part = lds.part;
  auto& jo = lds.jo;
  auto &jm = lds.jm, &jl = lds.jl;
  int& last = lds.last;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int n = lane & 15, g4 = lane >> 4;

  int32_t* weight = reinterpret_cast<int32_t*>(pre + a.B);         // [B] of a unit
  // Up to 64 requests: every wave has them in its lanes, and neither LDS nor barriers come
  // before its first loads (three requests of 100 to 250 keys 6.9 -> 6.4 us).
  uint32_t pre_lane = 0;
  int len_lane = 0;
  int64_t total = 0;
  bool lanes = a.B <= 64;
  if (lanes) {
    const Request r = request(a, lane < a.B ? lane : a.B - 1);
    len_lane = r.len;
    const int64_t w = lane < a.B ? weight_of<W, NB>(a, r) : 0;
    pre_lane = w < UINT32_MAX ? (uint32_t)w : UINT32_MAX;
#pragma unroll
    for (int n = 1; n < 64; n <<= 1) {
      const uint32_t x = __shfl_up(pre_lane, n, 64);
      if (lane >= n) pre_lane = __builtin_elementwise_add_sat(pre_lane, x);
    }
    total = (uint32_t)__builtin_amdgcn_readlane(pre_lane, 63);
    lanes = total < UINT32_MAX;        // else the sums may not fit
  }
  if (!lanes) {
    prefix_requests<kThreads>(a, pre, part, [&](const Request& r, int b) {
      weight[b] = quanta_of(r, kQuant) + kStart;
      return (int64_t)blocks_of<kRows>(r) * weight[b] * a.H;
    });
    total = uniform(pre[a.B - 1]);
  }
  // the request that has weight x, the weight before it, its units' weight
  auto find = [&](int64_t x) {
    return lanes ? __builtin_ctzll(__ballot(pre_lane > (uint32_t)x)) : uniform(find_request(pre, a.B, x));
  };
  auto before = [&](int b) {
    return b == 0 ? (int64_t)0
           : lanes ? (int64_t)(uint32_t)__builtin_amdgcn_readlane(pre_lane, b - 1) : uniform(pre[b - 1]);
  };
  auto length = [&](int b) { return __builtin_amdgcn_readlane(len_lane, b); };
  const int grid = group.grid;
  const int64_t share_q = uniform(divide(total + grid - 1, grid));
  const int64_t per = share_q > kLeast<W> ? share_q : kLeast<W>;
  const int small = per + kSplit < kSmall ? (int)per + kSplit : kSmall;
  auto share_of = [&](int64_t q) { return (int)divide(q, per); };
  // A share ends where its weight does, or at the nearer end of the unit there if that is
  // small: to split it would cost more, in its second start and the join, than it levels.
  auto share_end = [&](int64_t x) {
    if (x >= total) return total;
    const int b = find(x);
    const int64_t in_request = x - before(b), w = lanes ? quanta_of(length(b), kQuant) + kStart : weight[b];
    if (w > small) return x;
    const int64_t in_unit = in_request - divide(in_request, w) * w;
    return 2 * in_unit < w ? x - in_unit : x - in_unit + w;
  };
  const int me = xcd_order(group.block, grid);
  int64_t at = uniform(share_end(me * per));
  const int64_t end = uniform(share_end((me + 1) * per));
  if (at >= end) return;

  const int64_t plane = ((int64_t)a.N << a.log2p) * D;
  const int P1 = (1 << a.log2p) - 1;
  while (at < end) {
    const int b = find(at);
    const int64_t base = before(b);
    const Request r = lanes ? request(a, b, length(b)) : request(a, b);
    const int quanta = quanta_of(r, kQuant);
    const int64_t unit = divide(at - base, quanta + kStart);
    const int64_t unit0 = base + unit * (quanta + kStart);     // its first weight
    const int blocks = blocks_of<kRows>(r);       // of a head, which share its keys: on one XCD mostly
    const int h = uniform((int)divide(unit, blocks)), blk = uniform((int)(unit - (int64_t)h * blocks));
    const int64_t lo = at - unit0 - kStart, hi = end - unit0 - kStart;
    const int q0 = uniform(lo < 0 ? 0 : (int)lo), q1 = uniform(hi < quanta ? (int)hi : quanta);
    if (q0 >= q1) {      // only its start
      at = unit0 + kStart + quanta < end ? unit0 + kStart + quanta : end;
      continue;
    }

    // this lane's query row (the block's last one again past the end): its keys' limit, its
    // channels
    const int block_last = (blk + 1) * kRows < r.rows ? (blk + 1) * kRows - 1 : r.rows - 1;
    int lim[NB];                                                           // last key a row sees
    const int lim_lo = uniform(last_key(a, r, blk * kRows / a.G));         // least and largest
    const int lim_hi = uniform(last_key(a, r, block_last / a.G));          // of the block
    bf16x8_t qf[NB][2 * U][TERMS];
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      const int at_row = blk * kRows + 16 * i + n, row = at_row < block_last ? at_row : block_last;
      const int token = row / a.G, head = h * a.G + row % a.G;
      lim[i] = last_key(a, r, token);
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          const int64_t off = (int64_t)(r.row0 + token) * a.q_stride[0] + (int64_t)head * a.q_stride[1] +
                              64 * u + 16 * g4 + 8 * w;
          if (DT == 0) {
            qf[i][2 * u + w][0] = as_bf16x8(*reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.q) + off));
          } else {
            const float4 lo = *reinterpret_cast<const float4*>(static_cast<const float*>(a.q) + off);
            const float4 hi = *reinterpret_cast<const float4*>(static_cast<const float*>(a.q) + off + 4);
            const float x[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
            split_terms<TERMS>(x, qf[i][2 * u + w]);
          }
        }
    }

    const uint8_t* kc = a.codes + h * plane;
    const uint8_t* vc = a.codes + (a.H + h) * plane;
    const uint32_t k_lane = (uint32_t)n * D + 16 * g4, v_lane = (uint32_t)g4 * 4 * D + n * (D / 16);
    float m[NB], l[NB];
    f32x4_t o[NB][C];
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      m[i] = -INFINITY;
      l[i] = 0.0f;
#pragma unroll
      for (int c = 0; c < C; ++c) o[i][c] = (f32x4_t){0, 0, 0, 0};
    }

    // pages of this wave's next 32 steps: lane 2 s + t has tile t of step s
    for (int qa = q0; qa < q1; qa += 32) {
      const int qb = qa + 32 < q1 ? qa + 32 : q1;
      int page = -1;
      {
        const int64_t key = (int64_t)(qa + (lane >> 1)) * kQuant + wave * kStep + (lane & 1) * 16;
        if (key < r.len) page = a.tables[(int64_t)b * a.M + (key >> a.log2p)];
        if (page >= a.N) page = -1;
      }
      float ksc = 0.0f, vsc = 0.0f;
      if (page >= 0) {
        ksc = a.scales[(int64_t)h * a.N + page] * a.scale_log2;
        vsc = a.scales[(int64_t)(a.H + h) * a.N + page];
      }
      auto load = [&](Stage<D>& s, int q, bool keys, bool values) {
        const int key = q * kQuant + wave * kStep;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          int p = __builtin_amdgcn_readlane(page, 2 * (q - qa) + t);
          p = p < 0 ? 0 : p;
          const int64_t off = (((int64_t)p << a.log2p) + ((key + 16 * t) & P1)) * D;
          const uint8_t* kp = kc + off;
          const uint8_t* vp = vc + off;
          if (keys)
#pragma unroll
            for (int u = 0; u < U; ++u) s.k[t][u] = *reinterpret_cast<const uint4*>(kp + k_lane + 64 * u);
          if (!values) continue;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            if (D == 128) {
              const uint2 x = *reinterpret_cast<const uint2*>(vp + v_lane + j * D);
              s.v[4 * t + j][0] = x.x;
              s.v[4 * t + j][U - 1] = x.y;
            } else {
              s.v[4 * t + j][0] = *reinterpret_cast<const uint32_t*>(vp + v_lane + j * D);
            }
          }
        }
      };
      // then(): once the keys are in the scores
      auto compute = [&](Stage<D>& s, int q, auto then) {
        const int key = q * kQuant + wave * kStep;
        float x[NB][8];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          f32x4_t acc[NB];
#pragma unroll
          for (int i = 0; i < NB; ++i) acc[i] = (f32x4_t){0, 0, 0, 0};
#pragma unroll
          for (int u = 0; u < U; ++u) {
            const bf16x8_t k0 = bf16_octet(s.k[t][u].x, s.k[t][u].y), k1 = bf16_octet(s.k[t][u].z, s.k[t][u].w);
#pragma unroll
            for (int i = 0; i < NB; ++i)
#pragma unroll
              for (int e = 0; e < TERMS; ++e) {
                acc[i] = mfma(k0, qf[i][2 * u][e], acc[i]);
                acc[i] = mfma(k1, qf[i][2 * u + 1][e], acc[i]);
              }
          }
          const float sc = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(ksc), 2 * (q - qa) + t));
#pragma unroll
          for (int i = 0; i < NB; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) x[i][4 * t + e] = acc[i][e] * sc;
        }
        then();
        const int p0 = __builtin_amdgcn_readlane(page, 2 * (q - qa));
        const int p1 = __builtin_amdgcn_readlane(page, 2 * (q - qa) + 1);
        float v0 = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(vsc), 2 * (q - qa)));
        float v1 = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(vsc), 2 * (q - qa) + 1));
        if (p0 < 0 || p1 < 0 || key + kStep - 1 > lim_lo) {
          // values under a scale that is infinite or NaN are NaN
          const bool lost[2] = {!finite(v0), !finite(v1)};
          v0 = lost[0] ? 1.0f : v0;
          v1 = lost[1] ? 1.0f : v1;
          bool nan = false;
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            const int first = key + 16 * t + 4 * g4;      // this lane's first key; real, seen: its last
            const int real = (t ? p1 : p0) < 0 ? -1 : r.len - 1 - first;
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
              for (int w = 0; w < U; ++w) {
                if (lost[t]) s.v[4 * t + e][w] = kNan4;
                s.v[4 * t + e][w] = e > real ? 0 : s.v[4 * t + e][w];     // nobody's codes
                nan |= e4m3_nan(s.v[4 * t + e][w]) != 0;
              }
#pragma unroll
            for (int i = 0; i < NB; ++i) {
              const int seen = (t ? p1 : p0) < 0 ? -1 : lim[i] - first;
#pragma unroll
              for (int e = 0; e < 4; ++e) x[i][4 * t + e] = e > seen ? -INFINITY : x[i][4 * t + e];
            }
          }
          if (__any(nan)) {
            // NaN values count only in rows that see their key: they leave the product, and
            // go into the sums of the rows for which a product of marks finds one
#pragma unroll
            for (int i = 0; i < NB; ++i) {
              u32x4_t m8;
#pragma unroll
              for (int j = 0; j < 4; ++j)
                m8[j] = (x[i][2 * j] == -INFINITY ? 0u : 0x3f80u) | (x[i][2 * j + 1] == -INFINITY ? 0u : 0x3f800000u);
              const bf16x8_t sees = __builtin_bit_cast(bf16x8_t, m8);
#pragma unroll
              for (int w = 0; w < U; ++w)
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                  u32x4_t hit;
#pragma unroll
                  for (int j = 0; j < 4; ++j)
                    hit[j] = (e4m3_nan(s.v[2 * j][w]) >> (8 * c + 7) & 1) * 0x3f80u |
                             (e4m3_nan(s.v[2 * j + 1][w]) >> (8 * c + 7) & 1) * 0x3f800000u;
                  const f32x4_t count = mfma(__builtin_bit_cast(bf16x8_t, hit), sees, (f32x4_t){0, 0, 0, 0});
#pragma unroll
                  for (int e = 0; e < 4; ++e)
                    o[i][4 * w + c][e] = count[e] != 0.0f ? __builtin_nanf("") : o[i][4 * w + c][e];
                }
            }
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
              for (int w = 0; w < U; ++w) s.v[j][w] &= ~((e4m3_nan(s.v[j][w]) >> 7) * 0xffu);
          }
        }
        // The reference of the exponentials follows the maximum only when that has
        // grown by 2^8: the sums hold that, no lane has to ask the others in most
        // steps, and O is seldom rescaled.
        float top[NB];
        bool grown = false;
#pragma unroll
        for (int i = 0; i < NB; ++i) {
          top[i] = x[i][0];
#pragma unroll
          for (int j = 1; j < 8; ++j) top[i] = fmaxf(top[i], x[i][j]);
          grown |= top[i] > m[i] + kLazy;
        }
        if (__any(grown)) {
#pragma unroll
          for (int i = 0; i < NB; ++i) {
            const float now = fmaxf(m[i], quad_max(top[i]));
            const float keep = now == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m[i] - now);
            m[i] = now;
            l[i] *= keep;
#pragma unroll
            for (int c = 0; c < C; ++c) o[i][c] *= keep;
          }
        }
        bf16x8_t pf[NB][PT];
#pragma unroll
        for (int i = 0; i < NB; ++i) {
          const float ref = m[i] == -INFINITY ? 0.0f : m[i];
          float p[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            p[j] = __builtin_amdgcn_exp2f(x[i][j] - ref);
            l[i] += p[j];
          }
#pragma unroll
          for (int j = 0; j < 8; ++j) p[j] *= j < 4 ? v0 : v1;
          split_terms<PT>(p, pf[i]);
        }
#pragma unroll
        for (int w = 0; w < U; ++w) {
          uint32_t y[4][2];   // pairs of keys: bytes (c, c), (c + 1, c + 1) | the next two channels
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            y[j][0] = __builtin_amdgcn_perm(s.v[2 * j + 1][w], s.v[2 * j][w], 0x05010400u);
            y[j][1] = __builtin_amdgcn_perm(s.v[2 * j + 1][w], s.v[2 * j][w], 0x07030602u);
          }
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            u32x4_t f;
#pragma unroll
            for (int j = 0; j < 4; ++j)
              f[j] = c & 1 ? bf16_pair<true>(y[j][c >> 1]) : bf16_pair<false>(y[j][c >> 1]);
#pragma unroll
            for (int i = 0; i < NB; ++i)
#pragma unroll
              for (int e = 0; e < PT; ++e)
                o[i][4 * w + c] = mfma(__builtin_bit_cast(bf16x8_t, f), pf[i][e], o[i][4 * w + c]);
          }
        }
      };
      // this wave's steps with a key that some row sees
      const int64_t room = (int64_t)lim_hi - wave * kStep;
      int qe = room < 0 ? qa : (int)(room / kQuant) + 1;
      qe = qe < qb ? qe : qb;
      if constexpr (A::template kAhead<NB>) {
        // the next step's keys on the way behind the scores, in the registers of this one's
        Stage<D> s;
        if (qa < qe) load(s, qa, true, false);
        for (int q = qa; q < qe; ++q) {
          load(s, q, false, true);
          compute(s, q, [&] {
            if (q + 1 < qe) load(s, q + 1, true, false);
          });
        }
      } else {
        for (int q = qa; q < qe; ++q) {
          Stage<D> s;
          load(s, q, true, true);
          compute(s, q, [] {});
        }
      }
    }

    // the waves' sums: lane (n, g4) has of row 16 i + n the channels (4 g4 + e) C + c
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      const float sum16 = quad_sum(l[i]);
      if (g4 == 0) {
        jm[wave][16 * i + n] = m[i];
        jl[wave][16 * i + n] = sum16;
      }
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int c = 0; c < C; c += 4)
          *reinterpret_cast<f32x4_t*>(&jo[wave][(16 * i + n) * RS + (4 * g4 + e) * C + c]) =
              (f32x4_t){o[i][c][e], o[i][c + 1][e], o[i][c + 2][e], o[i][c + 3][e]};
    }
    __syncthreads();
    // thread = (row, 4 channels) from here on, IT of them kThreads / Q rows apart (its number
    // again, opaquely: what depends on it would be held in registers through the loop above)
    int at_thread = tid;
    asm volatile("" : "+v"(at_thread));
    constexpr int Q = D / 4, STRIDE = kThreads / Q, IT = (kRows + STRIDE - 1) / STRIDE;
    const int valid = block_last - blk * kRows + 1;                // rows of the block
    const int jr = at_thread / Q, jc = at_thread % Q * 4;
    float top[IT], den[IT];
    f32x4_t sum[IT];
#pragma unroll
    for (int x = 0; x < IT; ++x) {
      const int at_row = jr + x * STRIDE;
      top[x] = -INFINITY;
      den[x] = 0.0f;
      sum[x] = (f32x4_t){0, 0, 0, 0};
      if (at_row >= valid) continue;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) top[x] = fmaxf(top[x], jm[w][at_row]);
      const float ref = top[x] == -INFINITY ? 0.0f : top[x];
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float f = __builtin_amdgcn_exp2f(jm[w][at_row] - ref);   // 0 for a wave that saw nothing; NaN sums stay
        den[x] += f * jl[w][at_row];
        sum[x] += f * *reinterpret_cast<const f32x4_t*>(&jo[w][at_row * RS + jc]);
      }
    }
    // workgroups that share this unit: g0 .. g1, this one's part is number `mine_at`; small
    // units have one
    const int g0 = share_of(unit0 + kStart), g1 = share_of(unit0 + kStart + quanta - 1);
    bool done = g0 == g1 || quanta + kStart <= small;
    if constexpr (A::kJoinLater) {
      if (!done) {
        const int mine_at = uniform(me - g0);
        float* to = partial + (int64_t)(2 * me + (mine_at == 0 ? 1 : 0)) * SLOT;
#pragma unroll
        for (int x = 0; x < IT; ++x) {
          const int at_row = jr + x * STRIDE, out_row = blk * kRows + at_row;
          if (at_row >= valid) break;
          *reinterpret_cast<f32x4_t*>(to + at_row * D + jc) = sum[x];
          if (jc != 0) continue;
          *reinterpret_cast<float2*>(to + kRows * D + 2 * at_row) = make_float2(top[x], den[x]);
          if (mine_at == 0)
            a.parts[(int64_t)(r.row0 + out_row / a.G) * a.H * a.G + h * a.G + out_row % a.G] = parts_of(g0, g1, at_row);
        }
      }
    } else if (!done) {
      const int parts = uniform(g1 - g0) + 1, mine_at = uniform(me - g0);
      auto slot = [&](int i) { return 2 * (g0 + i) + (i == 0 ? 1 : 0); };
      // Partial sums pass between workgroups on different XCDs, each with its own L2: they
      // are written through and read past it (agent scope), which spares the write-back
      // of the whole L2 that a fence at that scope costs.
      auto put = [&](int i) {
        float* to = partial + (int64_t)slot(i) * SLOT;
#pragma unroll
        for (int x = 0; x < IT; ++x) {
          const int at_row = jr + x * STRIDE;
          if (at_row >= valid) break;
          put2(to + at_row * D + jc, sum[x][0], sum[x][1]);
          put2(to + at_row * D + jc + 2, sum[x][2], sum[x][3]);
          if (jc == 0) put2(to + kRows * D + 2 * at_row, top[x], den[x]);
        }
      };
      // Joins `count` partial sums first, first + stride, ..: the parts' weights, and kFly
      // parts of a thread's channels in flight at a time, the first with the weights.
      // With few rows the threads share the parts of a row.
      auto join = [&](int first, int stride, int count) {
        float* weight = &jo[0][0];                                 // [kJoin][kRows]
        f32x4_t* across = reinterpret_cast<f32x4_t*>(&jo[1][0]);   // [kThreads]
        const int items = valid * Q, shares = kThreads / items > 1 ? kThreads / items : 1;
        int share = 0, item = at_thread;
        if (shares > 1) {
          share = at_thread / items;
          item = at_thread - share * items;
        }
        const int at_row = item / Q < valid ? item / Q : 0;       // idle threads read a row too
        const float* from = partial + at_row * D + item % Q * 4;
        float2 v[kFly][2];
        auto fly = [&](int i0, int more) {
#pragma unroll
          for (int i = 0; i < kFly; ++i) {
            const int at_i = i0 + i * shares < count ? i0 + i * shares : count - 1;
            const uint32_t off = (uint32_t)slot(first + at_i * stride) * SLOT + more;
            v[i][0] = get2(from + off);
            v[i][1] = get2(from + off + 2);
          }
        };
        auto add = [&](f32x4_t& to, int i0, int row) {
#pragma unroll
          for (int i = 0; i < kFly; ++i) {
            const float f = i0 + i * shares < count ? weight[(i0 + i * shares) * kRows + row] : 0.0f;
            to += f * (f32x4_t){v[i][0].x, v[i][0].y, v[i][1].x, v[i][1].y};
          }
        };
        fly(share, 0);
        __syncthreads();                                 // jo, jm and jl have been read
        for (int row = at_thread >> 4; row < kRows; row += kThreads / 16) {   // 16 lanes a row
          const int sub = at_thread & 15;
          float2 md[kJoin / 16];
          float most = -INFINITY, l16 = 0.0f;
#pragma unroll
          for (int i = 0; i < kJoin / 16; ++i) {
            const int at_i = sub + 16 * i < count ? sub + 16 * i : count - 1;
            md[i] = get2(partial + (uint32_t)slot(first + at_i * stride) * SLOT + kRows * D + 2 * (row < valid ? row : 0));
            if (sub + 16 * i >= count) md[i] = make_float2(-INFINITY, 0.0f);
          }
#pragma unroll
          for (int i = 0; i < kJoin / 16; ++i) most = fmaxf(most, md[i].x);
#pragma unroll
          for (int n16 = 8; n16; n16 >>= 1) most = fmaxf(most, __shfl_xor(most, n16, 64));
          const float ref = most == -INFINITY ? 0.0f : most;
#pragma unroll
          for (int i = 0; i < kJoin / 16; ++i) {
            const float f = __builtin_amdgcn_exp2f(md[i].x - ref);
            l16 += f * md[i].y;
            weight[(sub + 16 * i) * kRows + row] = f;
          }
#pragma unroll
          for (int n16 = 8; n16; n16 >>= 1) l16 += __shfl_xor(l16, n16, 64);
          if (sub == 0) {
            jm[0][row] = most;
            jl[0][row] = l16;
          }
        }
        __syncthreads();
#pragma unroll
        for (int x = 0; x < IT; ++x) sum[x] = (f32x4_t){0, 0, 0, 0};
        if (share < shares) {
          add(sum[0], share, at_row);
          for (int i0 = share + kFly * shares; i0 < count; i0 += kFly * shares) {
            fly(i0, 0);
            add(sum[0], i0, at_row);
          }
        }
#pragma unroll
        for (int x = 1; x < IT; ++x)                      // shares == 1 where there are such rows
          if (jr + x * STRIDE < valid)
            for (int i0 = 0; i0 < count; i0 += kFly) {
              fly(i0, x * STRIDE * D);
              add(sum[x], i0, jr + x * STRIDE);
            }
        if (shares > 1) {
          if (share < shares) across[at_thread] = sum[0];
          __syncthreads();
          if (at_thread < items)
            for (int i = 1; i < shares; ++i) sum[0] += across[i * items + at_thread];
        }
#pragma unroll
        for (int x = 0; x < IT; ++x) {
          if (jr + x * STRIDE >= valid) break;
          top[x] = jm[0][jr + x * STRIDE];
          den[x] = jl[0][jr + x * STRIDE];
        }
      };
      put(mine_at);
      // Many partial sums are joined in two levels, by groups side by side, where one workgroup
      // would read 128 KB or more (16 rows of 16000 keys 29 -> 22 us; one row 12 against 15).
      int width = uniform(parts);
      if (width > kJoin || (width > kJoin / 2 && width * uniform(valid) * D > 32768))
        for (width = 6; width * width < parts; ++width) {}
      const int group = mine_at / width, groups = (parts + width - 1) / width;
      const int in_group = parts - group * width < width ? parts - group * width : width;
      if (arrive(counters + 2 * slot(group * width), in_group, &last)) {
        join(group * width, 1, in_group);
        done = groups == 1;
        if (!done) {
          __syncthreads();       // all have read the partial sums that put overwrites
          put(group * width);
          if (arrive(counters + 2 * slot(0) + 1, groups, &last)) {
            join(0, width, groups);
            done = true;
          }
        }
      }
    }
    if (done) {
      const auto finish = finisher(a, b);
#pragma unroll
      for (int x = 0; x < IT; ++x) {
        const int at_row = jr + x * STRIDE, out_row = blk * kRows + at_row;
        if (at_row >= valid) break;
        const int64_t to = (int64_t)(r.row0 + out_row / a.G) * a.H * a.G + h * a.G + out_row % a.G;
        finish.template row<DT, D>(a, to, jc, top[x], den[x], sum[x]);
      }
    }
    __syncthreads();    // the LDS arrays are free again
    at = unit0 + kStart + q1;
  }
}

// Which kernel: by what the host knows, rows, requests and a bound of the longest one (the
// tables' length if the caller states none).  Measured, us, with 8 KV heads, pages that no
// cache holds, B requests of `rows` query rows a head over `keys` keys.

// By rows (bf16 only): blocks of 256 rows share the widened codes.  Pays from 96 rows a
// request on where blocks are enough for the CUs or the work is, else its joins cost more.
//   d = 128, split / by rows    B = 64, 64 rows, 1000 keys 57 / 77    96 rows 79 / 78
//     B = 32, 128 rows, 300 keys 27 / 21     B = 16, 160 rows, 5000 keys 152 / 128
//     B = 8,  256 rows, 5000 keys 88 / 98, 16000 keys 262 / 224
//     B = 1,  2048 rows, 2178 keys 39 / 65, 16000 keys 226 / 198
//   d = 64   B = 64, 64 rows, 1000 keys 38 / 55    128 rows 61 / 56
bool may_go_by_rows(int B, int G, int T, int dtype) { return dtype == 0 && (int64_t)T * G >= (int64_t)B * 96; }
bool by_rows(const AttendArgs& a, int dtype, int d) {
  const int64_t rows = (int64_t)a.T * a.G, units = (rows / 256 > a.B ? rows / 256 : a.B) * a.H;
  const double work = (double)rows * a.H * a.keys * d;
  return may_go_by_rows(a.B, a.G, a.T, dtype) && (units >= 192 || work >= (units >= 128 ? 8589934592.0 : 17179869184.0));
}

// Blocks of 32 rows (bf16 only), whose codes are loaded and widened once for two row tiles,
// where a request brings more than one tile and the blocks' keys come to 512 a CU:
//   d = 128, 16 / 32 rows a block    B = 64, 32 rows, 1000 keys 48 / 34, 5000 keys 246 / 128
//     B = 8, 128 rows, 5000 keys 82 / 51     B = 2, 24 rows, 1000 keys 13 / 16
//   d = 64   B = 32, 32 rows, 5000 keys 62 / 41
bool two_tiles(const AttendArgs& a, int dtype) {
  const int64_t rows = (int64_t)a.T * a.G, blocks = rows / 32 > a.B ? rows / 32 : a.B;
  return dtype == 0 && rows > 16 * (int64_t)a.B && (double)blocks * a.H * a.keys >= 256 * 512;
}

// One large workgroup a CU instead of several of four waves: a unit then has fewer partial
// sums or none.
//   Blocks of 32 rows: fewer than two units a CU of 1024 keys and more (32 requests of 24 rows
//   and 2178 keys 44 -> 34, d = 64 33 -> 23; but 64 of 1000 32 against 37, 1560 rows of one over
//   1000 23 against 28).
//   Blocks of 16: where the units' keys come to 256 a CU (a decoding step of 32 requests of
//   2178 keys 42 -> 32, 16 of 1000 20 -> 15, 4 contexts up to 131070 101 -> 95), but not
//   - for few units of one to three rows, whose sums join fast, until their keys come to
//     2048 a CU (G = 1, 16000 keys 18 against 20);
//   - for two units a CU and more of requests of more than 32 rows (fp32: 8 requests of 128 rows
//     and 1000 keys 23 against 27, 2048 rows of one over 10240, d = 64, 141 against 157; with
//     fewer units 8 of 64 rows and 1000 keys 22 -> 17, 512 rows over 304 12.5 -> 10.1), or of
//     few keys, where starts and ends of small workgroups overlap (256 requests of 300 keys 45
//     against 66, of 1000 111 against 118, of 2178 233 -> 225), or with eight waves (fp32,
//     d = 128: 256 requests of 1000 keys 113 against 130).
template <int NB, int LARGE>
bool large_workgroups(const AttendArgs& a) {
  const int64_t rows = (int64_t)a.T * a.G, B = a.B, blocks = rows / (16 * NB) > B ? rows / (16 * NB) : B;
  const int64_t units = blocks * a.H, keys = a.keys;
  if (NB == 2) return units < 512 && keys >= 1024;
  const double least = units < 64 && rows < 4 * B ? 256 * 2048 : 256 * 256;
  return (double)units * keys >= least && (units < 512 || (rows <= 32 * B && LARGE >= 12 && keys > 1024));
}

// Workgroups that there can be quanta for; a grid: no more than that or than fill the chip; dynamic
// LDS.
template <int W, int NB>
double split_want(const AttendArgs& a) {
  const double units = ((double)a.T * a.G / (16 * NB) + a.B) * a.H, quant = W * kStep;
  return units * (a.keys / quant + 1 + kStart) / kLeast<W> + 1;
}
template <int DT, int D, int W, int NB>
unsigned split_grid(double want) {
  constexpr int kFill = W > 4 ? 256 : 256 * kOcc<DT, D, NB>;
  return ((want < kFill ? (unsigned)want : kFill) + kXcds - 1) / kXcds * kXcds;
}
template <int DT, int D, int W, int NB>
unsigned split_grid(const AttendArgs& a) { return split_grid<DT, D, W, NB>(split_want<W, NB>(a)); }
inline size_t split_lds(const AttendArgs& a) { return (size_t)a.B * (sizeof(int64_t) + sizeof(int32_t)); }

// f of the kernel for these sizes.
// A kernel's name, as a trace shows it; a static string.
template <typename K>
const char* name_of(K) {
  struct Name {
    char text[64];
    Name() { K::name(text, sizeof(text)); }
  };
  static const Name name;
  return name.text;
}
// Split, Rows: the kernels of the caller.
template <template <int, int, int, int> class Split, int DT, int D, int NB, typename F>
auto with_split(const AttendArgs& a, F f) {
  constexpr int LARGE = kLarge<DT, D, NB>;
  return large_workgroups<NB, LARGE>(a) ? f(Split<DT, D, LARGE, NB>()) : f(Split<DT, D, 4, NB>());
}
template <template <int, int, int, int> class Split, template <int> class Rows, typename F>
auto with_kernel(const AttendArgs& a, int dtype, int d, bool rows, F f) {
  if (rows) return d == 64 ? f(Rows<64>()) : f(Rows<128>());
  if (two_tiles(a, dtype)) return d == 64 ? with_split<Split, 0, 64, 2>(a, f) : with_split<Split, 0, 128, 2>(a, f);
  if (dtype == 0) return d == 64 ? with_split<Split, 0, 64, 1>(a, f) : with_split<Split, 0, 128, 1>(a, f);
  return d == 64 ? with_split<Split, 1, 64, 1>(a, f) : with_split<Split, 1, 128, 1>(a, f);
}

}  // namespace
}  // namespace kvx
