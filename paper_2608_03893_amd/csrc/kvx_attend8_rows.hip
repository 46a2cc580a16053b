// Attention over the 8-bit pool, split over the query rows: chunks of new tokens, bf16.
//
// A workgroup of 8 waves takes 8 * 16 NB query rows of a KV head (tokens times the G heads)
// through 128 keys at a time; a wave has 16 NB rows.  The codes become bf16 matrix
// operands once: each wave takes half of 32 keys (K or V) from memory to registers,
// widens them to the layout of the matrix instruction's first operand and leaves them in
// LDS, whole operands one after another, so that reads and writes of LDS are 16 bytes a
// lane without conflicts.  Two such buffers: while the waves compute on one, the loads of
// the next are in flight.  The products are those of the split kernel (kvx_attend8.hip).
// A value's scale is applied as the code is widened where it is a power of two, which is exact
// there, and else to the probabilities.
//
// Bound by the matrix cores, with the exponentials (16 cycles for 64) beside them:
// 2048 new tokens of 64 heads over 10240 keys, d = 128, 820 us: 755 TFLOP/s, and 1130 with the
// products of the probabilities' second term, where a large product of the library reaches
// 1230 (another card: 920 us).  With one term, to form a step's scores beside the exponentials of
// the step before took 8% longer.
//
// One workgroup a CU; each takes an equal share of the weight of all (request, head, block
// of rows), a block's weight being the keys that its last row sees.  Neighbouring
// shares lie on the same XCD, whose L2 then holds a head's codes for all of its blocks.
#include "kvx_attend8.h"

namespace kvx {
namespace {

constexpr int kThreads = 512, kWaves = 8;
constexpr int kSteps = 4, kStep = 32, kQuant = kSteps * kStep;
constexpr int kGrid = 256;                 // workgroups: one per CU
constexpr int kRing = 4;                   // operands on their way from LDS

// Codes 2 HALF and 2 HALF + 1 of a word times a power of two, as bf16.
template <bool HALF>
__device__ __forceinline__ uint32_t bf16_pair_by(uint32_t w, float by) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, by, HALF));
}

template <int NB>
struct Weights {
  static constexpr int kRows = kWaves * 16 * NB, kSlope = kRows / kQuant;
  // Weight of block k (0-based) of a request and head, in quanta times G: the keys before the
  // new tokens, and those up to its last row.
  __device__ static int64_t before(const Request& r, int G) {
    return (int64_t)G * ((r.len > r.tokens ? r.len - r.tokens : 0) / kQuant + 1);
  }
  __device__ static int blocks(const Request& r) { return (r.rows + kRows - 1) / kRows; }
  // of blocks 0 .. n - 1
  __device__ static int64_t sum(int64_t before, int64_t n) { return n * before + kSlope * (n * (n + 1) / 2); }
};

template <int D, int NB>
__global__ void __launch_bounds__(kThreads, 2) attend8_rows_kernel(AttendArgs a, float* partial, int* counters) {
  using WT = Weights<NB>;
  constexpr int U = D / 64, C = D / 16, KF = 4 * U, F = KF + C;   // operands of a step: keys, all
  constexpr int ROWS = WT::kRows;
  constexpr int SLOT = kWaves * NB * (4 * C + 2) * 64;            // floats of a partial sum
  __shared__ __attribute__((aligned(16))) u32x4_t kv[2][kSteps][F][64];
  __shared__ float ksc[2][kSteps][2];       // scale of the scores of a 16-key tile
  __shared__ float vsc[2][kSteps][2];       // what its probabilities have yet to be multiplied by
  // [0], bit t: tile t has no page; [1], bit 0: some value is NaN (where rows of the block
  // differ in what they see), bit 1: vsc is not one
  __shared__ int flags[2][kSteps][2];
  __shared__ uint32_t nans[2][kSteps][U][64];   // which
  __shared__ int64_t part[kWaves];
  __shared__ int last;
  static_assert(sizeof(kv) >= KVX_MAX_REQUESTS * sizeof(int64_t), "the prefix sums fit");
  int64_t* pre = reinterpret_cast<int64_t*>(kv);   // until the first unit
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int step_of = wave & 3;             // the step whose keys (waves 0-3) or values this wave widens

  prefix_requests<kThreads>(a, pre, part, [&](const Request& r, int) {
    return a.H * WT::sum(WT::before(r, a.G), WT::blocks(r));
  });
  const int64_t total = uniform(pre[a.B - 1]);
  int64_t per = uniform((total + kGrid - 1) / kGrid);
  per = per > a.G ? per : a.G;      // a quantum at least
  const int me = xcd_order(blockIdx.x, kGrid);
  int64_t at = uniform((int64_t)me * per);
  const int64_t end = uniform(at + per < total ? at + per : total);
  if (at >= end) return;
  int b = uniform(find_request(pre, a.B, at));
  int64_t base = uniform(b > 0 ? pre[b - 1] : (int64_t)0);
  __syncthreads();

  const int64_t plane = ((int64_t)a.N << a.log2p) * D;
  const int P1 = (1 << a.log2p) - 1;
  while (at < end) {
    // the unit (request, head, block) at `at`; a lane's offsets are formed anew, which
    // costs less than keeping them over the main loop
    int ln = lane;
    asm volatile("" : "+v"(ln));
    const int n = ln & 15, g4 = ln >> 4;
    const Request r = request(a, b);
    const int64_t before = WT::before(r, a.G);
    const int blocks = WT::blocks(r);
    const int64_t head_w = WT::sum(before, blocks);
    if (at >= base + a.H * head_w) {
      base += a.H * head_w;
      ++b;
      continue;
    }
    const int h = uniform((int)((at - base) / head_w));
    const int64_t z = at - base - h * head_w;
    int blk = 0;
    for (int left = blocks; left > 0;) {   // last block whose first weight is at most z
      const int half = left >> 1;
      if (WT::sum(before, blk + half + 1) <= z) { blk += half + 1; left -= half + 1; }
      else left = half;
    }
    blk = uniform(blk);
    const int64_t unit0 = uniform(base + h * head_w + WT::sum(before, blk));
    const int64_t weight = uniform(WT::sum(before, blk + 1) - WT::sum(before, blk));
    const int last_row = (blk + 1) * ROWS < r.rows ? (blk + 1) * ROWS - 1 : r.rows - 1;
    const int lim_block = uniform(r.len - r.tokens + last_row / a.G);     // last key of the block
    const int quanta = lim_block < 0 ? 1 : lim_block / kQuant + 1;
    const int q0 = uniform((int)((at - unit0) * quanta / weight));
    const int q1 = uniform(
        end - unit0 >= weight ? quanta : (int)((end - unit0) * quanta / weight));

    // the lane's query rows (the block's last one again past the end), the last key of each
    int lim[NB];
    bf16x8_t qf[2 * U][NB];
    const int row0 = blk * ROWS + wave * 16 * NB;
#pragma unroll
    for (int x = 0; x < NB; ++x) {
      const int row = row0 + 16 * x + n < r.rows ? row0 + 16 * x + n : r.rows - 1;
      const int token = row / a.G, head = h * a.G + row % a.G;
      lim[x] = r.len - r.tokens + token;
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int w = 0; w < 2; ++w)
          qf[2 * u + w][x] = __builtin_bit_cast(
              bf16x8_t, *reinterpret_cast<const u32x4_t*>(static_cast<const uint16_t*>(a.q) +
                                                          (int64_t)(r.row0 + token) * a.q_stride[0] +
                                                          (int64_t)head * a.q_stride[1] + 64 * u + 16 * g4 + 8 * w));
    }
    // least and largest of the wave's limits (none: -1), and the least of the block's
    const int wave_last = row0 + 16 * NB - 1 < r.rows ? row0 + 16 * NB - 1 : r.rows - 1;
    const int lim_lo = uniform(r.len - r.tokens + row0 / a.G);
    const int lim_hi = uniform(row0 < r.rows ? r.len - r.tokens + wave_last / a.G : -1);
    const int block_lo = uniform(r.len - r.tokens + blk * ROWS / a.G);

    f32x4_t o[NB][C];
    float m[NB], l[NB];
#pragma unroll
    for (int x = 0; x < NB; ++x) {
      m[x] = -INFINITY;
      l[x] = 0.0f;
#pragma unroll
      for (int c = 0; c < C; ++c) o[x][c] = (f32x4_t){0, 0, 0, 0};
    }

    const uint8_t* codes = a.codes + (wave < 4 ? h : a.H + h) * plane;
    const float* scales = a.scales + (int64_t)(wave < 4 ? h : a.H + h) * a.N;
    const uint32_t lane_off = wave < 4 ? (uint32_t)n * D + 16 * g4 : (uint32_t)g4 * 4 * D + n * (D / 16);
    int page = -1, qa = 0;        // lane 2 s + t: page of tile t of this wave's step in quantum qa + s
    float scale = 0.0f;
    uint32_t st[8 * U];
    auto pages = [&](int q) {
      qa = q;
      page = -1;
      scale = 1.0f;
      const int64_t key = (int64_t)(q + (lane >> 1)) * kQuant + step_of * kStep + (lane & 1) * 16;
      if (key < r.len) page = a.tables[(int64_t)b * a.M + (key >> a.log2p)];
      if (page >= a.N) page = -1;
      if (page >= 0) scale = scales[page];
    };
    auto load = [&](int q) {
      const int key = q * kQuant + step_of * kStep;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        int p = __builtin_amdgcn_readlane(page, 2 * (q - qa) + t);
        p = p < 0 ? 0 : p;
        const uint8_t* from = codes + (((int64_t)p << a.log2p) + ((key + 16 * t) & P1)) * D + lane_off;
        if (wave < 4) {
#pragma unroll
          for (int u = 0; u < U; ++u) {
            const u32x4_t v = *reinterpret_cast<const u32x4_t*>(from + 64 * u);
#pragma unroll
            for (int i = 0; i < 4; ++i) st[4 * (t * U + u) + i] = v[i];
          }
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            if (D == 128) {
              const uint2 v = *reinterpret_cast<const uint2*>(from + j * D);
              st[(4 * t + j) * U] = v.x;
              st[(4 * t + j) * U + U - 1] = v.y;
            } else {
              st[4 * t + j] = *reinterpret_cast<const uint32_t*>(from + j * D);
            }
          }
        }
      }
    };
    auto widen = [&](int q, int buf) {
      const int key = q * kQuant + step_of * kStep;
      const int p0 = __builtin_amdgcn_readlane(page, 2 * (q - qa)), p1 = __builtin_amdgcn_readlane(page, 2 * (q - qa) + 1);
      float s0 = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(scale), 2 * (q - qa)));
      float s1 = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(scale), 2 * (q - qa) + 1));
      if (wave < 4) {
#pragma unroll
        for (int i = 0; i < 2 * U; ++i) {
          kv[buf][step_of][2 * i][lane] = __builtin_bit_cast(u32x4_t, bf16_octet(st[4 * i], st[4 * i + 1]));
          kv[buf][step_of][2 * i + 1][lane] = __builtin_bit_cast(u32x4_t, bf16_octet(st[4 * i + 2], st[4 * i + 3]));
        }
        if (lane == 0) {
          ksc[buf][step_of][0] = s0 * a.scale_log2;
          ksc[buf][step_of][1] = s1 * a.scale_log2;
          flags[buf][step_of][0] = (p0 < 0 ? 1 : 0) | (p1 < 0 ? 2 : 0);
        }
      } else {
        bool nan = false;
        if (p0 < 0 || p1 < 0 || key + kStep - 1 > block_lo) {
          // values under a scale that is infinite or NaN are NaN
          const bool lost0 = !finite(s0), lost1 = !finite(s1);
          s0 = lost0 ? 1.0f : s0;
          s1 = lost1 ? 1.0f : s1;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const bool real = (j < 4 ? p0 : p1) >= 0 && key + 16 * (j >> 2) + 4 * g4 + (j & 3) < r.len;
#pragma unroll
            for (int w = 0; w < U; ++w) {
              if (j < 4 ? lost0 : lost1) st[j * U + w] = kNan4;
              if (!real) st[j * U + w] = 0;
              nan |= e4m3_nan(st[j * U + w]) != 0;
            }
          }
        }
        nan = __any(nan);
        if (nan) {      // kept apart where rows differ in what they see: bit 4 j + i is key j, byte i
#pragma unroll
          for (int w = 0; w < U; ++w) {
            uint32_t bits = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const uint32_t h = e4m3_nan(st[j * U + w]);
              bits |= ((h >> 7 & 1) | (h >> 14 & 2) | (h >> 21 & 4) | (h >> 28 & 8)) << (4 * j);
              st[j * U + w] &= ~((h >> 7) * 0xffu);
            }
            nans[buf][step_of][w][lane] = bits;
          }
        }
        // powers of two, normal and positive, are applied with the conversion
        auto exact = [](float s) { return (__float_as_uint(s) & 0x807fffffu) == 0 && s >= 0x1p-126f && finite(s); };
        const float f0 = exact(s0) ? s0 : 1.0f, f1 = exact(s1) ? s1 : 1.0f;
        if (lane == 0) {
          vsc[buf][step_of][0] = exact(s0) ? 1.0f : s0;
          vsc[buf][step_of][1] = exact(s1) ? 1.0f : s1;
          flags[buf][step_of][1] = (nan ? 1 : 0) | (exact(s0) && exact(s1) ? 0 : 2);
        }
#pragma unroll
        for (int w = 0; w < U; ++w) {
          uint32_t y[4][2];   // keys 2 j, 2 j + 1 of channels (c, c + 1 | c + 2, c + 3)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            y[j][0] = __builtin_amdgcn_perm(st[(2 * j + 1) * U + w], st[2 * j * U + w], 0x05010400u);
            y[j][1] = __builtin_amdgcn_perm(st[(2 * j + 1) * U + w], st[2 * j * U + w], 0x07030602u);
          }
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            u32x4_t f;
#pragma unroll
            for (int j = 0; j < 4; ++j)
              f[j] = c & 1 ? bf16_pair_by<true>(y[j][c >> 1], j < 2 ? f0 : f1) : bf16_pair_by<false>(y[j][c >> 1], j < 2 ? f0 : f1);
            kv[buf][step_of][KF + 4 * w + c][lane] = f;
          }
        }
      }
    };

    // A step takes its operands from LDS in order, the keys' and then the values', kRing of
    // them on the way at any time; the scheduling barriers keep that order.
    auto compute = [&](int q, int buf) {
      int key = q * kQuant;
      if (key > lim_hi) return;
      const u32x4_t* from = &kv[buf][0][0][lane];
      u32x4_t f[kRing];
#pragma unroll
      for (int i = 0; i < kRing; ++i) f[i] = from[i * 64];
#pragma unroll 1
      for (int s = 0; s < kSteps && key <= lim_hi; ++s, key += kStep) {
        // A SIMD's two waves take turns at going first, two steps each: left alone, one always
        // does, and waits at the barrier for a third of the time (834 -> 820 us).
        if ((s >> 1 ^ wave >> 2) & 1) __builtin_amdgcn_s_setprio(1);
        else __builtin_amdgcn_s_setprio(0);
        const float sc[2] = {ksc[buf][s][0], ksc[buf][s][1]};
        const int bad = uniform(flags[buf][s][0]), vflags = uniform(flags[buf][s][1]), nan = vflags & 1;
        const u32x4_t* next = s + 1 < kSteps ? from + F * 64 : from;   // the last step's are not used
        f32x4_t x[2][NB];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int i = 0; i < NB; ++i) x[t][i] = (f32x4_t){0, 0, 0, 0};
#pragma unroll
        for (int k = 0; k < KF; ++k) {
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int i = 0; i < NB; ++i)
            x[k / (2 * U)][i] = mfma(__builtin_bit_cast(bf16x8_t, f[k % kRing]), qf[k % (2 * U)][i], x[k / (2 * U)][i]);
          f[k % kRing] = from[(k + kRing) * 64];
        }
        __builtin_amdgcn_sched_barrier(0);
        // exponents: scores less the row's reference
        const bool masked = (bad | nan) != 0 || key + kStep - 1 > lim_lo;
        bool grown = false;
        float top[NB];
#pragma unroll
        for (int i = 0; i < NB; ++i) {
          const float ref = m[i] == -INFINITY ? 0.0f : m[i];
#pragma unroll
          for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) x[t][i][e] = __builtin_fmaf(x[t][i][e], sc[t], -ref);
        }
        if (masked) {
#pragma unroll
          for (int i = 0; i < NB; ++i)
#pragma unroll
            for (int t = 0; t < 2; ++t) {
              const int most = bad >> t & 1 ? -1 : lim[i] - (key + 16 * t + 4 * g4);   // last element seen
#pragma unroll
              for (int e = 0; e < 4; ++e) x[t][i][e] = e > most ? -INFINITY : x[t][i][e];
            }
          // NaN values count only in rows that see their key
          if (nan != 0) {
#pragma unroll
            for (int i = 0; i < NB; ++i) {
              u32x4_t w;
#pragma unroll
              for (int j = 0; j < 4; ++j)
                w[j] = (x[j >> 1][i][2 * (j & 1)] == -INFINITY ? 0u : 0x3f80u) |
                       (x[j >> 1][i][2 * (j & 1) + 1] == -INFINITY ? 0u : 0x3f800000u);
              const bf16x8_t seen = __builtin_bit_cast(bf16x8_t, w);
#pragma unroll
              for (int c = 0; c < C; ++c) {
                const uint32_t bits = nans[buf][s][c / 4][lane] >> (c % 4);   // bit 4 j: key j of channel c
                u32x4_t hit;
#pragma unroll
                for (int j = 0; j < 4; ++j)
                  hit[j] = (bits >> (8 * j) & 1) * 0x3f80u | (bits >> (8 * j + 4) & 1) * 0x3f800000u;
                const f32x4_t count = mfma(__builtin_bit_cast(bf16x8_t, hit), seen, (f32x4_t){0, 0, 0, 0});
#pragma unroll
                for (int e = 0; e < 4; ++e) o[i][c][e] = count[e] != 0.0f ? __builtin_nanf("") : o[i][c][e];
              }
            }
          }
        }
#pragma unroll
        for (int i = 0; i < NB; ++i) {
          top[i] = fmaxf(fmaxf(fmaxf(x[0][i][0], x[0][i][1]), fmaxf(x[0][i][2], x[0][i][3])),
                         fmaxf(fmaxf(x[1][i][0], x[1][i][1]), fmaxf(x[1][i][2], x[1][i][3])));
          grown |= top[i] > (m[i] == -INFINITY ? -INFINITY : kLazy);
        }
        // The reference follows the maximum only when that has grown by 2^8: the sums hold
        // that, no lane has to ask the others in most steps, and O is seldom rescaled.
        if (__any(grown)) {
#pragma unroll
          for (int i = 0; i < NB; ++i) {
            const float ref = m[i] == -INFINITY ? 0.0f : m[i];
            const float now = fmaxf(m[i], quad_max(top[i]) + ref);
            const float keep = now == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m[i] - now);
            const float shift = now == -INFINITY ? 0.0f : ref - now;
            m[i] = now;
            l[i] *= keep;
#pragma unroll
            for (int c = 0; c < C; ++c) o[i][c] *= keep;
#pragma unroll
            for (int t = 0; t < 2; ++t) x[t][i] += shift;
          }
        }
        bf16x8_t p[NB][kTerms<0>];
#pragma unroll
        for (int i = 0; i < NB; ++i) {
          float y[8];
#pragma unroll
          for (int t = 0; t < 2; ++t) {
#pragma unroll
            for (int e = 0; e < 4; ++e) y[4 * t + e] = __builtin_amdgcn_exp2f(x[t][i][e]);
            l[i] += (y[4 * t] + y[4 * t + 1]) + (y[4 * t + 2] + y[4 * t + 3]);
          }
          if (vflags & 2) {
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] *= vsc[buf][s][j >> 2];
          }
          split_terms<kTerms<0>>(y, p[i]);
        }
#pragma unroll
        for (int c = 0; c < C; ++c) {
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int e = 0; e < kTerms<0>; ++e)
#pragma unroll
            for (int i = 0; i < NB; ++i) o[i][c] = mfma(__builtin_bit_cast(bf16x8_t, f[(KF + c) % kRing]), p[i][e], o[i][c]);
          f[(KF + c) % kRing] = KF + c + kRing < F ? from[(KF + c + kRing) * 64] : next[(KF + c + kRing - F) * 64];
        }
        __builtin_amdgcn_sched_barrier(0);
        from = next;
      }
    };

    if (q0 < q1) {
      pages(q0);
      load(q0);
      widen(q0, 0);
      __syncthreads();
      for (int q = q0; q < q1; ++q) {
        const int buf = (q - q0) & 1;
        const bool more = q + 1 < q1;
        if (more) {
          if (q + 1 - qa == 32) pages(q + 1);
          load(q + 1);
        }
        compute(q, buf);
        if (more) widen(q + 1, buf ^ 1);
        __syncthreads();
      }
    }
#pragma unroll
    for (int x = 0; x < NB; ++x) l[x] = quad_sum(l[x]);

    // shares that hold a part of this unit: g0 .. g1, each gives a partial sum (of no key
    // where its share of the weight holds no whole quantum)
    const int64_t g0 = unit0 / per, g1 = (unit0 + weight - 1) / per;
    bool done = g0 == g1;
    asm volatile("" : "+v"(ln));
    if (!done) {
      const int parts = (int)(g1 - g0) + 1, mine_at = (int)(me - g0);
      auto slot = [&](int i) { return 2 * ((int)g0 + i) + (i == 0 ? 1 : 0); };
      auto put = [&](int i) {
        float* to = partial + (int64_t)slot(i) * SLOT + wave * NB * (4 * C + 2) * 64 + 2 * ln;
        if (row0 >= r.rows) return;
#pragma unroll
        for (int x = 0; x < NB; ++x) {
#pragma unroll
          for (int c = 0; c < C; ++c) {
            put2(to + (x * (2 * C + 1) + 2 * c) * 128, o[x][c][0], o[x][c][1]);
            put2(to + (x * (2 * C + 1) + 2 * c + 1) * 128, o[x][c][2], o[x][c][3]);
          }
          put2(to + (x * (2 * C + 1) + 2 * C) * 128, m[x], l[x]);
        }
      };
      auto join = [&](int first, int stride, int count) {
        if (row0 >= r.rows) return;
#pragma unroll
        for (int x = 0; x < NB; ++x) {
          m[x] = -INFINITY;
          l[x] = 0.0f;
#pragma unroll
          for (int c = 0; c < C; ++c) o[x][c] = (f32x4_t){0, 0, 0, 0};
        }
#pragma unroll 1
        for (int i = 0; i < count; ++i) {
          const float* from = partial + (int64_t)slot(first + i * stride) * SLOT + wave * NB * (4 * C + 2) * 64 + 2 * ln;
#pragma unroll
          for (int x = 0; x < NB; ++x) {
            float2 v[2 * C];
#pragma unroll
            for (int c = 0; c < 2 * C; ++c) v[c] = get2(from + (x * (2 * C + 1) + c) * 128);
            const float2 ml = get2(from + (x * (2 * C + 1) + 2 * C) * 128);
            const float now = fmaxf(m[x], ml.x), ref = now == -INFINITY ? 0.0f : now;
            const float keep = __builtin_amdgcn_exp2f(m[x] - ref), f = __builtin_amdgcn_exp2f(ml.x - ref);
            m[x] = now;
            l[x] = l[x] * keep + ml.y * f;
#pragma unroll
            for (int c = 0; c < C; ++c) {
              o[x][c][0] = o[x][c][0] * keep + v[2 * c].x * f;
              o[x][c][1] = o[x][c][1] * keep + v[2 * c].y * f;
              o[x][c][2] = o[x][c][2] * keep + v[2 * c + 1].x * f;
              o[x][c][3] = o[x][c][3] * keep + v[2 * c + 1].y * f;
            }
          }
        }
      };
      put(mine_at);
      // More than four parts are joined in two levels of about equal width, the first by
      // several workgroups at once (one alone reads 16 parts in 35 us).
      int width = parts;
      if (parts > 4)
        for (width = 3; width * width < parts;) ++width;
      const int group = mine_at / width, groups = (parts + width - 1) / width;
      const int in_group = parts - group * width < width ? parts - group * width : width;
      if (arrive(counters + 2 * slot(group * width), in_group, &last)) {
        join(group * width, 1, in_group);
        done = groups == 1;
        if (!done) {
          put(group * width);    // each wave overwrites what only it has read
          if (arrive(counters + 2 * slot(0) + 1, groups, &last)) {
            join(0, width, groups);
            done = true;
          }
        }
      }
    }
    if (done) {
#pragma unroll
      for (int x = 0; x < NB; ++x) {
        const int row = row0 + 16 * x + (ln & 15);
        if (row >= r.rows) continue;
        const int64_t to = (int64_t)(r.row0 + row / a.G) * a.H * a.G + h * a.G + row % a.G;
        const float f = l[x] == 0.0f ? 0.0f : 1.0f / l[x];    // no key: 0
        u32x4_t* y = reinterpret_cast<u32x4_t*>(static_cast<uint16_t*>(a.out) + to * D + 4 * C * (ln >> 4));
        // channel (4 g4 + i) C + c
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (C == 8) {
            u32x4_t w;
#pragma unroll
            for (int c = 0; c < 4; ++c) w[c] = pack2(o[x][(2 * c) % C][i] * f, o[x][(2 * c + 1) % C][i] * f);
            y[i] = w;
          } else if (i % 2 == 0) {
            y[i / 2] = (u32x4_t){pack2(o[x][0][i] * f, o[x][1][i] * f), pack2(o[x][2][i] * f, o[x][3][i] * f),
                                 pack2(o[x][0][i + 1] * f, o[x][1][i + 1] * f),
                                 pack2(o[x][2][i + 1] * f, o[x][3][i + 1] * f)};
          }
        }
        if (a.lse != nullptr && ln < 16)
          a.lse[to] = l[x] == 0.0f ? -INFINITY : (m[x] + __builtin_amdgcn_logf(l[x])) * 0.69314718055994530942f;
      }
    }
    __syncthreads();     // `last` and the buffers are free again
    at = uniform(unit0 + weight);
  }
}

constexpr int kNb = 2;

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
