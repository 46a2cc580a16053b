// Next tokens drawn from rows of logits: temperature, top-k, top-p, min-p, and a given uniform
// random number for each row.
//
// Order the tokens of a row by falling logit, equal ones by rising index.  Every restriction
// keeps a prefix of that order, so the kept tokens are those up to one of them, the cut.  The
// token drawn is the first, in order of the vocabulary, at which the sum of the kept weights
// exceeds u times their total.
//
// Weights are exp((x - top) / T) in 64 bits, held as multiples of 2^-43 in whole numbers, so
// that sums are the same in whatever order they are formed.  Tokens below 2^-44 of the best
// one's weight have none.
//
// A row is cut into chunks, one a workgroup, and into strips, one or several a wave, and goes
// through up to three launches; in each the workgroup that comes last at a row's counter goes on
// with what all have found.
//   1  The largest logits; the answer for greedy rows.  For a small top-k also the answer: a
//      workgroup lists the logits from a bound on that m of its own reach, which the maxima of its
//      lanes say, anew whenever four times as much has been seen (so that a list holds few times
//      m).  m is k where it has the whole row; else its share of k and what chance may add, and the
//      workgroup that comes last looks whether k of all are above the highest bound: then nothing
//      that was not listed is among them.  The lists' tokens above it, the cut, the draw.
//   2  Rows without top-k and top-p: the strips' sums of weights; last: the draw.  Others: a
//      histogram of counts and weights over the logits that have a weight; last: the bins that the
//      cuts lie in.
//   3  Rows of the last kind: the strips' sums of weights above these bins, the tokens in them as
//      a list; last: the cut, the draw.
// Where a list would not fit (thousands of equal logits at a cut) the row goes the next way, and at
// last one workgroup narrows the bins down over the whole row.
//
// A logit is read once by way of a list, two or three times else, the later ones from the caches.
// Large batches by lists are bound by these reads: 512 rows of 131072 fp32 logits, 268 MB, with one
// k and p take 82 us, 3.3 TB/s, 72 of them in the first launch.  All others are bound by chains of
// steps that wait for each other, each a microsecond or less: what says how a row goes, its logits,
// the counter, what all have found, sums over the workgroup, the cut, the draw.  One row of 131072
// takes 20 us (14.5 + 3 + 2.4 in the launches), 64 bf16 rows of 128257 with settings of their own 64
// (16.6 + 20.7 + 27), 16 fp32 rows of 150001 with flat distributions 44 (4.8 + 16.2 + 24.4).
// A workgroup of 1024 threads for each row took 39, 465, 659 us, and 152 for the batch.
#include "kvx_bf16.h"
#include "kvx_serve.h"

namespace kvx {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kList = 2048;                // most tokens of a list in LDS
constexpr int kShort = 2048;               // and in the first launch
constexpr int kLong = 2560;                // and of all workgroups of a row together
constexpr int kFew = 256;                  // most tokens that are ranked by counting
constexpr int kBins = 2048;
constexpr int kStrips = 256;               // most strips of a row, and waves
constexpr int kHeld = 4;                   // vectors of a lane that the first bound is from
constexpr int kFinal = 8;                  // logits of a thread in the last step of a draw
constexpr int kFraction = 43;              // bits of a weight behind the point
constexpr double kOne = 8796093022208.0;   // 2^43: the best token's weight
constexpr float kRange = 30.5f;            // 44 ln 2: what a weight of 2^-44 is below the best, over T
static_assert(kList % kThreads == 0 && kShort % kThreads == 0, "a thread's entries of the list");

template <int DT>
struct Logits;
template <>
struct Logits<0> {
  static constexpr int N = 8;
  typedef uint16_t T;
  __device__ __forceinline__ static float one(T x) { return __uint_as_float((uint32_t)x << 16); }
  __device__ __forceinline__ static void get(const u32x4_t& q, float* x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = lo_bf16(q[i]);
      x[2 * i + 1] = hi_bf16(q[i]);
    }
  }
};
template <>
struct Logits<1> {
  static constexpr int N = 4;
  typedef float T;
  __device__ __forceinline__ static float one(T x) { return x; }
  __device__ __forceinline__ static void get(const u32x4_t& q, float* x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(q[i]);
  }
};

__device__ __forceinline__ uint32_t uniform(uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); }
__device__ __forceinline__ float clean(float x) { return x == x ? x : -INFINITY; }   // NaN: not allowed

// Rising with x, equal for the two zeros.
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t u = __float_as_uint(x + 0.0f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float of_key(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }

// 2^(j / 64).
constexpr int kPowers = 64;
__constant__ double kPower[kPowers] = {
    0x1.0000000000000p+0, 0x1.02c9a3e778061p+0, 0x1.059b0d3158574p+0, 0x1.0874518759bc8p+0,
    0x1.0b5586cf9890fp+0, 0x1.0e3ec32d3d1a2p+0, 0x1.11301d0125b51p+0, 0x1.1429aaea92de0p+0,
    0x1.172b83c7d517bp+0, 0x1.1a35beb6fcb75p+0, 0x1.1d4873168b9aap+0, 0x1.2063b88628cd6p+0,
    0x1.2387a6e756238p+0, 0x1.26b4565e27cddp+0, 0x1.29e9df51fdee1p+0, 0x1.2d285a6e4030bp+0,
    0x1.306fe0a31b715p+0, 0x1.33c08b26416ffp+0, 0x1.371a7373aa9cbp+0, 0x1.3a7db34e59ff7p+0,
    0x1.3dea64c123422p+0, 0x1.4160a21f72e2ap+0, 0x1.44e086061892dp+0, 0x1.486a2b5c13cd0p+0,
    0x1.4bfdad5362a27p+0, 0x1.4f9b2769d2ca7p+0, 0x1.5342b569d4f82p+0, 0x1.56f4736b527dap+0,
    0x1.5ab07dd485429p+0, 0x1.5e76f15ad2148p+0, 0x1.6247eb03a5585p+0, 0x1.6623882552225p+0,
    0x1.6a09e667f3bcdp+0, 0x1.6dfb23c651a2fp+0, 0x1.71f75e8ec5f74p+0, 0x1.75feb564267c9p+0,
    0x1.7a11473eb0187p+0, 0x1.7e2f336cf4e62p+0, 0x1.82589994cce13p+0, 0x1.868d99b4492edp+0,
    0x1.8ace5422aa0dbp+0, 0x1.8f1ae99157736p+0, 0x1.93737b0cdc5e5p+0, 0x1.97d829fde4e50p+0,
    0x1.9c49182a3f090p+0, 0x1.a0c667b5de565p+0, 0x1.a5503b23e255dp+0, 0x1.a9e6b5579fdbfp+0,
    0x1.ae89f995ad3adp+0, 0x1.b33a2b84f15fbp+0, 0x1.b7f76f2fb5e47p+0, 0x1.bcc1e904bc1d2p+0,
    0x1.c199bdd85529cp+0, 0x1.c67f12e57d14bp+0, 0x1.cb720dcef9069p+0, 0x1.d072d4a07897cp+0,
    0x1.d5818dcfba487p+0, 0x1.da9e603db3285p+0, 0x1.dfc97337b9b5fp+0, 0x1.e502ee78b3ff6p+0,
    0x1.ea4afa2a490dap+0, 0x1.efa1bee615a27p+0, 0x1.f50765b6e4540p+0, 0x1.fa7c1819e90d8p+0,
};
// 2^43 times exp((x - top) / T), to the nearest whole number; by = log2(e) / T.  The exponent of 2
// is a whole number of 64ths, whose power is in `power` (LDS), and a rest r of half a 64th at most,
// for which a polynomial of degree 4 through four Chebyshev points and 1 at r = 0 is off by 4.9e-15
// (with a series of degree 11 over a whole unit 64 rows with settings of their own took 66.5 us
// instead of 64.6).  Without branches, so that the chains of several logits run side by side.
__device__ __forceinline__ uint64_t weight_of(float x, float top, double by, const double* power) {
  const double z = x == top ? 0.0 : ((double)x - (double)top) * by;
  const bool some = z > -45.0;      // (not where z is NaN)
  const double y = some ? z : 0.0;
  constexpr double kWhole = 6755399441055744.0;      // 1.5 2^52: a sum with it has the rounded number in its low bits
  const double sum = __builtin_fma(y, (double)kPowers, kWhole);
  const int n = (int)(uint32_t)__builtin_bit_cast(uint64_t, sum);
  const double r = __builtin_fma(y, (double)kPowers, kWhole - sum);
  double p = 0x1.3b2acb2c36b23p-31;
  p = __builtin_fma(p, r, 0x1.c6b0b9214b9aep-23);
  p = __builtin_fma(p, r, 0x1.ebfbdff82bb76p-15);
  p = __builtin_fma(p, r, 0x1.62e42fefa2417p-7);
  p = __builtin_fma(p, r, 1.0);
  const uint64_t whole = __builtin_bit_cast(uint64_t, power[n & (kPowers - 1)]);
  const uint64_t shift = (uint64_t)(uint32_t)(((n >> 6) + kFraction) * (1 << 20)) << 32;      // exponents of normal numbers
  // the sum with 2^52 has the rounded number in its low bits
  const double w = __builtin_fma(p, __builtin_bit_cast(double, whole + shift), 4503599627370496.0);
  return some ? __builtin_bit_cast(uint64_t, w) & 0xfffffffffffffull : 0;
}

// v of the lane that CTRL names, 0 in lanes of rows that ROWS leaves out and where there is none.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint64_t moved(uint64_t v) {
  const int lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, CTRL, ROWS, 0xf, false);
  const int hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(v >> 32), CTRL, ROWS, 0xf, false);
  return (uint64_t)(uint32_t)hi << 32 | (uint32_t)lo;
}
// Sum over the lanes up to this one; all lanes call.
__device__ __forceinline__ uint64_t wave_scan(uint64_t v) {
  v += moved<0x111, 0xf>(v);      // 1, 2, 4, 8 lanes on within rows of 16
  v += moved<0x112, 0xf>(v);
  v += moved<0x114, 0xf>(v);
  v += moved<0x118, 0xf>(v);
  v += moved<0x142, 0xa>(v);      // a row's last lane to the next row, the second row's to the upper half
  v += moved<0x143, 0xc>(v);
  return v;
}
__device__ __forceinline__ uint64_t wave_sum(uint64_t v) {
  v = wave_scan(v);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, 63);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(v >> 32), 63);
  return (uint64_t)hi << 32 | lo;
}

// A row's settings, restrictions that cannot bind switched off.
struct Setting {
  float top;            // its largest logit
  double by;            // log2(e) / T
  float bins;           // of the histogram, a unit of half the logits (see task_of)
  uint64_t least;       // weight that min-p asks for
  int32_t k;            // 0: all
  double p;             // 2: all
  double u;
};

template <int DT>
struct Row {
  using LG = Logits<DT>;
  using T = typename LG::T;
  const T* x;
  int32_t V, head, vecs;      // logits before the first 16-byte boundary, whole vectors behind it
  int32_t per;                // vectors of a strip
  __device__ __forceinline__ Row(const T* from, int32_t v, int32_t p) : x(from), V(v), per(p) {
    head = (int32_t)(-(reinterpret_cast<uintptr_t>(from) / sizeof(T)) & (LG::N - 1));
    head = head < V ? head : V;
    vecs = (V - head) / LG::N;
  }
  __device__ __forceinline__ float at(int32_t i) const { return clean(LG::one(x[i])); }
  // f(logits, their number, index of the first) for every vector of v0 .. v1 - 1 that thread `me`
  // of `n` has, from the last on where BACK: what was read last is still in the caches.  FLIGHT
  // loads of a thread are on the way while as many vectors go through f.  f is there once, in a
  // loop: rows run through it a few times only (a chunk's histogram in the second launch takes 6.0 us
  // so, 7.0 with f unrolled over the loads)
  template <bool BACK, int FLIGHT, typename F>
  __device__ __forceinline__ void vectors(int v0, int v1, int me, int n, F f) const {
    const u32x4_t* from = reinterpret_cast<const u32x4_t*>(x + head);
    const int steps = (v1 - v0 + n - 1) / n;
    u32x4_t q[FLIGHT], next[FLIGHT];
    auto vector = [&](int s) {      // -1: none
      const int v = v0 + (BACK ? steps - 1 - s : s) * n + me;
      return s < steps && v < v1 ? v : -1;
    };
    auto load = [&](int s) {
      const int v = vector(s);
      return from[v < 0 ? v0 : v];
    };
#pragma unroll
    for (int i = 0; i < FLIGHT; ++i) q[i] = load(i);
#pragma unroll 1
    for (int s = 0; s < steps; s += FLIGHT) {
      const int some = steps - s < FLIGHT ? steps - s : FLIGHT;
      if (s + FLIGHT < steps)
#pragma unroll
        for (int i = 0; i < FLIGHT; ++i) next[i] = load(s + FLIGHT + i);
#pragma unroll 1
      for (int i = 0; i < some; ++i) {
        const int v = vector(s + i);
        float y[LG::N];
        LG::get(q[0], y);
#pragma unroll
        for (int j = 0; j + 1 < FLIGHT; ++j) q[j] = q[j + 1];
#pragma unroll
        for (int e = 0; e < LG::N; ++e) y[e] = v < 0 ? -INFINITY : clean(y[e]);
        f(y, head + v * LG::N);
      }
#pragma unroll
      for (int i = 0; i < FLIGHT; ++i) q[i] = next[i];
    }
  }
  // Strip n of `strips`: its vectors, and its logits, those outside whole vectors with the first
  // and the last strip.
  struct Strip {
    int32_t v0, v1, lo, hi;
  };
  __device__ __forceinline__ Strip strip(int n, int strips) const {
    const int32_t first = n * per;
    Strip s;
    s.v0 = first < vecs ? first : vecs;
    s.v1 = first + per < vecs ? first + per : vecs;
    s.lo = n == 0 ? 0 : head + s.v0 * LG::N;
    s.hi = n == strips - 1 ? V : head + s.v1 * LG::N;
    return s;
  }
  __device__ __forceinline__ int strip_of(int32_t i, int strips) const {
    const int32_t v = (i - head) / LG::N;
    return i < head ? 0 : v < vecs ? v / per : strips - 1;
  }
  // f as in vectors, for all logits of a strip by a wave.
  template <bool BACK, int FLIGHT, typename F>
  __device__ __forceinline__ void of_strip(int n, int strips, F f) const {
    const int lane = threadIdx.x & 63;
    const Strip s = strip(n, strips);
    if (s.v0 < s.v1) vectors<BACK, FLIGHT>(s.v0, s.v1, lane, 64, f);
    if (n == 0 || n == strips - 1) {
      int32_t i = lane < 2 * LG::N ? loose(lane) : -1;
      if (i >= 0 && !(i < head ? n == 0 : n == strips - 1)) i = -1;
      float y[LG::N];
#pragma unroll
      for (int e = 0; e < LG::N; ++e) y[e] = -INFINITY;
      if (i >= 0) y[0] = at(i);
      f(y, i);
    }
  }
  // logits outside whole vectors: thread i < 2 N has one
  __device__ __forceinline__ int32_t loose(int i) const {
    if (i < head) return i;
    const int32_t at = head + vecs * LG::N + i - LG::N;
    return i >= LG::N && at < V ? at : -1;
  }
  // all logits, in no order that matters; whole waves call
  template <bool BACK, int FLIGHT, typename F>
  __device__ __forceinline__ void all(F f) const {
    if (vecs > 0) vectors<BACK, FLIGHT>(0, vecs, threadIdx.x, kThreads, f);
    if (threadIdx.x < 64) {
      const int32_t i = loose(threadIdx.x);
      float y[LG::N];
#pragma unroll
      for (int e = 0; e < LG::N; ++e) y[e] = -INFINITY;
      if (i >= 0) y[0] = at(i);
      f(y, i);
    }
  }
};

template <int LIST>
struct List {
  uint64_t entry[LIST];        // ~key, index: rises in the order of the tokens
  uint64_t weight[LIST];
};
struct Bins {
  uint64_t weight[kBins];
  uint32_t count[kBins];
};
struct SharedBase {
  double power[kPowers];       // a kernel copies them before its first barrier
  uint64_t part[kWaves];
  uint64_t found[4];
  uint64_t strip[kStrips];     // also a scratch value of each thread
  uint32_t rank[kThreads];
  uint32_t count, lowest, highest, slot;
  float logit;                 // of the token in `slot`
  int last;
};
static_assert(kStrips == kThreads && kStrips / kWaves <= 64, "a strip a thread, a chunk a lane");
struct SharedFirst : SharedBase {
  List<kShort> list;
  float lanes[kThreads];
  uint32_t kept;
};
struct SharedWeigh : SharedBase {
  Bins bin;
};
struct SharedCut : SharedBase {
  union {
    Bins bin;
    List<kList> list;
  };
  uint64_t few[kFew], few_weight[kFew];
};

template <typename SH>
__device__ __forceinline__ void put_powers(SH& s) {
  if (threadIdx.x < kPowers) s.power[threadIdx.x] = kPower[threadIdx.x];
}
template <typename SH>
__device__ __forceinline__ uint64_t block_sum(uint64_t v, SH& s) {
  v = wave_sum(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s.part[threadIdx.x >> 6] = v;
  __syncthreads();
  v = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) v += s.part[w];
  return v;
}
// Sum over the threads up to this one.
template <typename SH>
__device__ __forceinline__ uint64_t block_scan(uint64_t v, SH& s) {
  const int wave = threadIdx.x >> 6;
  v = wave_scan(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 63) s.part[wave] = v;
  __syncthreads();
  for (int w = 0; w < wave; ++w) v += s.part[w];
  return v;
}

// Rising order of n entries in LDS, by bitonic exchanges over the next power of two.
__device__ __forceinline__ void sort_entries(uint64_t* e, int n) {
  int size = 2;
  while (size < n) size <<= 1;
  for (int i = n + (int)threadIdx.x; i < size; i += kThreads) e[i] = ~0ull;
  for (int k = 2; k <= size; k <<= 1)
    for (int j = k >> 1; j; j >>= 1) {
      __syncthreads();
      for (int i = threadIdx.x; i < size / 2; i += kThreads) {
        const int a = 2 * i - (i & (j - 1)), b = a + j;
        const uint64_t x = e[a], y = e[b];
        if ((x > y) == ((a & k) == 0)) {
          e[a] = y;
          e[b] = x;
        }
      }
    }
  __syncthreads();
}

// A row in the workspace.
struct State {
  int mode;                   // what launch 3 does
  int32_t above, upto, at_k;  // bins: sums up to `above`, listed above .. upto and at_k (-1: none)
  uint32_t before_k;          // tokens in bins before at_k
  uint64_t weight_k;          // weights before at_k, before `above`, of all
  uint64_t weight_above, total;
};
enum { kDone = 0, kCut = 1, kNarrow = 2 };
struct alignas(256) Space {
  uint32_t listed;                       // entries of the list
  int arrived[3];                        // workgroups, in each launch; zero between calls, as listed
  int over;                              // the first launch's list did not hold
  State state;
  float top[kStrips], low[kStrips];      // of a wave; low: of rows by bins, else -inf
  float bound[kStrips / kWaves];         // of a workgroup's list
  uint32_t first[kStrips];               // index of the first largest (greedy rows)
  uint64_t sum[kStrips];
  uint64_t entry[kLong];
  uint64_t weight[kBins];
  uint32_t count[kBins];
};
static_assert(offsetof(Space, over) == KVX_SAMPLE_COUNTER_BYTES && sizeof(Space) % 256 == 0, "what a caller clears");

template <typename T>
__device__ __forceinline__ void put(T* to, T v) { __hip_atomic_store(to, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
template <typename T>
__device__ __forceinline__ T get(const T* from) { return __hip_atomic_load(from, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// True in the workgroup that comes last of `count` at a counter, which is zero again then; what all
// have put is there.
template <typename SH>
__device__ __forceinline__ bool come_last(int* counter, int count, SH& s) {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (count == 1) return true;
  if (threadIdx.x == 0) {
    s.last = __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == count - 1;
    if (s.last) put(counter, 0);
  }
  __syncthreads();
  return s.last != 0;
}

template <int DT, typename SH, int LIST>
struct Sampler {
  const Row<DT> row;
  SH& s;
  Setting set;
  static constexpr int N = Logits<DT>::N;

  __device__ __forceinline__ uint64_t weight(float x) const { return weight_of(x, set.top, set.by, s.power); }

  // Entries of the tokens that `take` accepts among y, to places of a list in LDS (below `most`)
  // that its counter gives out, to a lane at a time.
  template <typename F>
  __device__ __forceinline__ void append(const float* y, int32_t first, uint64_t* to, uint32_t* count, uint32_t most, F take) const {
    uint32_t mine = 0;
#pragma unroll
    for (int e = 0; e < N; ++e) mine += take(y[e]) ? 1 : 0;
    if (mine == 0) return;
    uint32_t at = atomicAdd(count, mine);
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (take(y[e])) {
        if (at < most) to[at] = (uint64_t)~key_of(y[e]) << 32 | (uint32_t)(first + e);
        ++at;
      }
  }
  // The row's tokens that `take` accepts, as entries; their number.
  template <typename F>
  __device__ __forceinline__ int gather(F take) {
    __syncthreads();
    if (threadIdx.x == 0) s.count = 0;
    __syncthreads();
    row.template all<true, 2>([&](const float* y, int32_t first) {
      append(y, first, s.list.entry, &s.count, LIST, take);
    });
    __syncthreads();
    return (int)s.count;
  }

  // Entries in order and their weights; a thread gets the sums up to each of its entries
  // (kList / kThreads neighbouring ones).
  static constexpr int kMine = LIST / kThreads;
  __device__ __forceinline__ void order(int n, uint64_t* sums) {
    sort_entries(s.list.entry, n);
    uint64_t mine = 0;
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
      const int at = threadIdx.x * kMine + i;
      const uint64_t w = at < n ? weight(of_key(~(uint32_t)(s.list.entry[at] >> 32))) : 0;
      s.list.weight[at] = w;
      mine += w;
      sums[i] = mine;
    }
    const uint64_t before = block_scan(mine, s) - mine;
#pragma unroll
    for (int i = 0; i < kMine; ++i) sums[i] += before;
    __syncthreads();
  }
  // Entries whose sum stays below t: the place of the first that reaches it.
  __device__ __forceinline__ int reach(int n, const uint64_t* sums, uint64_t t) {
    uint64_t less = 0;
#pragma unroll
    for (int i = 0; i < kMine; ++i) less += threadIdx.x * kMine + i < n && sums[i] < t;
    return (int)block_sum(less, s);
  }
  // The sum up to entry `at`.
  __device__ __forceinline__ uint64_t sum_at(const uint64_t* sums, int at) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kMine; ++i)
      if ((int)threadIdx.x * kMine + i == at) s.found[0] = sums[i];
    __syncthreads();
    return s.found[0];
  }
  // For i < n <= kFew, in thread i (all threads call): the number of entries j < n that are less than
  // entry i, in order of their tokens (BY_INDEX: of their indexes), and the sum of their weights,
  // formed by several threads where n is small.
  struct Counted {
    uint32_t number;
    uint64_t sum;
  };
  template <bool BY_INDEX>
  __device__ __forceinline__ Counted counted(int n, const uint64_t* entry, const uint64_t* weights) {
    const int each = n <= 64 ? 64 : n <= 128 ? 128 : 256;      // threads of a share
    const int i = threadIdx.x & (each - 1), share = threadIdx.x / each, shares = kThreads / each;
    const uint64_t mine = entry[i < n ? i : 0];
    Counted c = {0, 0};
#pragma unroll 8
    for (int j = share; j < n; j += shares) {
      const uint64_t e = entry[j], w = weights[j];
      const bool less = BY_INDEX ? (uint32_t)e < (uint32_t)mine : e < mine;
      c.number += less ? 1u : 0u;
      c.sum += less ? w : 0;
    }
    if (shares == 1) return c;
    s.strip[threadIdx.x] = c.sum;
    s.rank[threadIdx.x] = c.number;
    __syncthreads();
    if (share == 0)
      for (int x = 1; x < shares; ++x) {
        c.sum += s.strip[x * each + i];
        c.number += s.rank[x * each + i];
      }
    __syncthreads();
    return c;
  }

  // The entry among the first n of the list, in bins lo .. hi, behind which there are `target`
  // entries, itself included (or their weights reach it), and the sum of these weights.
  struct Picked {
    uint64_t entry, sum;
  };
  __device__ __forceinline__ Picked pick(int n, int lo, int hi, bool by_count, uint64_t target) {
    if (n <= kFew) {       // counted among all, less what comes before the range
      const int i = threadIdx.x;
      const uint64_t e = i < n ? s.list.entry[i] : 0;
      const int bin = i < n ? bin_of(of_key(~(uint32_t)(e >> 32))) : kBins;
      const uint64_t mine = i < n ? s.list.weight[i] : 0;
      const Counted before = counted<false>(n, s.list.entry, s.list.weight);
      const uint64_t ahead = block_sum(bin < lo ? (by_count ? 1 : mine) : 0, s);
      const uint64_t at = (by_count ? (uint64_t)before.number : before.sum) - ahead;
      if (bin >= lo && bin <= hi && at < target && target <= at + (by_count ? 1 : mine)) {
        s.found[0] = e;
        s.found[1] = before.sum + mine;
      }
      const uint64_t skipped = by_count ? block_sum(bin < lo ? mine : 0, s) : ahead;
      __syncthreads();
      return Picked{s.found[0], s.found[1] - skipped};
    }
    // 256 bins over the range, in LDS that sums of strips use otherwise
    const float scale = (float)kThreads / (float)(hi - lo + 1);
    auto sub = [&](float x) {
      const int i = (int)((place_of(x) - (float)lo) * scale);
      return i < 0 ? 0 : i < kThreads ? i : kThreads - 1;
    };
    auto logit = [&](uint64_t e) { return of_key(~(uint32_t)(e >> 32)); };
    auto inside = [&](float x) {
      const int i = bin_of(x);
      return i >= lo && i <= hi;
    };
    __syncthreads();
    s.strip[threadIdx.x] = 0;
    s.rank[threadIdx.x] = 0;
    if (threadIdx.x == 0) s.count = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kThreads) {
      const float x = logit(s.list.entry[i]);
      if (!inside(x)) continue;
      atomicAdd(&s.rank[sub(x)], 1u);
      atomicAdd(reinterpret_cast<unsigned long long*>(&s.strip[sub(x)]), (unsigned long long)s.list.weight[i]);
    }
    __syncthreads();
    const uint64_t c = s.rank[threadIdx.x], w = s.strip[threadIdx.x];
    const uint64_t c1 = block_scan(c, s), w1 = block_scan(w, s);
    const uint64_t a = by_count ? c1 : w1, z = by_count ? c : w;
    __syncthreads();
    if (a - z < target && target <= a) {
      s.found[0] = c1 - c;
      s.found[1] = w1 - w;
      s.found[2] = c;
      s.slot = threadIdx.x;
    }
    __syncthreads();
    const uint64_t before_c = s.found[0], before_w = s.found[1], own = s.found[2];
    const int bin = (int)s.slot;
    __syncthreads();
    if (own <= kFew) {
      for (int i = threadIdx.x; i < n; i += kThreads) {
        const uint64_t e = s.list.entry[i];
        const float x = logit(e);
        if (inside(x) && sub(x) == bin) s.few[atomicAdd(&s.count, 1u)] = e;
      }
      __syncthreads();
      const int m = (int)own;
      if ((int)threadIdx.x < m) s.few_weight[threadIdx.x] = weight(logit(s.few[threadIdx.x]));
      __syncthreads();
      const Counted before = counted<false>(m, s.few, s.few_weight);
      if ((int)threadIdx.x < m) {
        const uint64_t mine = s.few_weight[threadIdx.x], sum = before_w + before.sum;
        const bool it = by_count ? before_c + before.number + 1 == target : sum < target && target <= sum + mine;
        if (it) {
          s.found[0] = s.few[threadIdx.x];
          s.found[1] = sum + mine;
        }
      }
    } else {       // many equal ones: all in order
      uint64_t sums[kMine];
      order(n, sums);
      uint64_t ahead = 0;
#pragma unroll
      for (int i = 0; i < kMine; ++i) {
        const int at = threadIdx.x * kMine + i;
        ahead += at < n && bin_of(logit(s.list.entry[at])) < lo;
      }
      const int first = (int)block_sum(ahead, s);
      const uint64_t base = first > 0 ? sum_at(sums, first - 1) : 0;
      const int at = by_count ? first + (int)target - 1 : reach(n, sums, base + target);
      const uint64_t sum = sum_at(sums, at) - base;
      __syncthreads();
      if (threadIdx.x == 0) {
        s.found[0] = s.list.entry[at];
        s.found[1] = sum;
      }
    }
    __syncthreads();
    return Picked{s.found[0], s.found[1]};
  }

  __device__ __forceinline__ static uint64_t up_to(double p, uint64_t total) {     // what top-p's sum has to reach
    const double t = ceil(p * (double)total);
    return t < 1.0 ? 1 : t < (double)total ? (uint64_t)t : total;
  }
  __device__ __forceinline__ static uint64_t behind(double u, uint64_t total) {    // what the draw's sum has to exceed
    const uint64_t t = (uint64_t)(u * (double)total);
    return t < total ? t : total - 1;
  }

  __device__ __forceinline__ void put_token(const SampleArgs& a, int b, int32_t token, float x, uint64_t total) {
    a.tokens[b] = token;
    if (a.logprob != nullptr) {
      const double y = x == set.top ? 0.0 : ((double)x - (double)set.top) * set.by;
      a.logprob[b] = (float)(y * 0.69314718055994530942 - log((double)total / kOne));
    }
  }

  // The draw among the first n entries, whose weights come to `total`.
  __device__ __forceinline__ void draw_list(const SampleArgs& a, int b, int n, uint64_t total, double u) {
    const uint64_t t = behind(u, total);
    uint64_t e[kMine];
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
      const int at = threadIdx.x + i * kThreads;
      e[i] = at < n ? (s.list.entry[at] & 0xffffffffu) << 32 | (uint32_t)at : 0;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kMine; ++i)
      if ((int)threadIdx.x + i * kThreads < n) s.list.entry[threadIdx.x + i * kThreads] = e[i];
    sort_entries(s.list.entry, n);
    uint64_t mine = 0, w[kMine];
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
      const int at = threadIdx.x * kMine + i;
      w[i] = at < n ? s.list.weight[(uint32_t)s.list.entry[at]] : 0;
      mine += w[i];
    }
    uint64_t sum = block_scan(mine, s) - mine;
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
      if (sum <= t && t < sum + w[i]) {
        const int32_t token = (int32_t)(s.list.entry[threadIdx.x * kMine + i] >> 32);
        put_token(a, b, token, row.at(token), total);
      }
      sum += w[i];
    }
  }

  // Cuts and draw from a list of n <= kFew entries in any order, which holds the first k tokens.
  __device__ __forceinline__ void finish_few(const SampleArgs& a, int b, int n) {
    const int i = threadIdx.x;
    const bool mine = i < n;
    const uint64_t e = mine ? s.list.entry[i] : 0;
    const float x = mine ? of_key(~(uint32_t)(e >> 32)) : -INFINITY;
    const uint64_t w = mine ? weight(x) : 0;
    if (mine) s.list.weight[i] = w;
    __syncthreads();
    // (barriers inside: called by all threads, whatever they hold)
    const Counted better = counted<false>(n, s.list.entry, s.list.weight);
    bool keep = mine && better.number < (uint32_t)set.k;
    if (set.p <= 1.0) {
      const uint64_t t = up_to(set.p, block_sum(keep ? w : 0, s));
      keep = keep && better.sum < t;
    }
    keep = keep && w >= set.least;
    const uint64_t total = block_sum(keep ? w : 0, s);
    if (mine) s.list.weight[i] = keep ? w : 0;
    __syncthreads();
    const uint64_t t = behind(set.u, total);
    const uint64_t before = counted<true>(n, s.list.entry, s.list.weight).sum;
    if (keep && before <= t && t < before + w) put_token(a, b, (int32_t)(uint32_t)e, x, total);
  }

  // The place in lo .. hi - 1 at which the sum of f over it, in order of the vocabulary, first
  // exceeds t (less than all of it).
  template <typename F>
  __device__ __forceinline__ int32_t locate(int32_t lo, int32_t hi, uint64_t t, F f) {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    while (hi - lo > kThreads * kFinal) {
      const int32_t per = ((hi - lo + kWaves - 1) / kWaves + 63) / 64 * 64;
      uint64_t sum = 0;
      const int32_t a = lo + wave * per, z = a + per < hi ? a + per : hi;
      for (int32_t i = a + lane; i < z; i += 64 * kFinal) {
        float y[kFinal];
#pragma unroll
        for (int j = 0; j < kFinal; ++j) y[j] = row.at(i + 64 * j < z ? i + 64 * j : a);
#pragma unroll
        for (int j = 0; j < kFinal; ++j) sum += i + 64 * j < z ? f(y[j], i + 64 * j) : 0;
      }
      sum = wave_sum(sum);
      __syncthreads();
      if (lane == 0) s.part[wave] = sum;
      __syncthreads();
      int w = 0;
      while (w < kWaves - 1 && t >= s.part[w]) t -= s.part[w++];
      lo += w * per;
      hi = lo + per < hi ? lo + per : hi;
      __syncthreads();
    }
    const int32_t i = lo + (int32_t)threadIdx.x * kFinal;
    float y[kFinal];
    uint64_t v[kFinal], mine = 0;
#pragma unroll
    for (int j = 0; j < kFinal; ++j) y[j] = row.at(i + j < hi ? i + j : lo);
#pragma unroll
    for (int j = 0; j < kFinal; ++j) {
      v[j] = i + j < hi ? f(y[j], i + j) : 0;
      mine += v[j];
    }
    uint64_t sum = block_scan(mine, s) - mine;
#pragma unroll
    for (int j = 0; j < kFinal; ++j) {
      if (sum <= t && t < sum + v[j]) {
        s.slot = (uint32_t)(i + j);
        s.logit = y[j];
      }
      sum += v[j];
    }
    __syncthreads();
    return (int32_t)s.slot;
  }

  // The draw from the strips' sums (in s.strip) of f.
  template <typename F>
  __device__ __forceinline__ void draw_strips(const SampleArgs& a, int b, int strips, double u, F f) {
    const uint64_t v = (int)threadIdx.x < strips ? s.strip[threadIdx.x] : 0, upto = block_scan(v, s);
    __syncthreads();
    if (threadIdx.x == kThreads - 1) s.found[0] = upto;
    __syncthreads();
    const uint64_t total = s.found[0], t = behind(u, total);
    if (v > 0 && upto - v <= t && t < upto) {
      s.slot = threadIdx.x;
      s.found[1] = t - (upto - v);
    }
    __syncthreads();
    const typename Row<DT>::Strip where = row.strip((int)s.slot, strips);
    const int32_t token = locate(where.lo, where.hi, s.found[1], f);
    if (threadIdx.x == 0) put_token(a, b, token, s.logit, total);
  }

  // ---- the cut by histograms ----

  // What launch 3 has to look at, from the histogram of the row, which becomes sums up to each bin.
  __device__ __forceinline__ void plan(State& to) {
    constexpr int M = kBins / kThreads;      // neighbouring bins of a thread
    uint64_t c[M], w[M], c0 = 0, w0 = 0;
#pragma unroll
    for (int i = 0; i < M; ++i) {
      c[i] = c0 += s.bin.count[threadIdx.x * M + i];
      w[i] = w0 += s.bin.weight[threadIdx.x * M + i];
    }
    c0 = wave_scan(c0) - c0;
    w0 = wave_scan(w0) - w0;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (lane == 63) {
      s.part[wave] = w0 + w[M - 1];
      s.strip[wave] = c0 + c[M - 1];
    }
    __syncthreads();
    for (int x = 0; x < wave; ++x) {
      w0 += s.part[x];
      c0 += s.strip[x];
    }
#pragma unroll
    for (int i = 0; i < M; ++i) {
      c[i] += c0;
      w[i] += w0;
      s.bin.count[threadIdx.x * M + i] = (uint32_t)c[i];
      s.bin.weight[threadIdx.x * M + i] = w[i];
    }
    // the first bin up to which the count (or the weight) reaches the target; kBins: there is none
    auto first_bin = [&](const uint64_t* sums, uint64_t target) {
      uint64_t below = 0;
#pragma unroll
      for (int i = 0; i < M; ++i) below += sums[i] < target;
      return (int)block_sum(below, s);
    };
    __syncthreads();
    auto count = [&](int i) { return i < 0 ? 0u : s.bin.count[i]; };
    auto weight_to = [&](int i) { return i < 0 ? (uint64_t)0 : s.bin.weight[i]; };
    const bool by_k = set.k > 0 && (uint32_t)set.k < count(kBins - 1), by_p = set.p <= 1.0;
    State st;
    st.at_k = by_k ? first_bin(c, (uint64_t)set.k) : -1;
    st.before_k = by_k ? count(st.at_k - 1) : 0;
    st.weight_k = by_k ? weight_to(st.at_k - 1) : 0;
    st.total = weight_to(kBins - 1);
    if (by_p) {       // for the least and the largest weight that top-k may leave
      const uint64_t least = by_k ? st.weight_k : st.total, most = by_k ? weight_to(st.at_k) : st.total;
      st.above = least > 0 ? first_bin(w, up_to(set.p, least)) : 0;
      st.upto = most == least ? st.above : first_bin(w, up_to(set.p, most));
    } else {
      st.above = by_k ? st.at_k : kBins;       // else nothing is cut
      st.upto = by_k ? st.at_k : -1;
    }
    st.weight_above = weight_to(st.above - 1);
    uint32_t listed = st.upto >= st.above ? count(st.upto) - count(st.above - 1) : 0;
    if (by_k && st.at_k > st.upto) listed += count(st.at_k) - count(st.at_k - 1);
    if (threadIdx.x == 0) {
      to.above = st.above;
      to.upto = st.upto;
      to.at_k = st.at_k;
      to.before_k = st.before_k;
      to.weight_k = st.weight_k;
      to.weight_above = st.weight_above;
      to.total = st.total;
      to.mode = listed <= kList ? kCut : kNarrow;
    }
  }

  // A range of logits: those of one bin over the weights' range, or of keys lo .. hi.
  struct Range {
    int bin;               // -1: by keys
    uint32_t lo, hi;
  };
  // Where a logit is in the histogram, in bins; rises as x falls.  From half the logits, whose
  // difference fp32 always holds: at temperatures near the end of its range the whole one may pass
  // that though the logit has a weight.
  __device__ __forceinline__ float place_of(float x) const {
    return x == set.top ? 0.0f : __builtin_fmaf(-0.5f, x, 0.5f * set.top) * set.bins;
  }
  __device__ __forceinline__ int bin_of(float x) const {
    const float y = place_of(x);
    return y < (float)kBins && x != -INFINITY ? (int)y : kBins;
  }
  __device__ __forceinline__ bool in(const Range& r, float x) const {
    if (r.bin >= 0) return bin_of(x) == r.bin;
    const uint32_t k = key_of(x);
    return k >= r.lo && k <= r.hi;
  }
  // Counts and weights of the range's bins: of keys 2^shift apart, or over the weights' range.
  __device__ __forceinline__ void histogram(const Range& r, bool whole, int shift) {
    __syncthreads();
    for (int i = threadIdx.x; i < kBins; i += kThreads) {
      s.bin.weight[i] = 0;
      s.bin.count[i] = 0;
    }
    __syncthreads();
    row.template all<true, 1>([&](const float* y, int32_t) {
#pragma unroll
      for (int e = 0; e < N; ++e) {
        if (y[e] == -INFINITY || !(whole || in(r, y[e]))) continue;
        const int i = whole ? bin_of(y[e]) : (int)((r.hi - key_of(y[e])) >> shift);
        if (i >= kBins) continue;
        atomicAdd(&s.bin.count[i], 1u);
        atomicAdd(reinterpret_cast<unsigned long long*>(&s.bin.weight[i]), (unsigned long long)weight(y[e]));
      }
    });
    __syncthreads();
  }
  // The first bin at which the count (or the weight) reaches what is missing; count and weight
  // before it are added to `before`, its own count returned.  -1: no bin does.
  struct Sum {
    uint64_t count, weight;
  };
  __device__ __forceinline__ int find_bin(Sum& before, bool by_count, uint64_t target, uint32_t* own) {
    constexpr int M = kBins / kThreads;
    uint64_t c = 0, w = 0;
#pragma unroll
    for (int i = 0; i < M; ++i) {
      c += s.bin.count[threadIdx.x * M + i];
      w += s.bin.weight[threadIdx.x * M + i];
    }
    uint64_t c0 = before.count + block_scan(c, s) - c, w0 = before.weight + block_scan(w, s) - w;
    __syncthreads();
    if (threadIdx.x == 0) s.slot = ~0u;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < M; ++i) {
      const uint64_t ci = s.bin.count[threadIdx.x * M + i], wi = s.bin.weight[threadIdx.x * M + i];
      const uint64_t x = by_count ? c0 : w0, y = by_count ? ci : wi;
      if (x < target && target <= x + y) {
        s.slot = threadIdx.x * M + i;
        s.found[0] = c0;
        s.found[1] = w0;
        s.found[2] = ci;
      }
      c0 += ci;
      w0 += wi;
    }
    __syncthreads();
    const int bin = (int)s.slot;
    if (bin >= 0) {
      before.count = s.found[0];
      before.weight = s.found[1];
      *own = (uint32_t)s.found[2];
    }
    __syncthreads();
    return bin;
  }

  struct Cut {
    float x;
    int32_t index;
    uint64_t weight;      // of all kept tokens
    bool all;             // nothing is cut
  };
  // The cut behind the first `target` tokens, or where their weights reach `target`.
  __device__ __forceinline__ Cut find_cut(bool by_count, uint64_t target) {
    Sum before = {0, 0};
    Range r = {0, 0, 0};
    uint32_t own = 0;
    histogram(r, true, 0);
    r.bin = find_bin(before, by_count, target, &own);
    if (r.bin < 0) return {-INFINITY, 0, 0, true};
    while (own > LIST) {
      // the keys that there are
      __syncthreads();
      if (threadIdx.x == 0) {
        s.lowest = ~0u;
        s.highest = 0;
      }
      __syncthreads();
      uint32_t lo = ~0u, hi = 0;
      row.template all<true, 2>([&](const float* y, int32_t) {
#pragma unroll
        for (int e = 0; e < N; ++e)
          if (y[e] != -INFINITY && in(r, y[e])) {
            const uint32_t k = key_of(y[e]);
            lo = k < lo ? k : lo;
            hi = k > hi ? k : hi;
          }
      });
#pragma unroll
      for (int n = 32; n; n >>= 1) {
        const uint32_t x = (uint32_t)__shfl_xor((int)lo, n, 64), y = (uint32_t)__shfl_xor((int)hi, n, 64);
        lo = x < lo ? x : lo;
        hi = y > hi ? y : hi;
      }
      if ((threadIdx.x & 63) == 0) {
        atomicMin(&s.lowest, lo);
        atomicMax(&s.highest, hi);
      }
      __syncthreads();
      r = {-1, s.lowest, s.highest};
      if (r.lo == r.hi) {       // equal logits: by index
        const float x = of_key(r.lo);
        const uint64_t w = weight(x);
        const uint64_t m = by_count ? target - before.count : (target - before.weight + w - 1) / w;
        const int32_t index = locate(0, row.V, m - 1, [&](float y, int32_t) -> uint64_t { return y == x; });
        return {x, index, before.weight + m * w, false};
      }
      int shift = 0;
      while ((r.hi - r.lo) >> shift >= kBins) ++shift;
      histogram(r, false, shift);
      const int bin = find_bin(before, by_count, target, &own);
      const uint32_t top = r.hi - ((uint32_t)bin << shift);
      r.lo = top - r.lo > (1u << shift) - 1 ? top - ((1u << shift) - 1) : r.lo;
      r.hi = top;
    }
    const Range range = r;
    const int n = gather([&](float x) { return x != -INFINITY && in(range, x); });
    uint64_t sums[kMine];
    order(n, sums);
    const int at = by_count ? (int)(target - before.count) - 1 : reach(n, sums, target - before.weight);
    const uint64_t sum = sum_at(sums, at);
    const uint64_t e = s.list.entry[at];
    return {of_key(~(uint32_t)(e >> 32)), (int32_t)(uint32_t)e, before.weight + sum, false};
  }
};

// Settings of row b once its largest logit is known.
__device__ __forceinline__ Setting setting(const SampleArgs& a, int b, float top, float temperature) {
  Setting set;
  set.top = top;
  set.by = 1.4426950408889634 / (double)temperature;
  // (no more than fp32 holds: where temperatures come near zero the bins are coarser)
  set.bins = fminf(2.0f * (float)kBins / kRange / temperature, 0x1p127f);
  const int32_t k = a.top_k == nullptr ? 0 : a.top_k[b];
  set.k = k > 0 && k < a.V ? k : 0;
  const float p = a.top_p == nullptr ? 1.0f : a.top_p[b];
  set.p = p < 1.0f ? (double)p : 2.0;
  const float min_p = a.min_p == nullptr ? 0.0f : a.min_p[b];
  set.least = min_p > 0.0f ? (uint64_t)ceil((min_p < 1.0f ? (double)min_p : 1.0) * kOne) : 1;
  const float u = a.u[b];
  set.u = u > 0.0f ? (u < 1.0f ? (double)u : 1.0) : 0.0;
  return set;
}
__device__ __forceinline__ float temperature_of(const SampleArgs& a, int b) {
  return a.temperature == nullptr ? 1.0f : a.temperature[b];
}
// Logits of its own that a workgroup's list goes down to: of k spread over the chunks it holds more
// once in 10^5 rows or less (its share plus nine; the row goes by bins then).
__device__ __forceinline__ int listed_of(int k, int chunks) {
  const int m = chunks > 1 ? (2 * k + chunks - 1) / chunks + 9 : k;
  return m < k ? m : k;
}
// Which way a row goes: through the first launch alone, or the first two or three.  By a list where
// the maxima of a workgroup's lanes can say a bound for k (all lists' shares then come to 2 k + 10
// chunks, a third of their room): with k = 50 one row of 131072 takes 20.4 us by a list and 28.6 by
// bins, 512 rows 81 and 284.
enum { kPlain, kByList, kByBins };
__device__ __forceinline__ int way_of(const Setting& set) {
  if (set.k == 0) return set.p > 1.0 ? kPlain : kByBins;
  return set.k <= kThreads / 2 ? kByList : kByBins;
}

template <int DT>
__device__ __forceinline__ Row<DT> row_of(const SampleArgs& a, int b, int per) {
  return Row<DT>(static_cast<const typename Logits<DT>::T*>(a.logits) + b * a.stride, a.V, per);
}

// How a row is shared out.
struct Shape {
  int32_t chunks;      // workgroups
  int32_t subs;        // strips of a wave, one behind the other
  int32_t per;         // vectors of a strip
};

template <int DT, int HELD>
__global__ void __launch_bounds__(kThreads, 3) sample_kernel(SampleArgs a, Space* spaces, Shape shape) {
  using LG = Logits<DT>;
  constexpr int N = LG::N;
  using Z = Sampler<DT, SharedFirst, kShort>;
  __shared__ SharedFirst s;
  put_powers(s);
  const int chunks = shape.chunks, b = blockIdx.x / chunks, chunk = blockIdx.x - b * chunks;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = chunk * kWaves + wave, waves = chunks * kWaves;
  const Row<DT> row = row_of<DT>(a, b, 64);
  Space& space = spaces[b];

  // Vectors are dealt out to the waves sixteen at a time, so that neighbouring tokens, which are
  // often likely together, go to different workgroups.  The first ones of every lane stay in
  // registers.
  const u32x4_t* from = reinterpret_cast<const u32x4_t*>(row.x + row.head);
  const int vectors = (row.vecs + 64 * waves - 1) / (64 * waves);      // of a lane
  auto vector = [&](int i) { return ((i * 4 + (lane >> 4)) * waves + n) * 16 + (lane & 15); };
  u32x4_t q[HELD];
#pragma unroll
  for (int i = 0; i < HELD; ++i)
    if (vector(i) < row.vecs) q[i] = from[vector(i)];
  int32_t loose = n == 0 || n == waves - 1 ? (lane < 2 * N ? row.loose(lane) : -1) : -1;
  if (loose >= 0 && !(loose < row.head ? n == 0 : n == waves - 1)) loose = -1;
  const float single = loose >= 0 ? row.at(loose) : -INFINITY;
  const float temperature = temperature_of(a, b);
  const bool greedy = !(temperature > 0.0f);
  const Setting first_set = setting(a, b, 0.0f, temperature);
  const int way = greedy ? kByList : way_of(first_set);
  // f(N logits, index of the first) for the held ones and those outside whole vectors; for vectors
  // i0 .. i1 - 1 of every lane
  auto held = [&](auto f) {
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
      const int32_t v = vector(i);
      float y[N];
      LG::get(q[i], y);
#pragma unroll
      for (int e = 0; e < N; ++e) y[e] = v < row.vecs ? clean(y[e]) : -INFINITY;
      f(y, row.head + v * N);
    }
    if (n == 0 || n == waves - 1) {
      float y[N];
#pragma unroll
      for (int e = 0; e < N; ++e) y[e] = -INFINITY;
      y[0] = single;
      f(y, loose);
    }
  };
  auto stream = [&](int i0, int i1, auto f) {
    if (i0 >= i1) return;
    constexpr int FLIGHT = 8;
    u32x4_t p[FLIGHT];
    auto load = [&](int i) {
      const int v = vector(i);
      return from[i < i1 && v < row.vecs ? v : 0];
    };
#pragma unroll
    for (int i = 0; i < FLIGHT; ++i) p[i] = load(i0 + i);
    for (int i = i0; i < i1; i += FLIGHT) {
#pragma unroll
      for (int j = 0; j < FLIGHT; ++j) {
        if (i + j >= i1) break;
        const int v = vector(i + j);
        float y[N];
        LG::get(p[j], y);
        p[j] = load(i + j + FLIGHT);
#pragma unroll
        for (int e = 0; e < N; ++e) y[e] = v < row.vecs ? clean(y[e]) : -INFINITY;
        f(y, row.head + v * N);
      }
    }
  };

  float most = -INFINITY;
  auto largest_of = [&](const float* y, int32_t) {
#pragma unroll
    for (int e = 0; e < N; ++e) most = fmaxf(most, y[e]);
  };
  if (way != kByList) {
    float least = INFINITY;
    auto ends_of = [&](const float* y, int32_t at) {
      largest_of(y, at);
#pragma unroll
      for (int e = 0; e < N; ++e) least = fminf(least, y[e] == -INFINITY ? INFINITY : y[e]);
    };
    held(ends_of);
    stream(HELD, vectors, ends_of);
#pragma unroll
    for (int i = 32; i; i >>= 1) {
      most = fmaxf(most, __shfl_xor(most, i, 64));
      least = fminf(least, __shfl_xor(least, i, 64));
    }
    if (lane == 0) {
      space.top[n] = most;
      space.low[n] = least;
    }
    if (way == kByBins && chunks > 1)
      for (int i = chunk * kThreads + (int)threadIdx.x; i < kBins; i += chunks * kThreads) {
        space.weight[i] = 0;
        space.count[i] = 0;
      }
    return;
  }
  if (greedy) {
    uint32_t first = ~0u;
    auto best = [&](const float* y, int32_t at) {
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (y[e] > most || (y[e] == most && (uint32_t)(at + e) < first)) {
          most = y[e];
          first = (uint32_t)(at + e);
        }
    };
    auto over_wave = [&] {
#pragma unroll
      for (int i = 32; i; i >>= 1) {
        const float m = __shfl_xor(most, i, 64);
        const uint32_t f = (uint32_t)__shfl_xor((int)first, i, 64);
        if (m > most || (m == most && f < first)) {
          most = m;
          first = f;
        }
      }
    };
    held(best);
    stream(HELD, vectors, best);
    over_wave();
    if (lane == 0) {
      put(&space.top[n], most);
      put(&space.first[n], first);
    }
    if (!come_last(&space.arrived[0], chunks, s) || threadIdx.x >= 64) return;
    most = -INFINITY;
    first = ~0u;
    for (int i = lane; i < waves; i += 64) {
      const float m = get(&space.top[i]);
      const uint32_t f = get(&space.first[i]);
      if (m > most || (m == most && f < first)) {
        most = m;
        first = f;
      }
    }
    over_wave();
    if (lane == 0) {
      const bool none = most == -INFINITY;
      a.tokens[b] = none ? -1 : (int32_t)first;
      if (a.logprob != nullptr) a.logprob[b] = none ? -INFINITY : 0.0f;
    }
    return;
  }

  // A logit that m of the workgroup's reach: the largest number, to 16 bits, that m of its lanes'
  // maxima so far do.
  const int m = listed_of(first_set.k, chunks);
  auto bound_now = [&] {
    constexpr int M = kThreads / 64;
    __syncthreads();
    s.lanes[threadIdx.x] = most;
    __syncthreads();
    float v[M];
#pragma unroll
    for (int i = 0; i < M; ++i) v[i] = s.lanes[lane + 64 * i];
    uint32_t lo = key_of(-INFINITY), hi = key_of(INFINITY);    // m reach lo
#pragma unroll 1
    for (int step = 0; step < 16; ++step) {
      const uint32_t mid = lo + (hi - lo) / 2;
      const float x = of_key(mid);
      int reach = 0;
#pragma unroll
      for (int i = 0; i < M; ++i) reach += __popcll(__ballot(v[i] >= x));
      if (reach >= m) lo = mid;
      else hi = mid;
    }
    return of_key(lo);
  };
  Z z{row, s, first_set};
  held(largest_of);
  if (threadIdx.x == 0) s.count = s.kept = 0;
  float bound = bound_now();
  auto list = [&](const float* y, int32_t first) {
    z.append(y, first, s.list.entry, &s.count, kShort, [&](float x) { return x >= bound && x != -INFINITY; });
  };
  {       // the held ones at once
    uint32_t mine = 0;
    held([&](const float* y, int32_t) {
#pragma unroll
      for (int e = 0; e < N; ++e) mine += ((y[e] >= bound) & (y[e] != -INFINITY)) ? 1 : 0;
    });
    if (mine > 0) {
      uint32_t at = atomicAdd(&s.count, mine);
      held([&](const float* y, int32_t first) {
#pragma unroll
        for (int e = 0; e < N; ++e)
          if ((y[e] >= bound) & (y[e] != -INFINITY)) {
            if (at < kShort) s.list.entry[at] = (uint64_t)~key_of(y[e]) << 32 | (uint32_t)(first + e);
            ++at;
          }
      });
    }
  }
  for (int i = HELD; i < vectors; i *= 4) {
    stream(i, 4 * i < vectors ? 4 * i : vectors, [&](const float* y, int32_t first) {
      largest_of(y, first);
      list(y, first);
    });
    bound = bound_now();
  }
  float top = most;       // of the wave, for the launches behind
#pragma unroll
  for (int i = 32; i; i >>= 1) top = fmaxf(top, __shfl_xor(top, i, 64));
  if (lane == 0) {
    space.top[n] = top;
    space.low[n] = -INFINITY;
  }
  __syncthreads();
  uint32_t listed = uniform(s.count);
  bool over = listed > kShort;

  constexpr int M = kLong / kThreads;
  auto logit = [](uint64_t e) { return of_key(~(uint32_t)(e >> 32)); };
  uint64_t e[M];       // ~0: none
  // f(e[i]) for those that n entries come to
  auto every = [&](uint32_t n, auto f) {
#pragma unroll
    for (int i = 0; i < M; ++i)
      if ((uint32_t)(i * kThreads) < n) f(e[i], threadIdx.x + i * kThreads);
  };
  if (over) listed = 0;
  every(listed, [&](uint64_t& v, uint32_t j) { v = j < listed ? s.list.entry[j] : ~0ull; });
  float floor = -INFINITY;      // the highest bound of a list
  if (chunks > 1) {       // to all workgroups' list, what reaches the last bound
    uint32_t kept = 0, upto = 0;
    if (vectors > HELD) {
      every(listed, [&](uint64_t& v, uint32_t) {
        if (v != ~0ull && logit(v) < bound) v = ~0ull;
        kept += v != ~0ull;
      });
      upto = (uint32_t)block_scan(kept, s);
    }
    if (threadIdx.x == kThreads - 1) {
      const uint32_t all = over ? kLong + 1u : vectors > HELD ? upto : listed;
      s.slot = __hip_atomic_fetch_add(&space.listed, all, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      put(&space.bound[chunk], bound);
    }
    __syncthreads();
    uint32_t at = s.slot + upto - kept;
    every(listed, [&](uint64_t& v, uint32_t j) {
      if (v == ~0ull) return;
      const uint32_t to = vectors > HELD ? at : at + j;
      if (to < kLong) put(&space.entry[to], v);
      if (vectors > HELD) ++at;
    });
    if (!come_last(&space.arrived[0], chunks, s)) return;
    listed = uniform(get(&space.listed));
    floor = lane < chunks ? get(&space.bound[lane]) : -INFINITY;
    over = listed > kLong;
    every(over ? 0 : listed, [&](uint64_t& v, uint32_t j) { v = j < listed ? get(&space.entry[j]) : ~0ull; });
#pragma unroll
    for (int i = 32; i; i >>= 1) floor = fmaxf(floor, __shfl_xor(floor, i, 64));
    every(over ? 0 : listed, [&](uint64_t& v, uint32_t) {
      if (v != ~0ull && logit(v) < floor) v = ~0ull;
    });
  }
  // their largest and least logits
  uint32_t hi = 0, lo = ~0u;
  every(over ? 0 : listed, [&](uint64_t& v, uint32_t) {
    const uint32_t k = ~(uint32_t)(v >> 32);
    if (v == ~0ull) return;
    hi = k > hi ? k : hi;
    lo = k < lo ? k : lo;
  });
#pragma unroll
  for (int i = 32; i; i >>= 1) {
    const uint32_t x = (uint32_t)__shfl_xor((int)hi, i, 64), y = (uint32_t)__shfl_xor((int)lo, i, 64);
    hi = x > hi ? x : hi;
    lo = y < lo ? y : lo;
  }
  __syncthreads();       // all have read `listed`
  if (threadIdx.x == 0 && chunks > 1) put(&space.listed, 0u);
  if (lane == 0) s.part[wave] = (uint64_t)hi << 32 | lo;
  s.rank[threadIdx.x] = 0;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    hi = (uint32_t)(s.part[w] >> 32) > hi ? (uint32_t)(s.part[w] >> 32) : hi;
    lo = (uint32_t)s.part[w] < lo ? (uint32_t)s.part[w] : lo;
  }
  if (listed == 0 && !over) {      // nothing is allowed
    if (threadIdx.x == 0) {
      space.over = 0;
      a.tokens[b] = -1;
      if (a.logprob != nullptr) a.logprob[b] = -INFINITY;
    }
    return;
  }
  if (!over) {
    // first in the list: all, or those in the bins, of 256 between the two, that hold the first k
    z.set.top = of_key(hi);
    const float scale = (float)kThreads / (z.set.top - of_key(lo));
    auto bin = [&](float x) {      // infinite logits: all in the first
      const float y = (z.set.top - x) * scale;
      return y > 0.0f ? y < (float)kThreads ? (int)y : kThreads - 1 : 0;
    };
    int limit = kThreads;
    if (chunks > 1 || (listed > kThreads / 4 && listed > (uint32_t)z.set.k)) {
      every(listed, [&](uint64_t& v, uint32_t) {
        if (v != ~0ull) atomicAdd(&s.rank[bin(logit(v))], 1u);
      });
      __syncthreads();
      const uint32_t c = s.rank[threadIdx.x], upto = (uint32_t)block_scan(c, s), k = (uint32_t)z.set.k;
      if (threadIdx.x == 0) s.slot = kThreads;
      __syncthreads();
      if (upto >= k && upto - c < k) s.slot = threadIdx.x;
      __syncthreads();
      limit = (int)s.slot;
      // fewer than k above the highest bound: others may be among them that were not listed
      over = limit == kThreads && floor != -INFINITY;
    }
    uint32_t mine = 0;
    every(listed, [&](uint64_t& v, uint32_t) {
      if (v != ~0ull && bin(logit(v)) > limit) v = ~0ull;
      mine += v != ~0ull;
    });
    uint32_t at = mine > 0 ? atomicAdd(&s.kept, mine) : 0;
    every(listed, [&](uint64_t& v, uint32_t) {
      if (v == ~0ull) return;
      if (at < kShort) s.list.entry[at] = v;
      ++at;
    });
    __syncthreads();
    over = over || s.kept > kShort;
  }
  if (threadIdx.x == 0) space.over = over;
  if (over) {       // by bins
    for (int i = threadIdx.x; i < kBins; i += kThreads) {
      space.weight[i] = 0;
      space.count[i] = 0;
    }
    return;
  }
  const int rest = (int)s.kept;
  if (rest <= kFew) {
    z.finish_few(a, b, rest);
    return;
  }
  uint64_t upto[Z::kMine];
  z.order(rest, upto);
  int keep = z.set.k < rest ? z.set.k : rest;
  if (z.set.p <= 1.0) {
    const int reached = z.reach(rest, upto, z.up_to(z.set.p, z.sum_at(upto, keep - 1))) + 1;
    keep = reached < keep ? reached : keep;
  }
  uint64_t strong = 0;      // entries that min-p lets through come first
#pragma unroll
  for (int i = 0; i < Z::kMine; ++i) {
    const int j = threadIdx.x * Z::kMine + i;
    strong += j < rest && s.list.weight[j] >= z.set.least;
  }
  const int allowed = (int)block_sum(strong, s);
  keep = allowed < keep ? allowed : keep;
  z.draw_list(a, b, keep, z.sum_at(upto, keep - 1), z.set.u);
}

// What a row still needs after the first launch; all that says so is loaded at once.
struct Task {
  int way;            // kByList: nothing
  Setting set;
};
__device__ __forceinline__ Task task_of(const SampleArgs& a, int b, const Space& space, int chunks) {
  const int lane = threadIdx.x & 63, waves = chunks * kWaves;
  const float temperature = temperature_of(a, b);
  const int over = space.over;
  float top = -INFINITY, low = INFINITY;
#pragma unroll
  for (int i = 0; i < kStrips / 64; ++i) {
    const bool some = lane + 64 * i < waves;
    top = fmaxf(top, some ? space.top[lane + 64 * i] : -INFINITY);
    low = fminf(low, some ? space.low[lane + 64 * i] : INFINITY);
  }
  Task t;
  t.set = setting(a, b, 0.0f, temperature);
  t.way = !(temperature > 0.0f) ? kByList : way_of(t.set);
  if (t.way == kByList && temperature > 0.0f && over != 0) t.way = kByBins;
#pragma unroll
  for (int i = 32; i; i >>= 1) {
    top = fmaxf(top, __shfl_xor(top, i, 64));
    low = fminf(low, __shfl_xor(low, i, 64));
  }
  t.set.top = top;
  // The bins cover the logits that have a weight, or only those that there are, where the densest
  // bin would not fit a list well: of a normal distribution over 9 deviations it holds 0.4 9 / kBins
  // of the tokens (16 rows of 131072, top-p, T = 100: 41 us; over the weights' range, in whose first
  // bins all tokens are then, 677; but 64 rows of 128257 at ordinary temperatures take 63 with that
  // and 65 with more bins in use).  The lowest logit's is the last; not for differences whose
  // inverse fp32 does not hold.  A few logits far below all others, masked by a finite number, say,
  // leave a row at the weights' range, and at high temperatures one workgroup to narrow it down:
  // 16 rows of 131072, top-p, one in a thousand at -3e4 42 us at T = 10, 647 at 30, 687 at 100.
  const float spread = 0.5f * top - 0.5f * low, range = 0.5f * kRange * temperature;      // of half the logits
  constexpr float kDense = kList * 3 / 4 * (kBins / 3.6f);
  if (spread < range && (float)a.V * range > spread * kDense && spread > 1e-30f) t.set.bins = (float)(kBins - 1) / spread;
  return t;
}

template <int DT>
__global__ void __launch_bounds__(kThreads, 3) sample_weigh_kernel(SampleArgs a, Space* spaces, Shape shape) {
  constexpr int N = Logits<DT>::N;
  using Z = Sampler<DT, SharedWeigh, 0>;
  __shared__ SharedWeigh s;
  put_powers(s);
  const int chunks = shape.chunks, waves = chunks * kWaves, strips = waves * shape.subs;
  const int lane = threadIdx.x & 63;
  for (int item = blockIdx.x; item < a.B * chunks; item += gridDim.x) {
    // the rows that were read last first: what of them is still in the caches
    const int at = item / chunks, b = a.B - 1 - at, chunk = item - at * chunks;
    const int n0 = (chunk * kWaves + (threadIdx.x >> 6)) * shape.subs;      // the wave's first strip
    Space& space = spaces[b];
    const Task task = task_of(a, b, space, chunks);
    if (task.way == kByList) continue;
    if (task.set.top == -INFINITY) {
      if (chunk == 0 && threadIdx.x == 0) {
        space.state.mode = kDone;
        a.tokens[b] = -1;
        if (a.logprob != nullptr) a.logprob[b] = -INFINITY;
      }
      continue;
    }
    __syncthreads();       // the last row's LDS is free
    Z z{row_of<DT>(a, b, shape.per), s, task.set};
    const Setting& set = z.set;
    if (task.way == kPlain) {
      auto weight = [&](float x, int32_t) -> uint64_t {
        const uint64_t w = z.weight(x);
        return w >= set.least ? w : 0;
      };
      for (int n = n0; n < n0 + shape.subs; ++n) {
        uint64_t sum = 0;
        z.row.template of_strip<true, 4>(n, strips, [&](const float* y, int32_t i) {
#pragma unroll
          for (int e = 0; e < N; ++e) sum += weight(y[e], i);
        });
        sum = wave_sum(sum);
        if (lane == 0) put(&space.sum[n], sum);
      }
      if (!come_last(&space.arrived[1], chunks, s)) continue;
      if ((int)threadIdx.x < strips) s.strip[threadIdx.x] = get(&space.sum[threadIdx.x]);
      __syncthreads();
      z.draw_strips(a, b, strips, set.u, weight);
      continue;
    }

    // a histogram of the strips of this workgroup, then of all
    for (int i = threadIdx.x; i < kBins; i += kThreads) {
      s.bin.weight[i] = 0;
      s.bin.count[i] = 0;
    }
    __syncthreads();
    for (int n = n0; n < n0 + shape.subs; ++n)
      z.row.template of_strip<true, 4>(n, strips, [&](const float* y, int32_t) {
        uint64_t w[N];
#pragma unroll
        for (int e = 0; e < N; ++e) w[e] = z.weight(y[e]);
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const int i = z.bin_of(y[e]);
          if (i >= kBins) continue;
          atomicAdd(&s.bin.count[i], 1u);
          atomicAdd(reinterpret_cast<unsigned long long*>(&s.bin.weight[i]), (unsigned long long)w[e]);
        }
      });
    __syncthreads();
    if (chunks > 1) {
      for (int i = threadIdx.x; i < kBins; i += kThreads) {
        if (s.bin.count[i] == 0) continue;
        __hip_atomic_fetch_add(&space.count[i], s.bin.count[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __hip_atomic_fetch_add(&space.weight[i], s.bin.weight[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      }
      if (!come_last(&space.arrived[1], chunks, s)) continue;
      constexpr int M = kBins / kThreads;
      uint64_t w[M];
      uint32_t c[M];
#pragma unroll
      for (int i = 0; i < M; ++i) {
        w[i] = get(&space.weight[threadIdx.x + i * kThreads]);
        c[i] = get(&space.count[threadIdx.x + i * kThreads]);
      }
#pragma unroll
      for (int i = 0; i < M; ++i) {
        s.bin.weight[threadIdx.x + i * kThreads] = w[i];
        s.bin.count[threadIdx.x + i * kThreads] = c[i];
      }
      __syncthreads();
    }
    z.plan(space.state);
  }
}

template <int DT>
__global__ void __launch_bounds__(kThreads) sample_cut_kernel(SampleArgs a, Space* spaces, Shape shape) {
  using Z = Sampler<DT, SharedCut, kList>;
  constexpr int N = Logits<DT>::N;
  __shared__ SharedCut s;
  put_powers(s);
  const int chunks = shape.chunks, waves = chunks * kWaves, strips = waves * shape.subs;
  const int lane = threadIdx.x & 63;
  for (int item = blockIdx.x; item < a.B * chunks; item += gridDim.x) {
    const int b = item / chunks, chunk = item - b * chunks;
    const int n0 = (chunk * kWaves + (threadIdx.x >> 6)) * shape.subs;      // the wave's first strip
    Space& space = spaces[b];
    const State st = space.state;
    const Task task = task_of(a, b, space, chunks);
    if (task.way != kByBins) continue;
    if (st.mode == kDone || (st.mode == kNarrow && chunk != 0)) continue;
    __syncthreads();       // the last row's LDS is free
    Z z{row_of<DT>(a, b, shape.per), s, task.set};
    const Setting& set = z.set;
    typename Z::Cut cut = {-INFINITY, 0, 0, true};
    auto kept = [&](float x, int32_t i) -> uint64_t {
      const uint64_t w = z.weight(x);
      const bool in = (x > cut.x) | ((x == cut.x) & (cut.all | (i <= cut.index)));
      return (in & (w >= set.least)) ? w : 0;
    };
    uint64_t sum = 0;

    if (st.mode == kNarrow) {
      for (int stage = set.k > 0 ? 0 : 1; stage < (set.p <= 1.0 ? 2 : 1); ++stage) {      // top-k, top-p
        uint64_t target = (uint64_t)set.k;
        if (stage == 1) {
          uint64_t total = cut.weight;
          if (cut.all) {
            sum = 0;
            z.row.template all<true, 1>([&](const float* y, int32_t) {
#pragma unroll
              for (int e = 0; e < N; ++e) sum += y[e] == -INFINITY ? 0 : z.weight(y[e]);
            });
            total = block_sum(sum, s);
          }
          target = z.up_to(set.p, total);
        }
        cut = z.find_cut(stage == 0, target);
      }
      __syncthreads();
      for (int m = threadIdx.x >> 6; m < strips; m += kWaves) {
        sum = 0;
        z.row.template of_strip<true, 1>(m, strips, [&](const float* y, int32_t first) {
#pragma unroll
          for (int e = 0; e < N; ++e)
            if (y[e] != -INFINITY) sum += kept(y[e], first + e);
        });
        sum = wave_sum(sum);
        if (lane == 0) s.strip[m] = sum;
      }
      __syncthreads();
      z.draw_strips(a, b, strips, set.u, kept);
      continue;
    }

    if (threadIdx.x == 0) s.count = 0;
    __syncthreads();
    for (int n = n0; n < n0 + shape.subs; ++n) {
      sum = 0;
      z.row.template of_strip<true, 4>(n, strips, [&](const float* y, int32_t first) {
        bool some = false;
#pragma unroll
        for (int e = 0; e < N; ++e) some |= z.bin_of(y[e]) < st.above;
        if (__any(some)) {
#pragma unroll
          for (int e = 0; e < N; ++e) {
            const uint64_t w = kept(y[e], first + e);
            sum += z.bin_of(y[e]) < st.above ? w : 0;
          }
        }
        z.append(y, first, s.list.entry, &s.count, kList, [&](float x) {
          const int i = z.bin_of(x);
          return i < kBins && ((i >= st.above && i <= st.upto) || i == st.at_k);
        });
      });
      sum = wave_sum(sum);
      if (lane == 0) put(&space.sum[n], sum);
    }
    __syncthreads();
    const uint32_t mine = s.count;       // no more than the plan has counted, which fits
    if (threadIdx.x == 0)
      s.slot = mine == 0 ? 0 : __hip_atomic_fetch_add(&space.listed, mine, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < mine; i += kThreads) put(&space.entry[s.slot + i], s.list.entry[i]);
    if (!come_last(&space.arrived[2], chunks, s)) continue;
    const int listed = (int)get(&space.listed);
    {
      uint64_t e[kList / kThreads];
#pragma unroll
      for (int i = 0; i < kList / kThreads; ++i)
        e[i] = (int)threadIdx.x + i * kThreads < listed ? get(&space.entry[threadIdx.x + i * kThreads]) : 0;
      for (int i = 0; i < kList / kThreads; ++i) {
        const int at = threadIdx.x + i * kThreads;
        if (at < listed) s.list.entry[at] = e[i];
      }
      __syncthreads();
      for (int i = threadIdx.x; i < listed; i += kThreads)
        s.list.weight[i] = z.weight(of_key(~(uint32_t)(s.list.entry[i] >> 32)));
    }
    __syncthreads();       // all have read `listed`
    if (threadIdx.x == 0) put(&space.listed, 0u);
    uint64_t last = ~0ull;
    if (listed > 0) {
      uint64_t total = st.total;
#pragma unroll 1
      for (int stage = st.at_k >= 0 ? 0 : 1; stage < (set.p <= 1.0 ? 2 : 1); ++stage) {      // top-k, top-p
        const uint64_t t = z.up_to(set.p, total);
        const uint64_t target = stage == 0 ? (uint32_t)set.k - st.before_k : t > st.weight_above ? t - st.weight_above : 1;
        const typename Z::Picked to = z.pick(listed, stage == 0 ? st.at_k : st.above, stage == 0 ? st.at_k : st.upto, stage == 0, target);
        if (stage == 0) total = st.weight_k + to.sum;
        last = to.entry;
      }
      cut = {of_key(~(uint32_t)(last >> 32)), (int32_t)(uint32_t)last, 0, false};
    }
    if ((int)threadIdx.x < strips) s.strip[threadIdx.x] = get(&space.sum[threadIdx.x]);
    __syncthreads();
    for (int i = threadIdx.x; i < listed; i += kThreads) {
      const uint64_t e = s.list.entry[i], w = s.list.weight[i];
      if (e <= last && w >= set.least)
        atomicAdd(reinterpret_cast<unsigned long long*>(&s.strip[z.row.strip_of((int32_t)(uint32_t)e, strips)]),
                  (unsigned long long)w);
    }
    __syncthreads();
    z.draw_strips(a, b, strips, set.u, kept);
  }
}

// Workgroups of a row: as many as fill the chip, of kHeld vectors a lane at least.  With 512 of them
// 64 rows of 128257 with settings of their own take 79 us instead of 63 (512 rows by lists 85 instead
// of 81, 64 rows by lists 33 instead of 35), with 2048 the 512 rows take 102.  A list's first bound is
// from twice as many vectors where a lane has them: 64 rows of 131072 by lists take 34.7 us instead of
// 36.8; loaded for nothing where it has fewer they cost one row 1 us and the 64 rows with settings 3.
constexpr int kFill = 1024;
template <int DT>
hipError_t launch(const SampleArgs& a, void* ws, hipStream_t stream) {
  const int vecs = a.V / Logits<DT>::N, part = kHeld * kThreads, most = (vecs + part - 1) / part;
  Shape shape;
  shape.chunks = kFill / a.B < most ? kFill / a.B : most;
  shape.chunks = shape.chunks < 1 ? 1 : shape.chunks < kStrips / kWaves ? shape.chunks : kStrips / kWaves;
  const int waves = shape.chunks * kWaves, of_wave = (vecs + waves - 1) / waves;
  shape.subs = 1;
  while (2 * shape.subs * waves <= kStrips && of_wave >= 2 * shape.subs * 64 * kHeld) shape.subs *= 2;
  shape.per = ((of_wave + shape.subs - 1) / shape.subs + 63) / 64 * 64;
  shape.per = shape.per > 0 ? shape.per : 64;
  Space* spaces = static_cast<Space*>(ws);
  const dim3 grid((unsigned)(a.B * shape.chunks)), some((unsigned)(a.B * shape.chunks < kFill ? a.B * shape.chunks : kFill)),
      block(kThreads);
  if (vecs >= shape.chunks * kThreads * 2 * kHeld)
    hipLaunchKernelGGL((sample_kernel<DT, 2 * kHeld>), grid, block, 0, stream, a, spaces, shape);
  else
    hipLaunchKernelGGL((sample_kernel<DT, kHeld>), grid, block, 0, stream, a, spaces, shape);
  hipLaunchKernelGGL((sample_weigh_kernel<DT>), some, block, 0, stream, a, spaces, shape);
  if (a.top_k != nullptr || a.top_p != nullptr)      // else every row is answered by now
    hipLaunchKernelGGL((sample_cut_kernel<DT>), some, block, 0, stream, a, spaces, shape);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_sample(const SampleArgs& a, int dtype, void* ws, hipStream_t stream) {
  return dtype == 0 ? launch<0>(a, ws, stream) : launch<1>(a, ws, stream);
}

size_t sample_ws_bytes(int B) { return (size_t)B * sizeof(Space); }

}  // namespace kvx
