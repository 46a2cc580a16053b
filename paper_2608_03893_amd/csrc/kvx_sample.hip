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
// A workgroup takes a row.  Pass 1 finds the largest logit, and a bound that at least k logits
// reach: the least, over the waves, of the m-th largest maximum of a lane's logits.  Pass 2
// gathers the logits from that bound on into LDS, where they are sorted and cut.  Without top-k
// the bound is a guess, and pass 2 sums all weights to see whether the list holds enough of
// them.  Where the list is too short or too long, the cut is found by histograms of 2048 bins
// over the weights' range, and the draw takes sums over the whole row.
#include "kvx_bf16.h"
#include "kvx_serve.h"

namespace kvx {
namespace {

constexpr int kThreads = 512, kWaves = kThreads / 64;
constexpr int kList = 4096;                // most tokens sorted in LDS
constexpr int kBins = 2048;
constexpr int kFraction = 43;              // bits of a weight behind the point
constexpr double kOne = 8796093022208.0;   // 2^43: the best token's weight
constexpr float kRange = 30.5f;            // 44 ln 2: what a weight of 2^-44 is below the best, over T
static_assert(kList % kThreads == 0, "a thread's entries of the list");

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

__device__ __forceinline__ float clean(float x) { return x == x ? x : -INFINITY; }   // NaN: not allowed

// Rising with x, equal for the two zeros.
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t u = __float_as_uint(x + 0.0f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float of_key(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }

// 2^43 times exp((x - top) / T), to the nearest whole number; by = log2(e) / T.
__device__ __forceinline__ uint64_t weight_of(float x, float top, double by) {
  const double y = x == top ? 0.0 : ((double)x - (double)top) * by;
  if (!(y > -45.0)) return 0;
  const double n = rint(y), t = (y - n) * 0.69314718055994530942;
  double p = 1.0 / 39916800.0;      // the exponential's series to t^11: 6e-15
  p = __builtin_fma(p, t, 1.0 / 3628800.0);
  p = __builtin_fma(p, t, 1.0 / 362880.0);
  p = __builtin_fma(p, t, 1.0 / 40320.0);
  p = __builtin_fma(p, t, 1.0 / 5040.0);
  p = __builtin_fma(p, t, 1.0 / 720.0);
  p = __builtin_fma(p, t, 1.0 / 120.0);
  p = __builtin_fma(p, t, 1.0 / 24.0);
  p = __builtin_fma(p, t, 1.0 / 6.0);
  p = __builtin_fma(p, t, 0.5);
  p = __builtin_fma(p, t, 1.0);
  p = __builtin_fma(p, t, 1.0);
  // the sum with 2^52 has the rounded number in its low bits
  const double r = ldexp(p, (int)n + kFraction) + 4503599627370496.0;
  return __builtin_bit_cast(uint64_t, r) & 0xfffffffffffffull;
}

__device__ __forceinline__ uint64_t wave_sum(uint64_t v) {
#pragma unroll
  for (int n = 32; n; n >>= 1) v += (uint64_t)__shfl_xor((unsigned long long)v, n, 64);
  return v;
}
__device__ __forceinline__ uint64_t wave_scan(uint64_t v, int lane) {   // inclusive
#pragma unroll
  for (int n = 1; n < 64; n <<= 1) {
    const uint64_t u = (uint64_t)__shfl_up((unsigned long long)v, n, 64);
    if (lane >= n) v += u;
  }
  return v;
}

// A row's settings, restrictions that cannot bind switched off.
struct Setting {
  float top;            // its largest logit
  double by;            // log2(e) / T
  float bins;           // of the histogram, a unit of the logits
  uint64_t least;       // weight that min-p asks for
  int32_t k;            // 0: all
  double p;             // 2: all
};

template <int DT>
struct Row {
  using LG = Logits<DT>;
  using T = typename LG::T;
  const T* x;
  int32_t V, head, vecs;      // logits before the first 16-byte boundary, whole vectors behind it
  __device__ __forceinline__ Row(const T* from, int32_t v) : x(from), V(v) {
    head = (int32_t)(-(reinterpret_cast<uintptr_t>(from) / sizeof(T)) & (LG::N - 1));
    head = head < V ? head : V;
    vecs = (V - head) / LG::N;
  }
  __device__ __forceinline__ float at(int32_t i) const { return clean(LG::one(x[i])); }
  // f(logits, their number, index of the first) for every vector of v0 .. v1 - 1 that thread `me`
  // of `n` has, from the last on where BACK: what was read last is still in the caches.  FLIGHT:
  // loads of a thread on the way
  template <bool BACK, int FLIGHT, typename F>
  __device__ __forceinline__ void vectors(int v0, int v1, int me, int n, F f) const {
    const u32x4_t* from = reinterpret_cast<const u32x4_t*>(x + head);
    const int steps = (v1 - v0 + n - 1) / n;
    for (int s = 0; s < steps; s += FLIGHT) {
      u32x4_t q[FLIGHT];
      int v[FLIGHT];
#pragma unroll
      for (int i = 0; i < FLIGHT; ++i) {
        v[i] = v0 + (BACK ? steps - 1 - s - i : s + i) * n + me;
        if (s + i >= steps || v[i] >= v1) v[i] = -1;
        q[i] = from[v[i] < 0 ? v0 : v[i]];
      }
#pragma unroll
      for (int i = 0; i < FLIGHT; ++i) {
        float y[LG::N];
        LG::get(q[i], y);
#pragma unroll
        for (int e = 0; e < LG::N; ++e) y[e] = v[i] < 0 ? -INFINITY : clean(y[e]);
        f(y, head + v[i] * LG::N);
      }
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

struct Shared {
  union {
    struct {
      uint64_t weight[kBins];
      uint32_t count[kBins];
    } bin;
    struct {
      uint64_t entry[kList];       // ~key, index: rises in the order of the tokens
      uint64_t weight[kList];
    } list;
  };
  uint64_t part[kWaves];
  float fpart[kWaves];
  uint32_t count, lowest, highest, slot;
  uint64_t found[4];
};

__device__ __forceinline__ uint64_t block_sum(uint64_t v, Shared& s) {
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
__device__ __forceinline__ uint64_t block_scan(uint64_t v, Shared& s) {
  const int wave = threadIdx.x >> 6;
  v = wave_scan(v, threadIdx.x & 63);
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

template <int DT>
struct Sampler {
  const Row<DT> row;
  Shared& s;
  Setting set;
  static constexpr int N = Logits<DT>::N;

  __device__ __forceinline__ uint64_t weight(float x) const { return weight_of(x, set.top, set.by); }

  // Gathers the tokens that `take` accepts, as entries; returns their number, which may exceed
  // the list (which then holds some of them).  more(x): whatever else a pass does.
  template <int FLIGHT, typename F, typename M>
  __device__ __forceinline__ int gather(F take, M more) {
    __syncthreads();
    if (threadIdx.x == 0) s.count = 0;
    __syncthreads();
    row.template all<true, FLIGHT>([&](const float* y, int32_t first) {
      more(y);
      bool some = false;
#pragma unroll
      for (int e = 0; e < N; ++e) some |= take(y[e]);
      if (!__any(some)) return;
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const bool mine = take(y[e]);
        const uint64_t who = __ballot(mine);
        if (who == 0) continue;
        uint32_t at = 0;
        const int lane = threadIdx.x & 63;
        if (lane == __builtin_ctzll(who)) at = atomicAdd(&s.count, (uint32_t)__popcll(who));
        at = (uint32_t)__shfl((int)at, __builtin_ctzll(who), 64) + (uint32_t)__popcll(who & ((1ull << lane) - 1));
        if (mine && at < kList) s.list.entry[at] = (uint64_t)~key_of(y[e]) << 32 | (uint32_t)(first + e);
      }
    });
    __syncthreads();
    return (int)s.count;
  }

  // Entries in order and their weights; a thread gets the sums up to each of its entries
  // (kList / kThreads neighbouring ones).
  static constexpr int kMine = kList / kThreads;
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
  __device__ __forceinline__ static uint64_t up_to(double p, uint64_t total) {     // what top-p's sum has to reach
    const double t = ceil(p * (double)total);
    return t < 1.0 ? 1 : t < (double)total ? (uint64_t)t : total;
  }
  __device__ __forceinline__ static uint64_t behind(double u, uint64_t total) {    // what the draw's sum has to exceed
    const uint64_t t = (uint64_t)(u * (double)total);
    return t < total ? t : total - 1;
  }

  __device__ __forceinline__ void put(const SampleArgs& a, int b, int32_t token, float x, uint64_t total) {
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
        put(a, b, token, row.at(token), total);
      }
      sum += w[i];
    }
  }

  // The place in lo .. hi - 1 at which the sum of f over it, in order of the vocabulary, first
  // exceeds t (less than all of it).
  template <typename F>
  __device__ __forceinline__ int32_t locate(int32_t lo, int32_t hi, uint64_t t, F f) {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    while (hi - lo > kThreads) {
      const int32_t per = ((hi - lo + kWaves - 1) / kWaves + 63) / 64 * 64;
      uint64_t sum = 0;
      const int32_t a = lo + wave * per, z = a + per < hi ? a + per : hi;
      for (int32_t i = a + lane; i < z; i += 64) sum += f(row.at(i), i);
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
    const int32_t i = lo + (int32_t)threadIdx.x;
    const uint64_t v = i < hi ? f(row.at(i), i) : 0, sum = block_scan(v, s);
    if (v > 0 && sum - v <= t && t < sum) s.slot = (uint32_t)i;
    __syncthreads();
    return (int32_t)s.slot;
  }

  // Sums of f over the whole row, each wave's part of it in order of the vocabulary; then the
  // draw from them.
  template <typename F>
  __device__ __forceinline__ void draw_row(const SampleArgs& a, int b, double u, F f) {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int per = ((row.vecs + kWaves - 1) / kWaves + 63) / 64 * 64;
    const int v0 = wave * per < row.vecs ? wave * per : row.vecs, v1 = v0 + per < row.vecs ? v0 + per : row.vecs;
    // its logits: whole vectors, the loose ones at both ends with the first and the last wave
    const int32_t lo = wave == 0 ? 0 : row.head + v0 * N, hi = wave == kWaves - 1 ? row.V : row.head + v1 * N;
    uint64_t sum = 0;
    if (v0 < v1)
      row.template vectors<true, 1>(v0, v1, lane, 64, [&](const float* y, int32_t first) {
#pragma unroll
        for (int e = 0; e < N; ++e)
          if (y[e] != -INFINITY) sum += f(y[e], first + e);
      });
    if (wave == 0 || wave == kWaves - 1) {
      const int32_t i = lane < 2 * N ? row.loose(lane) : -1;
      if (i >= 0 && (wave == 0) == (i < row.head)) sum += f(row.at(i), i);
    }
    sum = wave_sum(sum);
    __syncthreads();
    if (lane == 0) s.part[wave] = sum;
    __syncthreads();
    uint64_t total = 0;
    for (int w = 0; w < kWaves; ++w) total += s.part[w];
    uint64_t t = behind(u, total);
    int w = 0;
    while (w < kWaves - 1 && t >= s.part[w]) t -= s.part[w++];
    __syncthreads();
    if (wave == w && lane == 0) {
      s.found[1] = (uint64_t)lo;
      s.found[2] = (uint64_t)hi;
    }
    __syncthreads();
    const int32_t token = locate((int32_t)s.found[1], (int32_t)s.found[2], t, f);
    if (threadIdx.x == 0) put(a, b, token, row.at(token), total);
  }

  // ---- the cut by histograms ----

  // A range of logits: those of one bin over the weights' range, or of keys lo .. hi.
  struct Range {
    int bin;               // -1: by keys
    uint32_t lo, hi;
  };
  __device__ __forceinline__ int bin_of(float x) const {
    const float y = x == set.top ? 0.0f : (set.top - x) * set.bins;    // rises as x falls
    return y < (float)kBins ? (int)y : kBins;
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
    while (own > kList) {
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
    const int n = gather<2>([&](float x) { return x != -INFINITY && in(range, x); }, [](const float*) {});
    uint64_t sums[kMine];
    order(n, sums);
    const int at = by_count ? (int)(target - before.count) - 1 : reach(n, sums, target - before.weight);
    const uint64_t sum = sum_at(sums, at);
    const uint64_t e = s.list.entry[at];
    return {of_key(~(uint32_t)(e >> 32)), (int32_t)(uint32_t)e, before.weight + sum, false};
  }
};

template <int DT>
__global__ void __launch_bounds__(kThreads) sample_kernel(SampleArgs a) {
  using LG = Logits<DT>;
  constexpr int N = LG::N;
  __shared__ Shared s;
  const int b = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const Row<DT> row(static_cast<const typename LG::T*>(a.logits) + b * a.stride, a.V);
  const float temperature = a.temperature == nullptr ? 1.0f : a.temperature[b];
  const bool greedy = !(temperature > 0.0f);

  // pass 1: the largest logit
  float most = -INFINITY;
  row.template all<false, 4>([&](const float* y, int32_t) {
#pragma unroll
    for (int e = 0; e < N; ++e) most = fmaxf(most, y[e]);
  });
  float top = most;
#pragma unroll
  for (int n = 32; n; n >>= 1) top = fmaxf(top, __shfl_xor(top, n, 64));
  if (lane == 0) s.fpart[wave] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWaves; ++w) top = fmaxf(top, s.fpart[w]);
  if (top == -INFINITY) {      // nothing is allowed
    if (threadIdx.x == 0) {
      a.tokens[b] = -1;
      if (a.logprob != nullptr) a.logprob[b] = -INFINITY;
    }
    return;
  }
  if (greedy) {
    if (threadIdx.x == 0) s.lowest = ~0u;
    __syncthreads();
    uint32_t first = ~0u;
    row.template all<true, 2>([&](const float* y, int32_t at) {
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (y[e] == top && (uint32_t)(at + e) < first) first = (uint32_t)(at + e);
    });
    if (first != ~0u) atomicMin(&s.lowest, first);
    __syncthreads();
    if (threadIdx.x == 0) {
      a.tokens[b] = (int32_t)s.lowest;
      if (a.logprob != nullptr) a.logprob[b] = 0.0f;
    }
    return;
  }

  Setting set;
  set.top = top;
  set.by = 1.4426950408889634 / (double)temperature;
  set.bins = (float)kBins / kRange / temperature;
  const int32_t k = a.top_k == nullptr ? 0 : a.top_k[b];
  set.k = k > 0 && k < a.V ? k : 0;
  const float p = a.top_p == nullptr ? 1.0f : a.top_p[b];
  set.p = p < 1.0f ? (double)p : 2.0;
  const float min_p = a.min_p == nullptr ? 0.0f : a.min_p[b];
  set.least = min_p > 0.0f ? (uint64_t)ceil((min_p < 1.0f ? (double)min_p : 1.0) * kOne) : 1;
  float r = a.u[b];
  const double u = r > 0.0f ? (r < 1.0f ? (double)r : 1.0) : 0.0;
  const bool by_p = set.p <= 1.0;
  Sampler<DT> z{row, s, set};

  if (set.k == 0 && !by_p) {
    z.draw_row(a, b, u, [&](float x, int32_t) -> uint64_t {
      const uint64_t w = z.weight(x);
      return w >= set.least ? w : 0;
    });
    return;
  }
  uint64_t sum = 0;
  auto add = [&](const float* y) {
#pragma unroll
    for (int e = 0; e < N; ++e) sum += y[e] == -INFINITY ? 0 : z.weight(y[e]);
  };
  if (set.k <= 512) {
    // the m-th largest of a wave's lanes, the least of which at least k logits reach
    const int m = set.k > 0 ? (set.k + kWaves - 1) / kWaves : 16;
    float v = most;
#pragma unroll
    for (int size = 2; size <= 64; size <<= 1)
#pragma unroll
      for (int j = size >> 1; j; j >>= 1) {
        const float o = __shfl_xor(v, j, 64);
        const bool larger = ((lane & j) == 0) == ((lane & size) == 0);
        v = larger ? fmaxf(v, o) : fminf(v, o);
      }
    v = __shfl(v, m - 1, 64);
    __syncthreads();
    if (lane == 0) s.fpart[wave] = v;
    __syncthreads();
    float bound = s.fpart[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) bound = fminf(bound, s.fpart[w]);
    const bool sums = set.k == 0;
    auto take = [&](float x) { return x >= bound && x != -INFINITY; };
    const int n = sums ? z.template gather<1>(take, add) : z.template gather<4>(take, [](const float*) {});
    if (n <= kList) {
      if (sums) sum = block_sum(sum, s);
      uint64_t upto[Sampler<DT>::kMine];
      z.order(n, upto);
      int keep = set.k > 0 && set.k < n ? set.k : n;
      bool enough = true;
      if (by_p) {
        const uint64_t total = sums ? sum : z.sum_at(upto, keep - 1);
        const int at = z.reach(n, upto, z.up_to(set.p, total));
        enough = at < n;
        keep = at + 1 < keep ? at + 1 : keep;
      }
      if (enough) {
        uint64_t strong = 0;      // entries that min-p lets through come first
#pragma unroll
        for (int i = 0; i < Sampler<DT>::kMine; ++i) {
          const int at = threadIdx.x * Sampler<DT>::kMine + i;
          strong += at < n && s.list.weight[at] >= set.least;
        }
        const int most_p = (int)block_sum(strong, s);
        keep = most_p < keep ? most_p : keep;
        z.draw_list(a, b, keep, z.sum_at(upto, keep - 1), u);
        return;
      }
    }
  }
  typename Sampler<DT>::Cut cut = {-INFINITY, 0, 0, true};
  for (int stage = set.k > 0 ? 0 : 1; stage < (by_p ? 2 : 1); ++stage) {      // top-k, top-p
    uint64_t target = (uint64_t)set.k;
    if (stage == 1) {
      uint64_t total = cut.weight;
      if (cut.all) {
        sum = 0;
        row.template all<true, 1>([&](const float* y, int32_t) { add(y); });
        total = block_sum(sum, s);
      }
      target = z.up_to(set.p, total);
    }
    cut = z.find_cut(stage == 0, target);
  }
  z.draw_row(a, b, u, [&](float x, int32_t i) -> uint64_t {
    if (!(x > cut.x || (x == cut.x && (cut.all || i <= cut.index)))) return 0;
    const uint64_t w = z.weight(x);
    return w >= set.least ? w : 0;
  });
}

}  // namespace

hipError_t launch_sample(const SampleArgs& a, int dtype, void* ws, hipStream_t stream) {
  if (dtype == 0)
    hipLaunchKernelGGL((sample_kernel<0>), dim3(a.B), dim3(kThreads), 0, stream, a);
  else
    hipLaunchKernelGGL((sample_kernel<1>), dim3(a.B), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

size_t sample_ws_bytes(int B, int V, int dtype) { return 0; }

}  // namespace kvx
