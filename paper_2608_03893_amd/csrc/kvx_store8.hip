// 8-bit store: packed rows into the pool of e4m3 codes, a power-of-two scale for each
// (layer, K|V, head, page).
//
// Codes are x / s for the page's s = 2^j >= amax / 448.  Division by a power of two is
// exact, so a code carries one rounding (e4m3's), the same whether the page was written
// at once or token by token, unless its scale grew and a code fell below e4m3's least
// normal value.
//
// Bound by memory: 2 or 4 bytes read and one written per element.  Measured, bf16, d = 128, 8
// heads: 8192 rows of 64 layers 560 to 610 us (5.3 to 5.8 TB/s read and written, whatever the
// pages; a copy reaches 4.7), 333 rows of 40 layers 18.7 us (4.4), 64 rows of one 3.3 us.
#include "kvx_e4m3.h"
#include "kvx_serve.h"

namespace kvx {
namespace {

constexpr int kWaves = 4;

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int n = 32; n; n >>= 1) v = fmaxf(v, __shfl_xor(v, n, 64));
  return v;
}

// 16 bytes of a row as floats: 8 of bf16, 4 of fp32.
template <int DT>
struct Vec;
template <>
struct Vec<0> {
  static constexpr int N = 8;
  uint4 q;
  __device__ float amax() const {
    float m = 0.0f;
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) m = fmaxf(m, fmaxf(finite_abs(lo_bf16(w[i])), finite_abs(hi_bf16(w[i]))));
    return m;
  }
  __device__ void put(uint8_t* to, float r) const {
    uint2 c;
    c.x = to_e4m3x4(lo_bf16(q.x), hi_bf16(q.x), lo_bf16(q.y), hi_bf16(q.y), r);
    c.y = to_e4m3x4(lo_bf16(q.z), hi_bf16(q.z), lo_bf16(q.w), hi_bf16(q.w), r);
    *reinterpret_cast<uint2*>(to) = c;
  }
};
template <>
struct Vec<1> {
  static constexpr int N = 4;
  uint4 q;
  __device__ float amax() const {
    return fmaxf(fmaxf(finite_abs(__uint_as_float(q.x)), finite_abs(__uint_as_float(q.y))),
                 fmaxf(finite_abs(__uint_as_float(q.z)), finite_abs(__uint_as_float(q.w))));
  }
  __device__ void put(uint8_t* to, float r) const {
    *reinterpret_cast<uint32_t*>(to) = to_e4m3x4(__uint_as_float(q.x), __uint_as_float(q.y),
                                                 __uint_as_float(q.z), __uint_as_float(q.w), r);
  }
};

// Rows s .. e - 1 of a page by one wave: the largest value, the scale, the codes.  LOADS
// times ROWS rows stay in registers between the two; more are read again, from L2.
template <int DT, int D, int LOADS, typename T>
__device__ __forceinline__ void store_page(const StoreArgs& a, const T* x, int64_t ts, uint8_t* codes, float* scales,
                                           int s, int e, uint32_t first, float old) {
  constexpr int E = Vec<DT>::N, LANES = D / E, ROWS = 64 / LANES;   // lanes a row, rows a load
  const int lane = threadIdx.x & 63, sub = lane / LANES;
  const int P = 1 << a.log2p, held = first & (P - 1);               // earlier rows of the page
  const uint32_t page = first >> a.log2p;
  Vec<DT> v[LOADS];
  uint32_t slot[LOADS];
  auto load = [&](int t0) {
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int t = t0 + i * ROWS + sub < e ? t0 + i * ROWS + sub : e - 1;   // the last row again
      v[i].q = *reinterpret_cast<const uint4*>(x + t * ts);
      slot[i] = (uint32_t)a.slots[t];
    }
  };
  float m = 0.0f;
  for (int t0 = s; t0 < e; t0 += LOADS * ROWS) {
    load(t0);
#pragma unroll
    for (int i = 0; i < LOADS; ++i) m = fmaxf(m, v[i].amax());
  }
  float scale = pow2_scale(wave_max(m));
  if (held > 0) {
    if (old < scale) {
      const float r = old / scale;
      uint8_t* c = codes + (int64_t)page * P * D;
      for (int i = 16 * lane; i < held * D; i += 1024) {
        uint4 q = *reinterpret_cast<const uint4*>(c + i);
        uint32_t* w = reinterpret_cast<uint32_t*>(&q);
#pragma unroll
        for (int j = 0; j < 4; ++j)
          w[j] = to_e4m3x4(from_e4m3<0>(w[j]), from_e4m3<1>(w[j]), from_e4m3<2>(w[j]), from_e4m3<3>(w[j]), r);
        *reinterpret_cast<uint4*>(c + i) = q;
      }
    } else {
      scale = old;
    }
  }
  if (lane == 0) scales[page] = scale;
  const float r = 1.0f / scale;
  for (int t0 = s; t0 < e; t0 += LOADS * ROWS) {
    if (e - s > LOADS * ROWS) load(t0);
#pragma unroll
    for (int i = 0; i < LOADS; ++i)
      if (t0 + i * ROWS + sub < e) v[i].put(codes + (int64_t)slot[i] * D + (lane % LANES) * E, r);
  }
}

// A wave takes the pages whose first row of the call lies in its window of rows, whole.
// LOADS: what a page takes, up to 32; fewer registers leave room for more waves, but rows that
// do not fit are read twice (128-token pages 725 us with 16, 596 with 32).
template <int DT, int D, int LOADS>
__global__ void __launch_bounds__(64 * kWaves) store8_kernel(StoreArgs a, int window, int n_windows) {
  const int lane = threadIdx.x & 63;
  const int64_t unit = (int64_t)blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int plane = (int)(unit / n_windows);
  if (plane >= a.L * 2 * a.H) return;
  const int h = plane % a.H, kv = plane / a.H % 2, l = plane / (2 * a.H);
  const int t0 = (int)(unit - (int64_t)plane * n_windows) * window;
  const int t1 = t0 + window < a.T ? t0 + window : a.T;
  constexpr int E = Vec<DT>::N, LANES = D / E, ROWS = 64 / LANES;
  using T = typename std::conditional<DT == 0, uint16_t, float>::type;
  const int64_t* st = a.stride[kv];
  const T* x = static_cast<const T*>(a.x[kv]) + l * st[0] + h * st[1] + (lane % LANES) * E;
  uint8_t* codes = a.codes + ((int64_t)plane * a.N << a.log2p) * D;
  float* scales = a.scales + (int64_t)plane * a.N;
  const uint32_t num_slots = (uint32_t)a.N << a.log2p;

  // 64 rows from c on, a lane each: its slot, and which rows go on with the page before
  auto look = [&](int c, uint32_t& slot) {
    const int t = c + lane;
    slot = t < a.T ? (uint32_t)a.slots[t] : num_slots;
    const uint32_t before = t > 0 && t <= a.T ? (uint32_t)a.slots[t - 1] : num_slots;
    return __ballot(slot < num_slots && before < num_slots && slot >> a.log2p == before >> a.log2p);
  };
  for (int c = t0; c < t1; c += 64) {
    uint32_t slot;
    const uint64_t on = look(c, slot);
    uint64_t starts = __ballot(slot < num_slots && c + lane < t1) & ~on;
    while (starts) {
      const int i = __ffsll((unsigned long long)starts) - 1;
      starts &= starts - 1;
      const uint32_t first = (uint32_t)__builtin_amdgcn_readlane((int)slot, i);
      const float old = scales[first >> a.log2p];
      // rows that follow on the page, past these 64 too
      uint64_t rest = i < 63 ? ~(on >> (i + 1)) : ~0ull;
      int e = c + i + 1 + (rest ? __ffsll((unsigned long long)rest) - 1 : 64);
      for (int from = c + 64; e == from; from += 64) {
        uint32_t ignored;
        rest = ~look(from, ignored);
        e = from + (rest ? __ffsll((unsigned long long)rest) - 1 : 64);
      }
      if (e - (c + i) <= ROWS) store_page<DT, D, 1>(a, x, st[2], codes, scales, c + i, e, first, old);
      else store_page<DT, D, LOADS>(a, x, st[2], codes, scales, c + i, e, first, old);
    }
  }
}

template <int DT, int D>
hipError_t launch(const StoreArgs& a, hipStream_t stream) {
  // A wave's window is a page of rows, or less where waves would be fewer than 8 a CU (rows of
  // one page each would wait for one another: 512 single rows of 8 heads 10.0 us with 4 a CU,
  // 7.4 with 8, 6.5 with 32; but waves without a page cost too: 2048 rows 7.2, 8.5, 14.3);
  // up to eight pages of 2 KB or less, where waves are many (d = 64, 16-token pages, 8192 rows
  // of 64 layers 455 -> 400 us; pages of 4 KB 608 -> 623).
  const int64_t planes = (int64_t)a.L * 2 * a.H;
  const int loads = (D / Vec<DT>::N << a.log2p) / 64;
  int window = 1 << a.log2p;
  for (int i = 0; i < 3 && loads <= 2 && planes * (a.T / (2 * window)) >= 32768; ++i) window *= 2;
  while (window > 1 && planes * ((a.T + window - 1) / window) < 2048) window /= 2;
  const int n = (a.T + window - 1) / window;
  const int64_t wg = (planes * n + kWaves - 1) / kWaves;
  if (wg >= (int64_t)1 << 31) return hipErrorInvalidValue;
  const dim3 grid((unsigned)wg), block(64 * kWaves);
  if (loads <= 4) hipLaunchKernelGGL((store8_kernel<DT, D, 4>), grid, block, 0, stream, a, window, n);
  else if (loads <= 8) hipLaunchKernelGGL((store8_kernel<DT, D, 8>), grid, block, 0, stream, a, window, n);
  else if (loads <= 16) hipLaunchKernelGGL((store8_kernel<DT, D, 16>), grid, block, 0, stream, a, window, n);
  else hipLaunchKernelGGL((store8_kernel<DT, D, 32>), grid, block, 0, stream, a, window, n);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_store(const StoreArgs& a, int dtype, int d, hipStream_t stream) {
  if (dtype == 0) return d == 64 ? launch<0, 64>(a, stream) : launch<0, 128>(a, stream);
  return d == 64 ? launch<1, 64>(a, stream) : launch<1, 128>(a, stream);
}

}  // namespace kvx
