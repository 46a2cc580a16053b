// 8-bit store: packed rows into the pool of e4m3 codes, a power-of-two scale for each
// (layer, K|V, head, page).
//
// Codes are x / s for the page's s = 2^j >= amax / 448.  Division by a power of two is
// exact, so a code carries one rounding (e4m3's), the same whether the page was written
// at once or token by token, unless its scale grew and a code fell below e4m3's least
// normal value.
//
// Bound by memory: 2 or 4 bytes read and one written per element.
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

// A wave takes the pages whose first row of the call lies in its window of rows, whole:
// the largest value over the page's rows, the scale, the codes.
template <int DT, int D>
__global__ void __launch_bounds__(64 * kWaves) store8_kernel(StoreArgs a, int window, int n_windows) {
  const int lane = threadIdx.x & 63;
  const int64_t unit = (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6);
  const int plane = (int)(unit / n_windows);
  if (plane >= a.L * 2 * a.H) return;
  const int h = plane % a.H, kv = plane / a.H % 2, l = plane / (2 * a.H);
  const int t0 = (int)(unit % n_windows) * window;
  const int t1 = t0 + window < a.T ? t0 + window : a.T;
  constexpr int E = Vec<DT>::N, LANES = D / E, ROWS = 64 / LANES;   // lanes a row, rows a load
  using T = typename std::conditional<DT == 0, uint16_t, float>::type;
  const T* x = static_cast<const T*>(a.x[kv]) + l * a.stride[kv][0] + h * a.stride[kv][1] + (lane % LANES) * E;
  const int64_t ts = a.stride[kv][2];
  const int P = 1 << a.log2p;
  uint8_t* codes = a.codes + (int64_t)plane * a.N * P * D;
  const uint32_t num_slots = (uint32_t)a.N << a.log2p;

  for (int s = t0; s < t1; ++s) {
    const uint32_t slot = (uint32_t)a.slots[s];
    if (slot >= num_slots) continue;
    const uint32_t page = slot >> a.log2p;
    if (s > 0) {
      const uint32_t before = (uint32_t)a.slots[s - 1];
      if (before < num_slots && before >> a.log2p == page) continue;
    }
    // rows s .. e - 1 are the page's
    int e = s + 1;
    for (;;) {
      const int t = e + lane;
      const uint32_t u = t < a.T ? (uint32_t)a.slots[t] : num_slots;
      const uint64_t other = __ballot(!(u < num_slots && u >> a.log2p == page));
      if (other) { e += __ffsll((unsigned long long)other) - 1; break; }
      e += 64;
    }
    float m = 0.0f;
    for (int t = s + lane / LANES; t < e; t += ROWS) {
      Vec<DT> v;
      v.q = *reinterpret_cast<const uint4*>(x + t * ts);
      m = fmaxf(m, v.amax());
    }
    float scale = pow2_scale(wave_max(m));
    const int held = slot & (P - 1);   // earlier rows of the page
    float* sp = a.scales + (int64_t)plane * a.N + page;
    if (held > 0) {
      const float old = *sp;
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
    if (lane == 0) *sp = scale;
    const float r = 1.0f / scale;
    for (int t = s + lane / LANES; t < e; t += ROWS) {
      Vec<DT> v;
      v.q = *reinterpret_cast<const uint4*>(x + t * ts);
      v.put(codes + (int64_t)(uint32_t)a.slots[t] * D + (lane % LANES) * E, r);
    }
    s = e - 1;
  }
}

template <int DT, int D>
hipError_t launch(const StoreArgs& a, hipStream_t stream) {
  const int64_t planes = (int64_t)a.L * 2 * a.H;
  int window = 1 << a.log2p;
  while (window > 1 && planes * ((a.T + window - 1) / window) < 8192) window /= 2;
  const int n = (a.T + window - 1) / window;
  const int64_t wg = (planes * n + kWaves - 1) / kWaves;
  if (wg >= (int64_t)1 << 31) return hipErrorInvalidValue;
  hipLaunchKernelGGL((store8_kernel<DT, D>), dim3((unsigned)wg), dim3(64 * kWaves), 0, stream, a, window, n);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_store(const StoreArgs& a, int dtype, int d, hipStream_t stream) {
  if (dtype == 0) return d == 64 ? launch<0, 64>(a, stream) : launch<0, 128>(a, stream);
  return d == 64 ? launch<1, 64>(a, stream) : launch<1, 128>(a, stream);
}

}  // namespace kvx
