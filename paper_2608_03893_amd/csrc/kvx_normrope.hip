// RMS norm and position rotation of query and key heads, in one pass.
//
// y = R(p) (x / sqrt(mean x^2 + eps) * w) for every head of a row, the norm left out where no
// weights are given.  All of it in fp32 from the elements as they are, rounded once, to the
// output; the angles p w_j in fp64, reduced to a fraction of a turn before sine and cosine.
//
// A lane holds E channels of a head's first half and the E that half-split planes pair with
// them (16 bytes each), so that a plane's two channels meet in a lane in both layouts, and a
// row's squares are summed over 4 to 16 neighbouring lanes.  A wave takes 64 / lanes heads of a
// token, with that token's d / 2 sines and cosines, one plane a lane, shared through LDS that is
// its own, without a barrier.  They are formed again for every wave of a token while its heads are
// on the way: a wave for several heads a token, with the next ones loaded ahead, was no faster (8192
// tokens of 72 heads 59 us, 1024 of 72 9.5; now 55.6 and 8.2), nor is a loop over the heads, which
// keeps the sine's constants in registers that other waves could have (60 us).
//
// Bound by memory, every element read once and written once: 8192 tokens of 72 bf16 heads of 128
// channels, 302 MB, in 55.6 us, 5.4 TB/s.  A step of 16 tokens of 48 heads runs for 3.4 us, hardly
// more than an empty kernel, and takes 7 us a call, the host's time.
#include "kvx_bf16.h"
#include "kvx_serve.h"

namespace kvx {
namespace {

constexpr int kWaves = 4;
constexpr int64_t kMost = 1 << 23;      // workgroups of a launch, whose threads are counted in 32 bits

// 16 bytes of a row as floats, and back.
template <int DT>
struct Oct;
template <>
struct Oct<0> {
  static constexpr int N = 8;
  typedef uint16_t T;
  __device__ static void get(const u32x4_t& q, float* x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = lo_bf16(q[i]);
      x[2 * i + 1] = hi_bf16(q[i]);
    }
  }
  __device__ static u32x4_t put(const float* x) {
    return (u32x4_t){pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(x[4], x[5]), pack2(x[6], x[7])};
  }
};
template <>
struct Oct<1> {
  static constexpr int N = 4;
  typedef float T;
  __device__ static void get(const u32x4_t& q, float* x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(q[i]);
  }
  __device__ static u32x4_t put(const float* x) {
    return (u32x4_t){__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
  }
};

template <int DT, int D, int STYLE>
__global__ void __launch_bounds__(64 * kWaves) norm_rope_kernel(NormRopeArgs a) {
  using O = Oct<DT>;
  using T = typename O::T;
  constexpr int E = O::N, LANES = D / (2 * E), HEADS = 64 / LANES, HALF = D / 2;
  __shared__ __attribute__((aligned(16))) float2 turn[kWaves][HALF];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int sub = lane / LANES, at = lane % LANES * E;       // head of the group, channel of the half
  const int heads = a.heads[0] + a.heads[1], all = (heads + HEADS - 1) / HEADS;
  const int64_t tasks = (int64_t)a.T * all;
  const int64_t task = a.first + (int64_t)blockIdx.x * kWaves + wave;
  if (task >= tasks) return;
  const int64_t token = tasks >> 32 == 0 ? (int64_t)((uint32_t)task / (uint32_t)all) : task / all;
  const int h = (int)(task - token * all) * HEADS + sub;
  const bool live = h < heads, key = live && h >= a.heads[0];
  const int head = live ? (key ? h - a.heads[0] : h) : 0;       // in its tensor
  const T* from = static_cast<const T*>(key ? a.x[1] : a.x[0]) + token * a.stride[key][0] + head * a.stride[key][1] + at;
  const u32x4_t lower = *reinterpret_cast<const u32x4_t*>(from), upper = *reinterpret_cast<const u32x4_t*>(from + HALF);
  const T* weight = static_cast<const T*>(key ? a.weight[1] : a.weight[0]);
  const T* weights = weight != nullptr ? weight + at : from;      // (not used then)
  const u32x4_t w_lower = *reinterpret_cast<const u32x4_t*>(weights), w_upper = *reinterpret_cast<const u32x4_t*>(weights + HALF);

  // sine and cosine of plane `lane`, of a fraction of a turn
  const double p = (double)a.positions[token];
  if (lane < HALF) {
    const double t = p * a.turns.w[lane];
    double s, c;
    sincospi(2.0 * (t - rint(t)), &s, &c);
    turn[wave][lane] = make_float2((float)c, (float)s);
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  float cs[E], sn[E];        // planes at .. at + E - 1, or of the lane's channel pairs
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int plane = STYLE == 0 ? at + e : (e < E / 2 ? at / 2 + e : HALF / 2 + at / 2 + e - E / 2);
    const float2 v = turn[wave][plane];
    cs[e] = v.x;
    sn[e] = v.y;
  }

  float x[2 * E];
  O::get(lower, x);
  O::get(upper, x + E);
  if (weight != nullptr) {
    float y[2 * E], sum = 0.0f;
    O::get(w_lower, y);
    O::get(w_upper, y + E);
#pragma unroll
    for (int i = 0; i < 2 * E; ++i) sum = __builtin_fmaf(x[i], x[i], sum);
#pragma unroll
    for (int n = 1; n < LANES; n <<= 1) sum += __shfl_xor(sum, n, 64);
    const float v = __builtin_fmaf(sum, 1.0f / D, a.eps);
    float by = __builtin_amdgcn_rsqf(v);
    by *= __builtin_fmaf(-0.5f * v * by, by, 1.5f);        // a Newton step: the last bits
    if (v > 0x1p-90f && v < 0x1p110f) {
#pragma unroll
      for (int i = 0; i < 2 * E; ++i) x[i] = x[i] * by * y[i];      // (by times a weight may pass fp32's range)
    } else {      // squares that fp32 does not hold (all lanes of a head agree)
      double wide = 0.0;
#pragma unroll
      for (int i = 0; i < 2 * E; ++i) wide += (double)x[i] * (double)x[i];
#pragma unroll
      for (int n = 1; n < LANES; n <<= 1) wide += __shfl_xor(wide, n, 64);
      const double by64 = 1.0 / sqrt(wide / D + (double)a.eps);
#pragma unroll
      for (int i = 0; i < 2 * E; ++i) x[i] = (float)((double)x[i] * by64) * y[i];
    }
  }
#pragma unroll
  for (int e = 0; e < E; ++e) {
    // plane (i, j): channels that pair up
    const int i = STYLE == 0 ? e : (e < E / 2 ? 2 * e : E + 2 * (e - E / 2)), j = STYLE == 0 ? E + e : i + 1;
    const float u = x[i], v = x[j];
    x[i] = __builtin_fmaf(u, cs[e], -v * sn[e]);
    x[j] = __builtin_fmaf(v, cs[e], u * sn[e]);
  }
  if (live) {
    T* to = static_cast<T*>(key ? a.out[1] : a.out[0]) + (token * a.heads[key] + head) * D + at;
    *reinterpret_cast<u32x4_t*>(to) = O::put(x);
    *reinterpret_cast<u32x4_t*>(to + HALF) = O::put(x + E);
  }
}

template <int DT, int D>
hipError_t launch(NormRopeArgs a, int style, hipStream_t stream) {
  constexpr int HEADS = 64 / (D / (2 * Oct<DT>::N));
  const int64_t tasks = (int64_t)a.T * ((a.heads[0] + a.heads[1] + HEADS - 1) / HEADS);
  for (a.first = 0; a.first < tasks; a.first += kMost * kWaves) {
    const int64_t want = (tasks - a.first + kWaves - 1) / kWaves;
    const dim3 grid((unsigned)(want < kMost ? want : kMost)), block(64 * kWaves);
    if (style == 0)
      hipLaunchKernelGGL((norm_rope_kernel<DT, D, 0>), grid, block, 0, stream, a);
    else
      hipLaunchKernelGGL((norm_rope_kernel<DT, D, 1>), grid, block, 0, stream, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_norm_rope(const NormRopeArgs& a, int dtype, int d, int style, hipStream_t stream) {
  if (dtype == 0) return d == 64 ? launch<0, 64>(a, style, stream) : launch<0, 128>(a, style, stream);
  return d == 64 ? launch<1, 64>(a, style, stream) : launch<1, 128>(a, style, stream);
}

}  // namespace kvx
