// Attention over the 8-bit pool.
#include "kvx_e4m3.h"
#include "kvx_serve.h"

namespace kvx {
namespace {

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int n = 32; n; n >>= 1) v = fmaxf(v, __shfl_xor(v, n, 64));
  return v;
}
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int n = 32; n; n >>= 1) v += __shfl_xor(v, n, 64);
  return v;
}

// A wave for each (row, query head): 64 keys at a time, a lane each for the scores, then
// the lanes' channels for the sum of values.
template <int DT, int D>
__global__ void __launch_bounds__(64) attend8_kernel(AttendArgs a) {
  __shared__ float qs[D];
  const int lane = threadIdx.x, head = blockIdx.y, h = head / a.G, Hq = a.H * a.G;
  const int t = blockIdx.x;
  // the request of row t: the first one whose rows end behind it
  int b = 0, n = a.B;
  while (n > 0) {
    const int half = n >> 1;
    if (a.cu[b + half + 1] > t) n = half;
    else { b += half + 1; n -= half + 1; }
  }
  if (b == a.B || a.cu[b] > t) return;
  const int end = a.cu[b + 1] < a.T ? a.cu[b + 1] : a.T;
  const int64_t cap = (int64_t)a.M << a.log2p;
  const int len = a.lens[b] < cap ? a.lens[b] : (int)cap;
  const int seen = len - (end - t) + 1;   // keys 0 .. seen - 1
  for (int c = lane; c < D; c += 64) {
    const int64_t at = t * a.q_stride[0] + head * a.q_stride[1] + c;
    qs[c] = DT == 0 ? lo_bf16(static_cast<const uint16_t*>(a.q)[at]) : static_cast<const float*>(a.q)[at];
  }
  __syncthreads();
  const int64_t plane = ((int64_t)a.N << a.log2p) * D;
  const uint8_t* kc = a.codes + h * plane;
  const uint8_t* vc = a.codes + (a.H + h) * plane;
  const float* ks = a.scales + (int64_t)h * a.N;
  const float* vs = a.scales + (int64_t)(a.H + h) * a.N;
  float top = -INFINITY, total = 0.0f, o[D / 64] = {};
  for (int j0 = 0; j0 < seen; j0 += 64) {
    const int j = j0 + lane;
    float s = -INFINITY, sv = 0.0f;
    int64_t row = 0;
    if (j < seen) {
      const int page = a.tables[(int64_t)b * a.M + (j >> a.log2p)];
      if (page >= 0 && page < a.N) {
        row = (((int64_t)page << a.log2p) + (j & ((1 << a.log2p) - 1))) * D;
        float dot = 0.0f;
        for (int c = 0; c < D; c += 4) {
          const uint32_t w = *reinterpret_cast<const uint32_t*>(kc + row + c);
          dot = fmaf(qs[c], from_e4m3<0>(w), dot);
          dot = fmaf(qs[c + 1], from_e4m3<1>(w), dot);
          dot = fmaf(qs[c + 2], from_e4m3<2>(w), dot);
          dot = fmaf(qs[c + 3], from_e4m3<3>(w), dot);
        }
        s = dot * (ks[page] * a.scale_log2);
        sv = vs[page];
      }
    }
    const float now = fmaxf(top, wave_max(s));
    const float ref = now == -INFINITY ? 0.0f : now;
    const float keep = exp2f(top - ref);
    const float p = s == -INFINITY ? 0.0f : exp2f(s - ref);   // NaN stays
    total = total * keep + wave_sum(p);
    top = now;
    for (int i = 0; i < D / 64; ++i) o[i] *= keep;
    const float pv = p * sv;
    for (int i = 0; i < 64; ++i) {
      if (__shfl(s, i, 64) == -INFINITY) continue;
      const float w = __shfl(pv, i, 64);
      const uint8_t* v = vc + __shfl((long long)row, i, 64);
      for (int c = 0; c < D / 64; ++c) o[c] = fmaf(w, from_e4m3<0>(v[lane + 64 * c]), o[c]);
    }
  }
  const float r = total == 0.0f ? 0.0f : 1.0f / total;   // NaN stays
  const int64_t at = (int64_t)t * Hq + head;
  for (int c = 0; c < D / 64; ++c) {
    if (DT == 0) static_cast<uint16_t*>(a.out)[at * D + lane + 64 * c] = (uint16_t)pack2(o[c] * r, 0.0f);
    else static_cast<float*>(a.out)[at * D + lane + 64 * c] = o[c] * r;
  }
  if (a.lse != nullptr && lane == 0)
    a.lse[at] = total == 0.0f ? -INFINITY : (top + log2f(total)) * 0.69314718055994530942f;
}

}  // namespace

size_t attend_ws_bytes(int, int, int, int, int, int) { return 0; }

hipError_t launch_attend(const AttendArgs& a, int dtype, int d, void*, hipStream_t stream) {
  const dim3 grid(a.T, a.H * a.G);
  if (dtype == 0 && d == 64) hipLaunchKernelGGL((attend8_kernel<0, 64>), grid, dim3(64), 0, stream, a);
  else if (dtype == 0) hipLaunchKernelGGL((attend8_kernel<0, 128>), grid, dim3(64), 0, stream, a);
  else if (d == 64) hipLaunchKernelGGL((attend8_kernel<1, 64>), grid, dim3(64), 0, stream, a);
  else hipLaunchKernelGGL((attend8_kernel<1, 128>), grid, dim3(64), 0, stream, a);
  return hipGetLastError();
}

}  // namespace kvx
