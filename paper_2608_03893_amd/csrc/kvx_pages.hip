// Page plan: block tables, slots and positions of a step's new tokens from request
// lengths, and the ring of free pages.
//
// With grow_b = max(add_b, 0), pages p(n) = ceil(n / P) and prefix sums over b,
//   end_b  = sum grow          rows of requests 0 .. b
//   pend_b = sum ask           ask_b = p(len_b + grow_b) - p(len_b), 0 where the
//                              request passes the table or the step's rows
//   rend_b = sum p(len_b) of ended requests
// row t belongs to the first b with end_b > t, the j-th page taken to the first b
// with pend_b > j, the j-th page given back to the first b with rend_b > j.
#include "kvx_serve.h"

namespace kvx {
namespace {

constexpr int kThreads = 256;

// Sums that stop at 2^32 - 1 instead of wrapping: still associative, and beyond any row or
// page that a request may get.
__device__ __forceinline__ uint32_t plus(uint32_t a, uint32_t b) { return __builtin_elementwise_add_sat(a, b); }

// Exclusive sums of a pair over the workgroup's threads; every thread calls it.  `part`: one
// pair per wave.
__device__ uint2 block_scan(uint2 v, uint2* part) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint2 sum = v;
#pragma unroll
  for (int n = 1; n < 64; n <<= 1) {
    const uint32_t x = __shfl_up(sum.x, n, 64), y = __shfl_up(sum.y, n, 64);
    if (lane >= n) sum = make_uint2(plus(sum.x, x), plus(sum.y, y));
  }
  if (lane == 63) part[wave] = sum;
  uint2 before = make_uint2(__shfl_up(sum.x, 1, 64), __shfl_up(sum.y, 1, 64));
  if (lane == 0) before = make_uint2(0, 0);
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kThreads / 64 - 1; ++w)
    if (w < wave) before = make_uint2(plus(before.x, part[w].x), plus(before.y, part[w].y));
  return before;
}

// First b with end[b] > x, at most B (end rises).
__device__ __forceinline__ int find(const int32_t* end, int B, int32_t x) {
  int lo = 0, n = B;
  while (n > 0) {
    const int half = n >> 1;
    if (end[lo + half] > x) n = half;
    else { lo += half + 1; n -= half + 1; }
  }
  return lo;
}

// What a request asks for, its rows' end known.
struct Request {
  int32_t len, grow, have, ask, back;
  bool fits;
};
__device__ __forceinline__ Request request(const PlanArgs& a, int32_t len, int32_t add, uint32_t end) {
  Request r;
  r.len = len > 0 ? len : 0;
  r.grow = add > 0 ? add : 0;
  const int64_t up = (1 << a.log2p) - 1;
  const int64_t have = (r.len + up) >> a.log2p, need = (r.len + (int64_t)r.grow + up) >> a.log2p;
  r.have = (int32_t)have;
  r.fits = r.grow == 0 || (need <= a.M && end <= (uint32_t)a.T);
  r.ask = r.fits ? (int32_t)(need - have) : 0;
  r.back = add < 0 ? (int32_t)(have < a.M ? have : a.M) : 0;
  return r;
}
__device__ __forceinline__ Request request(const PlanArgs& a, int b, int32_t end) {
  return request(a, a.lens[b], a.add[b], (uint32_t)end);
}

__device__ __forceinline__ int32_t least(int64_t x, int64_t most) {
  return (int32_t)(x < most ? x : most);
}

// Every workgroup sums over all requests (a few loads a thread) and keeps the three
// prefix sums in LDS, so one launch does it all; then the workgroups share the rows,
// the pages and the requests.
//
// Bound by its chain of waits (a launch, lengths, two scans, table or ring, stores), so
// what can wait side by side does: a step of 16 requests 6.6 -> 4.9 us (one row a thread),
// new turns of 160 requests, 300000 rows, 8.1 -> 6.7 us (pages apart from rows).
__global__ void __launch_bounds__(kThreads) plan_pages_kernel(PlanArgs a) {
  extern __shared__ int32_t lds[];
  int32_t* end = lds;
  int32_t* pend = lds + a.B;
  int32_t* rend = lds + 2 * a.B;
  __shared__ uint2 part[2][kThreads / 64];
  __shared__ int32_t refused;
  const int tid = threadIdx.x, B = a.B, T = a.T, N = a.N;
  const int chunk = (B + kThreads - 1) / kThreads;
  const int b0 = tid * chunk < B ? tid * chunk : B, b1 = b0 + chunk < B ? b0 + chunk : B;
  // A thread's first request (the only one of up to 256) is loaded once, with the ring's
  // state, before all waits.
  int32_t len0 = 0, add0 = 0;
  if (b0 < b1) {
    len0 = a.lens[b0];
    add0 = a.add[b0];
  }
  auto len_of = [&](int b) { return b == b0 ? len0 : a.lens[b]; };
  auto add_of = [&](int b) { return b == b0 ? add0 : a.add[b]; };
  int32_t count = a.free_in[1];
  count = count < 0 ? 0 : count > N ? N : count;
  const int32_t head = (int32_t)((uint32_t)a.free_in[0] % (uint32_t)N);
  if (tid == 0) refused = 0;

  uint32_t rows = 0;
  for (int b = b0; b < b1; ++b) rows = plus(rows, add_of(b) > 0 ? add_of(b) : 0);
  const uint32_t row0 = block_scan(make_uint2(rows, 0), part[0]).x;
  uint32_t at = row0;
  uint2 pages = make_uint2(0, 0);     // asked for, given back
  for (int b = b0; b < b1; ++b) {
    at = plus(at, add_of(b) > 0 ? add_of(b) : 0);
    end[b] = least(at, (int64_t)T + 1);
    const Request r = request(a, len_of(b), add_of(b), end[b]);
    pages = make_uint2(plus(pages.x, r.ask), plus(pages.y, r.back));
  }
  pages = block_scan(pages, part[1]);
  int32_t bad = 0;
  for (int b = b0; b < b1; ++b) {
    const Request r = request(a, len_of(b), add_of(b), end[b]);
    pages = make_uint2(plus(pages.x, r.ask), plus(pages.y, r.back));
    pend[b] = least(pages.x, (int64_t)N + 1);
    rend[b] = least(pages.y, (int64_t)N + 1);
    bad += !r.fits || (r.ask > 0 && pend[b] > count);
  }
  if (bad) atomicAdd(&refused, bad);
  __syncthreads();

  // The requests that get pages are those whose sum fits the free ones.
  const int n_ok = find(pend, B, count);
  const int32_t taken = n_ok > 0 ? pend[n_ok - 1] : 0;
  const int32_t total = B > 0 ? least(end[B - 1], T) : 0;
  const int32_t back = B > 0 ? least(rend[B - 1], N - count) : 0;

  // Entry of the ring n places after the first free page's; n <= N.
  auto place = [&](int32_t n) {
    const int64_t at = (int64_t)head + n;
    return at >= N ? at - N : at;
  };

  const int first = blockIdx.x * kThreads + tid, step = gridDim.x * kThreads;
  for (int b = first; b < B; b += step) {
    // rows past T: any end past it refuses
    const Request r = request(a, len_of(b), add_of(b), end[b]);
    const bool granted = r.fits && (r.ask == 0 || pend[b] <= count);
    a.lens_out[b] = add_of(b) < 0 ? 0 : granted ? r.len + r.grow : len_of(b);
    a.cu[b + 1] = least(end[b], T);
  }
  if (first == 0) {
    a.cu[0] = 0;
    a.free_out[0] = (int32_t)place(taken);
    a.free_out[1] = count - taken + back;
    a.free_out[2] = refused;
    a.free_out[3] = total;
  }
  // pages from the last workgroup on, rows from the first: neither waits for the other
  const int first_page = (gridDim.x - 1 - blockIdx.x) * kThreads + tid;
  for (int j = first_page; j < taken; j += step) {
    const int b = find(pend, B, j);
    const Request r = request(a, b, end[b]);
    const int32_t j0 = b > 0 ? pend[b - 1] : 0;
    a.tables[(int64_t)b * a.M + r.have + (j - j0)] = a.ring[place(j)];
  }
  for (int j = first_page; j < back; j += step) {
    const int b = find(rend, B, j);
    const int32_t j0 = b > 0 ? rend[b - 1] : 0;
    a.ring[place(count + j)] = a.tables[(int64_t)b * a.M + (j - j0)];
  }
  // Four rows a thread and step, written together; one where there are threads enough, since
  // rows of different requests wait for their tables one after another.
  const int width = T <= step ? 1 : 4;
  for (int t0 = first * width; t0 < T; t0 += step * width) {
    int32_t pos[4], slot[4];
    int b = find(end, B, t0);
    Request r;
    bool granted = false;
    int32_t start = 0, pstart = 0, stop = -1;   // of request b; stop: its last row's successor
    int32_t of = -1, page = -1;                 // a page's number in the request, the page
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int t = t0 + i;
      pos[i] = 0;
      slot[i] = -1;
      if (i >= width || t >= total) continue;
      if (t >= stop) {
        while (end[b] <= t) ++b;
        r = request(a, b, end[b]);
        granted = r.fits && (r.ask == 0 || pend[b] <= count);
        start = b > 0 ? end[b - 1] : 0;
        pstart = b > 0 ? pend[b - 1] : 0;
        stop = end[b];
        of = -1;
      }
      const int64_t p = (int64_t)r.len + (t - start);
      pos[i] = (int32_t)p;
      if (!granted) continue;
      const int32_t n = (int32_t)(p >> a.log2p);
      if (n != of) {
        of = n;
        page = n < r.have ? a.tables[(int64_t)b * a.M + n] : a.ring[place(pstart + (n - r.have))];
      }
      if (page >= 0 && page < N) slot[i] = (page << a.log2p) + (int32_t)(p & ((1 << a.log2p) - 1));
    }
    if (width == 1) {
      a.positions[t0] = pos[0];
      a.slots[t0] = slot[0];
    } else if (t0 + 3 < T) {
      *reinterpret_cast<int4*>(a.positions + t0) = make_int4(pos[0], pos[1], pos[2], pos[3]);
      *reinterpret_cast<int4*>(a.slots + t0) = make_int4(slot[0], slot[1], slot[2], slot[3]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (t0 + i < T) {
          a.positions[t0 + i] = pos[i];
          a.slots[t0 + i] = slot[i];
        }
    }
  }
}

}  // namespace

hipError_t launch_plan(const PlanArgs& a, hipStream_t stream) {
  // a thread for four rows and one for eight pages of the ring (most steps move few)
  int64_t wg = ((int64_t)a.T / 4 + a.N / 8 + kThreads) / kThreads;
  if (wg > 768) wg = 768;
  hipLaunchKernelGGL(plan_pages_kernel, dim3((unsigned)wg), dim3(kThreads), (size_t)a.B * 12, stream, a);
  return hipGetLastError();
}

}  // namespace kvx
