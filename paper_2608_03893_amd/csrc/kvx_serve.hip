// Host side of the serving entry points of include/kvx.h (page plan, 8-bit store,
// attention over the 8-bit pool, norm and rotation, token sampling): argument checks and
// launches.  Every check runs
// before the first HIP call, so a rejected call enqueues nothing.
#include "kvx_serve.h"

#include <cmath>
#include <cstring>

namespace {

using kvx::set_error;

kvx_status ok() { return set_error(KVX_OK, "%s", ""); }

bool aligned(const void* p, uintptr_t n) { return ((uintptr_t)p % n) == 0; }

// An operand's bytes, for the overlap checks.
struct Span {
  const void* p;
  uint64_t bytes;
  const char* name;
};

bool overlap(const Span& a, const Span& b) {
  if (a.p == nullptr || b.p == nullptr || a.bytes == 0 || b.bytes == 0) return false;
  const uintptr_t a0 = (uintptr_t)a.p, b0 = (uintptr_t)b.p;
  return a0 < b0 + b.bytes && b0 < a0 + a.bytes;
}

// No output may share bytes with an input or with another output.
kvx_status check_alias(const Span* out, int n_out, const Span* in, int n_in) {
  for (int o = 0; o < n_out; ++o) {
    for (int i = 0; i < n_in; ++i)
      if (overlap(out[o], in[i]))
        return set_error(KVX_ERR_ALIAS, "%s overlaps %s", out[o].name, in[i].name);
    for (int i = o + 1; i < n_out; ++i)
      if (overlap(out[o], out[i]))
        return set_error(KVX_ERR_ALIAS, "%s overlaps %s", out[o].name, out[i].name);
  }
  return KVX_OK;
}

kvx_status check_pool(const kvx_pool* pool, bool tables, int* log2p) {
  if (pool == nullptr) return set_error(KVX_ERR_NULL, "pool is NULL");
  const kvx_pool& p = *pool;
  if (p.num_pages < 1 || p.page_size < 1 || (tables && p.max_pages < 1))
    return set_error(KVX_ERR_SHAPE, "pool out of range: num_pages=%d page_size=%d max_pages=%d",
                     p.num_pages, p.page_size, p.max_pages);
  *log2p = 0;
  for (int n = 4; n <= 7; ++n)
    if (p.page_size == 1 << n) *log2p = n;
  if (*log2p == 0)
    return set_error(KVX_ERR_UNSUPPORTED, "page_size=%d is not built (16, 32, 64 or 128)",
                     p.page_size);
  if ((int64_t)p.num_pages * p.page_size >= ((int64_t)1 << 31))
    return set_error(KVX_ERR_SHAPE, "num_pages * page_size = %lld reaches 2^31",
                     (long long)p.num_pages * p.page_size);
  return KVX_OK;
}

// Row numbers step past the last one in 32 bits.
kvx_status check_rows(int32_t T) {
  if (T > 1 << 30) return set_error(KVX_ERR_UNSUPPORTED, "T=%d exceeds 2^30 rows", T);
  return KVX_OK;
}

kvx_status check_requests(int32_t B, int32_t T) {
  if (B < 0 || T < 0) return set_error(KVX_ERR_SHAPE, "B=%d and T=%d must not be negative", B, T);
  if (B > KVX_MAX_REQUESTS)
    return set_error(KVX_ERR_UNSUPPORTED, "B=%d exceeds %d requests", B, KVX_MAX_REQUESTS);
  return check_rows(T);
}

kvx_status check_dtype(kvx_dtype dtype) {
  if (dtype != KVX_BF16 && dtype != KVX_F32)
    return set_error(KVX_ERR_DTYPE, "unknown dtype %d (0 = bf16, 1 = f32)", (int)dtype);
  return KVX_OK;
}

kvx_status check_d(int32_t d) {
  if (d != 64 && d != 128)
    return set_error(d < 1 ? KVX_ERR_SHAPE : KVX_ERR_UNSUPPORTED,
                     "head dimension d=%d is not built (64 or 128)", d);
  return KVX_OK;
}

// Strides in elements: rows start on 16 bytes, and the operand ends below 2^60 bytes.
kvx_status check_strides(const char* name, const int64_t* s, const int32_t* n, int rank, int es,
                         int d, uint64_t* bytes) {
  if (s == nullptr) return set_error(KVX_ERR_NULL, "%s strides are NULL", name);
  unsigned __int128 end = (unsigned)d;
  for (int i = 0; i < rank; ++i) {
    if (n[i] == 1) continue;   // never stepped
    if (s[i] < 0)
      return set_error(KVX_ERR_SHAPE, "%s stride %lld is negative", name, (long long)s[i]);
    if (s[i] % (16 / es) != 0)
      return set_error(KVX_ERR_UNSUPPORTED, "%s stride of %lld elements is not a multiple of 16 bytes",
                       name, (long long)s[i]);
    end += (unsigned __int128)(n[i] - 1) * (uint64_t)s[i];
  }
  if (end * es >= (uint64_t)1 << 60) return set_error(KVX_ERR_SHAPE, "%s strides reach too far", name);
  *bytes = (uint64_t)end * es;
  return KVX_OK;
}

kvx_status check_pointers(const Span* s, int n, uintptr_t align) {
  for (int i = 0; i < n; ++i) {
    if (s[i].p == nullptr) return set_error(KVX_ERR_NULL, "%s is NULL", s[i].name);
    if (!aligned(s[i].p, align))
      return set_error(KVX_ERR_UNSUPPORTED, "%s is not %d-byte aligned", s[i].name, (int)align);
  }
  return KVX_OK;
}

kvx_status check_workspace(const void* workspace, size_t bytes, uint64_t need) {
  if (need == 0) return KVX_OK;
  if (workspace == nullptr)
    return set_error(KVX_ERR_WORKSPACE, "workspace is NULL (%llu bytes needed)", (unsigned long long)need);
  if (bytes < need)
    return set_error(KVX_ERR_WORKSPACE, "workspace has %llu bytes, %llu needed", (unsigned long long)bytes,
                     (unsigned long long)need);
  if (!aligned(workspace, 256)) return set_error(KVX_ERR_WORKSPACE, "workspace is not 256-byte aligned");
  return KVX_OK;
}

}  // namespace

extern "C" {

kvx_status kvx_plan_pages(const kvx_pool* pool, int32_t B, int32_t T, const int32_t* lens,
                          const int32_t* add, int32_t* block_tables, int32_t* free_ring,
                          const int32_t* free_in, int32_t* lens_out, int32_t* cu_out,
                          int32_t* positions, int32_t* slot_mapping, int32_t* free_out,
                          void* stream) {
  int log2p;
  kvx_status st = check_pool(pool, true, &log2p);
  if (st != KVX_OK) return st;
  if ((st = check_requests(B, T)) != KVX_OK) return st;
  const uint64_t b4 = (uint64_t)B * 4, t4 = (uint64_t)T * 4;
  const Span in[] = {{free_in, 8, "free_in"}, {lens, b4, "lens"}, {add, b4, "add"}};
  const Span out[] = {{free_ring, (uint64_t)pool->num_pages * 4, "free_ring"},
                      {cu_out, b4 + 4, "cu_out"},
                      {free_out, 16, "free_out"},
                      {block_tables, b4 * pool->max_pages, "block_tables"},
                      {lens_out, b4, "lens_out"},
                      {positions, t4, "positions"},
                      {slot_mapping, t4, "slot_mapping"}};
  // an empty batch has no lengths and tables, an empty step no rows
  if ((st = check_pointers(in, B > 0 ? 3 : 1, 4)) != KVX_OK) return st;
  if ((st = check_pointers(out, B > 0 ? 5 : 3, 4)) != KVX_OK) return st;
  if (T > 0 && (st = check_pointers(out + 5, 2, 16)) != KVX_OK) return st;
  if ((st = check_alias(out, 7, in, 3)) != KVX_OK) return st;
  kvx::PlanArgs a;
  std::memset(&a, 0, sizeof(a));
  a.lens = lens;
  a.add = add;
  a.tables = block_tables;
  a.ring = free_ring;
  a.free_in = free_in;
  a.lens_out = lens_out;
  a.cu = cu_out;
  a.positions = positions;
  a.slots = slot_mapping;
  a.free_out = free_out;
  a.B = B;
  a.T = T;
  a.M = pool->max_pages;
  a.N = pool->num_pages;
  a.log2p = log2p;
  const hipError_t e = kvx::launch_plan(a, reinterpret_cast<hipStream_t>(stream));
  if (e != hipSuccess) return set_error(KVX_ERR_HIP, "page plan launch: %s", hipGetErrorString(e));
  return ok();
}

kvx_status kvx_store_cache8(const kvx_pool* pool, kvx_dtype dtype, int32_t L, int32_t H, int32_t T,
                            int32_t d, const void* k, const int64_t* k_strides, const void* v,
                            const int64_t* v_strides, const int32_t* slot_mapping, uint8_t* codes,
                            float* scales, void* stream) {
  int log2p;
  kvx_status st = check_pool(pool, false, &log2p);
  if (st != KVX_OK) return st;
  if ((st = check_dtype(dtype)) != KVX_OK) return st;
  if ((st = check_d(d)) != KVX_OK) return st;
  if (L < 1 || H < 1 || T < 0)
    return set_error(KVX_ERR_SHAPE, "L=%d H=%d T=%d out of range (L, H >= 1, T >= 0)", L, H, T);
  if ((st = check_rows(T)) != KVX_OK) return st;
  if ((int64_t)L * H * 2 > 65535)
    return set_error(KVX_ERR_UNSUPPORTED, "L*H*2=%lld exceeds 65535 planes", (long long)L * H * 2);
  if (T == 0) return ok();
  const int es = dtype == KVX_BF16 ? 2 : 4;
  const int32_t n[3] = {L, H, T};
  uint64_t kb, vb;
  if ((st = check_strides("k", k_strides, n, 3, es, d, &kb)) != KVX_OK) return st;
  if ((st = check_strides("v", v_strides, n, 3, es, d, &vb)) != KVX_OK) return st;
  const uint64_t planes = (uint64_t)L * 2 * H, pages = (uint64_t)pool->num_pages;
  const Span in[] = {{k, kb, "k"}, {v, vb, "v"}, {slot_mapping, (uint64_t)T * 4, "slot_mapping"}};
  const Span out[] = {{codes, planes * pages * pool->page_size * d, "codes"},
                      {scales, planes * pages * 4, "scales"}};
  if ((st = check_pointers(in, 2, 16)) != KVX_OK) return st;
  if ((st = check_pointers(in + 2, 1, 4)) != KVX_OK) return st;
  if ((st = check_pointers(out, 1, 16)) != KVX_OK) return st;
  if ((st = check_pointers(out + 1, 1, 4)) != KVX_OK) return st;
  if ((st = check_alias(out, 2, in, 3)) != KVX_OK) return st;
  kvx::StoreArgs a;
  std::memset(&a, 0, sizeof(a));
  a.x[0] = k;
  a.x[1] = v;
  for (int i = 0; i < 3; ++i) {
    a.stride[0][i] = k_strides[i];
    a.stride[1][i] = v_strides[i];
  }
  a.slots = slot_mapping;
  a.codes = codes;
  a.scales = scales;
  a.L = L;
  a.H = H;
  a.T = T;
  a.N = pool->num_pages;
  a.log2p = log2p;
  const hipError_t e = kvx::launch_store(a, dtype == KVX_BF16 ? 0 : 1, d,
                                         reinterpret_cast<hipStream_t>(stream));
  if (e != hipSuccess) return set_error(KVX_ERR_HIP, "8-bit store launch: %s", hipGetErrorString(e));
  return ok();
}

static kvx_status check_attend(const kvx_attend_dims* dims, kvx_dtype dtype) {
  if (dims == nullptr) return set_error(KVX_ERR_NULL, "dims is NULL");
  kvx_status st = check_dtype(dtype);
  if (st != KVX_OK) return st;
  if ((st = check_d(dims->d)) != KVX_OK) return st;
  if ((st = check_requests(dims->B, dims->T)) != KVX_OK) return st;
  if (dims->H < 1 || dims->G < 1)
    return set_error(KVX_ERR_SHAPE, "H=%d and G=%d must be at least 1", dims->H, dims->G);
  if (dims->longest < 0) return set_error(KVX_ERR_SHAPE, "longest=%d is negative", dims->longest);
  if ((int64_t)dims->H * dims->G > 65535 || (int64_t)dims->T * dims->G >= ((int64_t)1 << 30))
    return set_error(KVX_ERR_UNSUPPORTED, "H*G=%lld exceeds 65535 or T*G=%lld reaches 2^30",
                     (long long)dims->H * dims->G, (long long)dims->T * dims->G);
  return KVX_OK;
}

// The sizes that a launch goes by.
static kvx::AttendArgs attend_sizes(const kvx_attend_dims& m, const kvx_pool& pool, int log2p) {
  kvx::AttendArgs a;
  std::memset(&a, 0, sizeof(a));
  a.B = m.B;
  a.H = m.H;
  a.G = m.G;
  a.T = m.T;
  a.M = pool.max_pages;
  a.N = pool.num_pages;
  a.log2p = log2p;
  a.keys = (int64_t)a.M << log2p;
  if (m.longest > 0 && m.longest < a.keys) a.keys = m.longest;
  return a;
}

const char* kvx_attend_kernel_name(const kvx_attend_dims* dims, const kvx_pool* pool, kvx_dtype dtype) {
  int log2p;
  if (check_pool(pool, true, &log2p) != KVX_OK || check_attend(dims, dtype) != KVX_OK || dims->B == 0 || dims->T == 0)
    return nullptr;
  return kvx::attend_kernel_name(attend_sizes(*dims, *pool, log2p), dtype == KVX_BF16 ? 0 : 1, dims->d);
}

size_t kvx_attend_workspace_bytes(const kvx_attend_dims* dims, kvx_dtype dtype) {
  if (check_attend(dims, dtype) != KVX_OK || dims->B == 0 || dims->T == 0) return 0;
  return kvx::attend_ws_bytes(dims->B, dims->G, dims->T, dims->d, dtype == KVX_BF16 ? 0 : 1);
}

kvx_status kvx_attend_cache8(const kvx_attend_dims* dims, const kvx_pool* pool, kvx_dtype dtype,
                             const void* q, const int64_t* q_strides, const uint8_t* codes,
                             const float* scales, const int32_t* block_tables,
                             const int32_t* lens, const int32_t* cu, float scale, void* out,
                             float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  int log2p;
  kvx_status st = check_pool(pool, true, &log2p);
  if (st != KVX_OK) return st;
  if ((st = check_attend(dims, dtype)) != KVX_OK) return st;
  const kvx_attend_dims& m = *dims;
  if (!std::isfinite(scale)) return set_error(KVX_ERR_SHAPE, "scale must be finite");
  if (m.B == 0 || m.T == 0) return ok();
  const int dt = dtype == KVX_BF16 ? 0 : 1, es = dt == 0 ? 2 : 4;
  const int32_t n[2] = {m.T, m.H * m.G};
  uint64_t qb;
  if ((st = check_strides("q", q_strides, n, 2, es, m.d, &qb)) != KVX_OK) return st;
  const uint64_t pages = (uint64_t)2 * m.H * pool->num_pages, b4 = (uint64_t)m.B * 4;
  const uint64_t rows = (uint64_t)m.T * m.H * m.G;
  const uint64_t need = kvx::attend_ws_bytes(m.B, m.G, m.T, m.d, dt);
  const Span in[] = {{q, qb, "q"},
                     {codes, pages * pool->page_size * m.d, "codes"},
                     {scales, pages * 4, "scales"},
                     {block_tables, b4 * pool->max_pages, "block_tables"},
                     {lens, b4, "lens"},
                     {cu, b4 + 4, "cu"}};
  const Span outs[] = {{out, rows * m.d * es, "out"}, {lse, rows * 4, "lse"},
                       {workspace, need, "workspace"}};
  if ((st = check_pointers(in, 2, 16)) != KVX_OK) return st;
  if ((st = check_pointers(in + 2, 4, 4)) != KVX_OK) return st;
  if ((st = check_pointers(outs, 1, 16)) != KVX_OK) return st;
  if (lse != nullptr && (st = check_pointers(outs + 1, 1, 4)) != KVX_OK) return st;
  if ((st = check_workspace(workspace, workspace_bytes, need)) != KVX_OK) return st;
  if ((st = check_alias(outs, 3, in, 6)) != KVX_OK) return st;
  kvx::AttendArgs a = attend_sizes(m, *pool, log2p);
  a.q = q;
  a.q_stride[0] = q_strides[0];
  a.q_stride[1] = q_strides[1];
  a.codes = codes;
  a.scales = scales;
  a.tables = block_tables;
  a.lens = lens;
  a.cu = cu;
  a.out = out;
  a.lse = lse;
  a.scale_log2 = scale * 1.44269504088896340736f;
  const hipError_t e = kvx::launch_attend(a, dt, m.d, workspace, reinterpret_cast<hipStream_t>(stream));
  if (e != hipSuccess) return set_error(KVX_ERR_HIP, "attention launch: %s", hipGetErrorString(e));
  return ok();
}

kvx_status kvx_norm_rope(kvx_dtype dtype, int32_t T, int32_t Hq, int32_t Hk, int32_t d, const void* q,
                         const int64_t* q_strides, const void* k, const int64_t* k_strides,
                         const void* q_weight, const void* k_weight, float eps, const kvx_rope* rope,
                         const int32_t* positions, void* q_out, void* k_out, void* stream) {
  kvx_status st = check_dtype(dtype);
  if (st != KVX_OK) return st;
  if ((st = check_d(d)) != KVX_OK) return st;
  if (T < 0 || Hq < 1 || Hk < 0)
    return set_error(KVX_ERR_SHAPE, "T=%d Hq=%d Hk=%d out of range (T, Hk >= 0, Hq >= 1)", T, Hq, Hk);
  if ((st = check_rows(T)) != KVX_OK) return st;
  if ((int64_t)Hq + Hk > 65535)
    return set_error(KVX_ERR_UNSUPPORTED, "Hq+Hk=%lld exceeds 65535 heads", (long long)Hq + Hk);
  if (!std::isfinite(eps) || eps < 0) return set_error(KVX_ERR_SHAPE, "eps must be finite and not negative");
  if ((st = kvx::check_rope_params(rope, "target")) != KVX_OK) return st;
  if (T == 0) return ok();
  const int es = dtype == KVX_BF16 ? 2 : 4;
  const int32_t heads[2] = {Hq, Hk};
  const void* x[2] = {q, k};
  const int64_t* strides[2] = {q_strides, k_strides};
  const char* names[2] = {"q", "k"};
  uint64_t bytes[2] = {0, 0};
  const int operands = Hk > 0 ? 2 : 1;
  for (int i = 0; i < operands; ++i) {
    const int32_t n[2] = {T, heads[i]};
    if ((st = check_strides(names[i], strides[i], n, 2, es, d, &bytes[i])) != KVX_OK) return st;
  }
  const uint64_t wb = (uint64_t)d * es;
  const Span in[] = {{q, bytes[0], "q"},       {k, bytes[1], "k"}, {q_weight, wb, "q_weight"},
                     {k_weight, operands > 1 ? wb : 0, "k_weight"}, {positions, (uint64_t)T * 4, "positions"}};
  const Span out[] = {{q_out, (uint64_t)T * Hq * d * es, "q_out"}, {k_out, (uint64_t)T * Hk * d * es, "k_out"}};
  if ((st = check_pointers(in, operands, 16)) != KVX_OK) return st;
  for (int i = 0; i < operands; ++i)
    if (in[2 + i].p != nullptr && (st = check_pointers(in + 2 + i, 1, 16)) != KVX_OK) return st;
  if ((st = check_pointers(in + 4, 1, 4)) != KVX_OK) return st;
  if ((st = check_pointers(out, operands, 16)) != KVX_OK) return st;
  // an output may be its own dense input: every element is read before it is written, by its lane
  Span others[5];
  for (int i = 0; i < operands; ++i) {
    const bool in_place = out[i].p == x[i] && (heads[i] == 1 || strides[i][1] == d) &&
                          (T == 1 || strides[i][0] == (int64_t)heads[i] * d);
    for (int j = 0; j < 5; ++j) others[j] = in[j];
    if (in_place) others[i].bytes = 0;
    if ((st = check_alias(out + i, 1, others, 5)) != KVX_OK) return st;
  }
  if ((st = check_alias(out, operands, nullptr, 0)) != KVX_OK) return st;
  kvx::NormRopeArgs a;
  std::memset(&a, 0, sizeof(a));
  for (int i = 0; i < operands; ++i) {
    a.x[i] = x[i];
    a.stride[i][0] = strides[i][0];
    a.stride[i][1] = strides[i][1];
    a.weight[i] = in[2 + i].p;
    a.out[i] = i == 0 ? q_out : k_out;
    a.heads[i] = heads[i];
  }
  a.positions = positions;
  a.eps = eps;
  a.T = T;
  kvx::rope_frequencies(*rope, d, a.turns);
  for (int j = 0; j < d / 2; ++j) a.turns.w[j] *= 0.15915494309189533576888376337251;   // 1 / (2 pi)
  const hipError_t e = kvx::launch_norm_rope(a, dtype == KVX_BF16 ? 0 : 1, d, rope->style,
                                             reinterpret_cast<hipStream_t>(stream));
  if (e != hipSuccess) return set_error(KVX_ERR_HIP, "norm and rotation launch: %s", hipGetErrorString(e));
  return ok();
}

static kvx_status check_prefix(const kvx_prefix_dims* p) {
  if (p == nullptr) return set_error(KVX_ERR_NULL, "prefix is NULL");
  if (p->S < 0 || p->max_pages < 1 || p->longest < 0)
    return set_error(KVX_ERR_SHAPE, "prefix out of range: S=%d max_pages=%d longest=%d", p->S, p->max_pages, p->longest);
  if (p->S > KVX_MAX_REQUESTS)
    return set_error(KVX_ERR_UNSUPPORTED, "S=%d exceeds %d prefixes", p->S, KVX_MAX_REQUESTS);
  return KVX_OK;
}

// The workspace: counters and partial sums of the own part on its own, then for each part the
// partial sums of its workgroups, a row's sums, statistics and where they are (of the own one where
// both may go in one launch; calls of more rows need no less than the largest of these, so that a
// workspace for many rows is enough for fewer).
struct PrefixSpace {
  struct Part {
    uint64_t partial, sums, stats, parts;
  } part[2];
  uint64_t bytes;
};
static PrefixSpace prefix_space(const kvx_attend_dims& m, int32_t S, int dt) {
  PrefixSpace s;
  std::memset(&s, 0, sizeof(s));
  s.bytes = kvx::attend_ws_bytes(m.B, m.G, m.T, m.d, dt);
  const uint64_t rows = (uint64_t)m.T * m.H * m.G;
  auto take = [&](uint64_t n) {
    const uint64_t at = (s.bytes + 255) / 256 * 256;
    s.bytes = at + n;
    return at;
  };
  for (int i = 0; S > 0 && i < (rows <= (uint64_t)kvx::kPrefixRows ? 2 : 1); ++i) {
    s.part[i].partial = take(i == 0 ? kvx::prefix_partial_bytes(S, m.G, m.T, m.d, dt)
                                    : (uint64_t)2 * kvx::prefix_groups(16) * 16 * (m.d + 2) * 4);
    s.part[i].sums = take(rows * m.d * 4);
    s.part[i].stats = take(rows * 8);
    s.part[i].parts = take(rows * 8);
  }
  const int64_t most = kvx::kPrefixRows / ((int64_t)m.H * m.G);
  if (S > 0 && m.T > most && most > 0) {
    kvx_attend_dims fewer = m;
    fewer.T = (int32_t)most;
    const uint64_t n = prefix_space(fewer, S, dt).bytes;
    if (n > s.bytes) s.bytes = n;
  }
  return s;
}

size_t kvx_prefix_workspace_bytes(const kvx_attend_dims* dims, const kvx_prefix_dims* prefix, kvx_dtype dtype) {
  if (check_attend(dims, dtype) != KVX_OK || check_prefix(prefix) != KVX_OK || dims->B == 0 || dims->T == 0) return 0;
  return prefix_space(*dims, prefix->S, dtype == KVX_BF16 ? 0 : 1).bytes;
}

// The common part's sizes.
static void common_sizes(kvx::PrefixArgs& c, const kvx_prefix_dims& p, int log2p) {
  c.B = p.S;
  c.M = p.max_pages;
  c.keys = (int64_t)c.M << log2p;
  if (p.longest > 0 && p.longest < c.keys) c.keys = p.longest;
}

kvx_status kvx_prefix_kernel_names(const kvx_attend_dims* dims, const kvx_prefix_dims* prefix, const kvx_pool* pool,
                                   kvx_dtype dtype, const char** common, const char** own) {
  if (common == nullptr || own == nullptr) return set_error(KVX_ERR_NULL, "common or own is NULL");
  *common = *own = nullptr;
  int log2p;
  kvx_status st = check_pool(pool, true, &log2p);
  if (st != KVX_OK) return st;
  if ((st = check_attend(dims, dtype)) != KVX_OK) return st;
  if ((st = check_prefix(prefix)) != KVX_OK) return st;
  if (dims->B == 0 || dims->T == 0) return ok();
  kvx::PrefixArgs o;
  std::memset(&o, 0, sizeof(o));
  static_cast<kvx::AttendArgs&>(o) = attend_sizes(*dims, *pool, log2p);
  const int dt = dtype == KVX_BF16 ? 0 : 1;
  if (prefix->S == 0) {
    *own = kvx::attend_kernel_name(o, dt, dims->d);
    return ok();
  }
  kvx::PrefixArgs c = o;
  common_sizes(c, *prefix, log2p);
  kvx::prefix_kernel_names(c, o, dt, dims->d, common, own);
  return ok();
}

kvx_status kvx_attend_prefix8(const kvx_attend_dims* dims, const kvx_prefix_dims* prefix, const kvx_pool* pool,
                              kvx_dtype dtype, const void* q, const int64_t* q_strides, const uint8_t* codes,
                              const float* scales, const int32_t* prefix_tables, const int32_t* prefix_lens,
                              const int32_t* prefix_cu, const int32_t* block_tables, const int32_t* lens,
                              const int32_t* cu, float scale, void* out, float* lse, void* workspace,
                              size_t workspace_bytes, void* stream) {
  int log2p;
  kvx_status st = check_pool(pool, true, &log2p);
  if (st != KVX_OK) return st;
  if ((st = check_attend(dims, dtype)) != KVX_OK) return st;
  if ((st = check_prefix(prefix)) != KVX_OK) return st;
  const kvx_attend_dims& m = *dims;
  if (!std::isfinite(scale)) return set_error(KVX_ERR_SHAPE, "scale must be finite");
  if (m.B == 0 || m.T == 0) return ok();
  const int dt = dtype == KVX_BF16 ? 0 : 1, es = dt == 0 ? 2 : 4;
  const int32_t n[2] = {m.T, m.H * m.G}, S = prefix->S;
  uint64_t qb;
  if ((st = check_strides("q", q_strides, n, 2, es, m.d, &qb)) != KVX_OK) return st;
  const uint64_t pages = (uint64_t)2 * m.H * pool->num_pages, b4 = (uint64_t)m.B * 4, s4 = (uint64_t)S * 4;
  const uint64_t rows = (uint64_t)m.T * m.H * m.G;
  const PrefixSpace space = prefix_space(m, S, dt);
  const Span in[] = {{q, qb, "q"},
                     {codes, pages * pool->page_size * m.d, "codes"},
                     {scales, pages * 4, "scales"},
                     {block_tables, b4 * pool->max_pages, "block_tables"},
                     {lens, b4, "lens"},
                     {cu, b4 + 4, "cu"},
                     {prefix_tables, s4 * prefix->max_pages, "prefix_tables"},
                     {prefix_lens, s4, "prefix_lens"},
                     {prefix_cu, S > 0 ? s4 + 4 : 0, "prefix_cu"}};
  const Span outs[] = {{out, rows * m.d * es, "out"}, {lse, rows * 4, "lse"}, {workspace, space.bytes, "workspace"}};
  if ((st = check_pointers(in, 2, 16)) != KVX_OK) return st;
  if ((st = check_pointers(in + 2, S > 0 ? 7 : 4, 4)) != KVX_OK) return st;
  if ((st = check_pointers(outs, 1, 16)) != KVX_OK) return st;
  if (lse != nullptr && (st = check_pointers(outs + 1, 1, 4)) != KVX_OK) return st;
  if ((st = check_workspace(workspace, workspace_bytes, space.bytes)) != KVX_OK) return st;
  if ((st = check_alias(outs, 3, in, 9)) != KVX_OK) return st;
  kvx::PrefixArgs a;
  std::memset(&a, 0, sizeof(a));
  static_cast<kvx::AttendArgs&>(a) = attend_sizes(m, *pool, log2p);
  a.q = q;
  a.q_stride[0] = q_strides[0];
  a.q_stride[1] = q_strides[1];
  a.codes = codes;
  a.scales = scales;
  a.tables = block_tables;
  a.lens = lens;
  a.cu = cu;
  a.out = out;
  a.lse = lse;
  a.scale_log2 = scale * 1.44269504088896340736f;
  hipStream_t on = reinterpret_cast<hipStream_t>(stream);
  hipError_t e;
  if (S == 0) {
    e = kvx::launch_attend(a, dt, m.d, workspace, on);
  } else {
    a.shares = prefix_cu;
    a.prefixes = S;
    a.requests = m.B;
    kvx::PrefixArgs part[2] = {a, a};
    for (int i = 0; i < 2; ++i) {
      char* ws = static_cast<char*>(workspace);
      part[i].partial = reinterpret_cast<const float*>(ws + space.part[i].partial);
      part[i].sums = reinterpret_cast<float*>(ws + space.part[i].sums);
      part[i].stats = reinterpret_cast<float*>(ws + space.part[i].stats);
      part[i].parts = reinterpret_cast<uint64_t*>(ws + space.part[i].parts);
    }
    kvx::PrefixArgs& c = part[0];
    common_sizes(c, *prefix, log2p);
    c.tables = prefix_tables;
    c.lens = prefix_lens;
    e = kvx::launch_prefix(c, part[1], dt, m.d, workspace, on);
  }
  if (e != hipSuccess) return set_error(KVX_ERR_HIP, "prefix attention launch: %s", hipGetErrorString(e));
  return ok();
}

static kvx_status check_sample(kvx_dtype dtype, int32_t B, int32_t V) {
  kvx_status st = check_dtype(dtype);
  if (st != KVX_OK) return st;
  if (B < 0 || V < 1) return set_error(KVX_ERR_SHAPE, "B=%d V=%d out of range (B >= 0, V >= 1)", B, V);
  if (B > KVX_MAX_DRAWS || V > KVX_MAX_VOCABULARY)
    return set_error(KVX_ERR_UNSUPPORTED, "B=%d exceeds %d rows or V=%d exceeds %d tokens", B, KVX_MAX_DRAWS, V,
                     KVX_MAX_VOCABULARY);
  return KVX_OK;
}

size_t kvx_sample_workspace_bytes(kvx_dtype dtype, int32_t B, int32_t V) {
  if (check_sample(dtype, B, V) != KVX_OK || B == 0) return 0;
  return kvx::sample_ws_bytes(B);
}

kvx_status kvx_sample_tokens(kvx_dtype dtype, int32_t B, int32_t V, const void* logits, int64_t stride,
                             const float* u, const float* temperature, const int32_t* top_k,
                             const float* top_p, const float* min_p, int32_t* tokens, float* logprob,
                             void* workspace, size_t workspace_bytes, void* stream) {
  kvx_status st = check_sample(dtype, B, V);
  if (st != KVX_OK) return st;
  const int dt = dtype == KVX_BF16 ? 0 : 1, es = dt == 0 ? 2 : 4;
  if (B > 1 && stride < 0) return set_error(KVX_ERR_SHAPE, "logits stride %lld is negative", (long long)stride);
  const unsigned __int128 bytes = ((unsigned __int128)(B > 1 ? B - 1 : 0) * (uint64_t)(B > 1 ? stride : 0) + (uint32_t)V) * es;
  if (bytes >= (uint64_t)1 << 60) return set_error(KVX_ERR_SHAPE, "logits stride reaches too far");
  if (B == 0) return ok();
  const uint64_t b4 = (uint64_t)B * 4, need = kvx::sample_ws_bytes(B);
  const Span in[] = {{logits, (uint64_t)bytes, "logits"}, {u, b4, "u"},          {temperature, b4, "temperature"},
                     {top_k, b4, "top_k"},               {top_p, b4, "top_p"}, {min_p, b4, "min_p"}};
  const Span out[] = {{tokens, b4, "tokens"}, {logprob, b4, "logprob"}, {workspace, need, "workspace"}};
  if ((st = check_pointers(in, 1, es)) != KVX_OK) return st;
  if ((st = check_pointers(in + 1, 1, 4)) != KVX_OK) return st;
  for (int i = 2; i < 6; ++i)
    if (in[i].p != nullptr && (st = check_pointers(in + i, 1, 4)) != KVX_OK) return st;
  if ((st = check_pointers(out, 1, 4)) != KVX_OK) return st;
  if (logprob != nullptr && (st = check_pointers(out + 1, 1, 4)) != KVX_OK) return st;
  if ((st = check_workspace(workspace, workspace_bytes, need)) != KVX_OK) return st;
  if ((st = check_alias(out, 3, in, 6)) != KVX_OK) return st;
  kvx::SampleArgs a;
  std::memset(&a, 0, sizeof(a));
  a.logits = logits;
  a.stride = stride;
  a.u = u;
  a.temperature = temperature;
  a.top_k = top_k;
  a.top_p = top_p;
  a.min_p = min_p;
  a.tokens = tokens;
  a.logprob = logprob;
  a.B = B;
  a.V = V;
  const hipError_t e = kvx::launch_sample(a, dt, workspace, reinterpret_cast<hipStream_t>(stream));
  if (e != hipSuccess) return set_error(KVX_ERR_HIP, "token sampling launch: %s", hipGetErrorString(e));
  return ok();
}

}  // extern "C"
