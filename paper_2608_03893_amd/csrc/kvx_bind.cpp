// Argument marshalling of the serving calls (the extension module _kvx_bind; plain C++).
//
// They take 3 to 20 us on the GPU, a launch takes 3 us on the host, and to look at a dozen
// tensors and make the outputs in Python takes 4 to 10 us more.  Here that takes one: the
// same checks and the same exceptions, then the entry point of libkvx.so, whose address
// `bind` gets from the binding.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <c10/core/DeviceGuard.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <climits>
#include <cmath>

#include "kvx.h"

namespace {

decltype(&kvx_plan_pages) plan_pages_entry = nullptr;
decltype(&kvx_store_cache8) store_cache8_entry = nullptr;
decltype(&kvx_attend_cache8) attend_cache8_entry = nullptr;
decltype(&kvx_attend_workspace_bytes) attend_workspace_bytes_entry = nullptr;
decltype(&kvx_norm_rope) norm_rope_entry = nullptr;
decltype(&kvx_sample_workspace_bytes) sample_workspace_bytes_entry = nullptr;
decltype(&kvx_sample_tokens) sample_tokens_entry = nullptr;
decltype(&kvx_prefix_workspace_bytes) prefix_workspace_bytes_entry = nullptr;
decltype(&kvx_attend_prefix8) attend_prefix8_entry = nullptr;
PyObject* check_status = nullptr;    // raises for a status that is not KVX_OK
PyObject* plan_type = nullptr;       // the tuple plan_pages returns
PyObject* current_stream = nullptr;  // raw handle of a device's current stream

const at::Tensor& tensor(PyObject* o, const char* name) {
  TORCH_CHECK_TYPE(THPVariable_Check(o), name, " must be a tensor");
  return THPVariable_Unpack(o);
}

int32_t size32(int64_t n) {
  TORCH_CHECK_VALUE(n >= INT_MIN && n <= INT_MAX, "a size of ", n, " does not fit 32 bits");
  return (int32_t)n;
}

// The device of a call, that of one of its tensors; the others have to live there too.
struct Place {
  at::Device device;
  void check(const at::Tensor& t, const char* name) const {
    TORCH_CHECK_VALUE(t.is_cuda(), name, " must live on the GPU");
    TORCH_CHECK_VALUE(t.device() == device, name, " lives on ", t.device(), ", other operands on ", device);
  }
};

void* address(const Place& place, const at::Tensor& t, const char* name) {
  place.check(t, name);
  TORCH_CHECK_VALUE(t.is_contiguous(), name, " must be contiguous");
  return t.data_ptr();
}

// A tensor whose last dimension is dense, whatever its other strides.
const void* rows_address(const Place& place, const at::Tensor& t, const char* name) {
  place.check(t, name);
  TORCH_CHECK_VALUE(t.stride(-1) == 1 || t.size(-1) <= 1, name, " must be dense in its last dimension");
  return t.data_ptr();
}

int32_t* int32_at(const Place& place, const at::Tensor& t, const char* name, at::IntArrayRef shape) {
  TORCH_CHECK_VALUE(t.scalar_type() == at::kInt && t.sizes() == shape, name, " must be int32 ", shape, ", got ",
                    t.scalar_type(), ' ', t.sizes());
  return static_cast<int32_t*>(address(place, t, name));
}

kvx_dtype dtype_of(const at::Tensor& t) {
  if (t.scalar_type() == at::kBFloat16) return KVX_BF16;
  TORCH_CHECK_TYPE(t.scalar_type() == at::kFloat, "unsupported dtype ", t.scalar_type(), " (bfloat16 or float32)");
  return KVX_F32;
}

// kvx_pool of an 8-bit pool [*lead, num_slots, d] and its scales [*lead, num_pages].
kvx_pool pool_of(const at::Tensor& pool, const at::Tensor& scales, at::IntArrayRef lead, int32_t max_pages) {
  const int64_t n = (int64_t)lead.size();
  TORCH_CHECK_VALUE(pool.scalar_type() == at::kFloat8_e4m3fn && pool.dim() == n + 2 && pool.sizes().slice(0, n) == lead,
                    "pool must be float8_e4m3fn ", lead, " + [num_slots, d]");
  TORCH_CHECK_VALUE(scales.scalar_type() == at::kFloat && scales.dim() == n + 1 && scales.sizes().slice(0, n) == lead,
                    "scales must be float32 ", lead, " + [num_pages]");
  const int64_t slots = pool.size(n), pages = scales.size(n);
  TORCH_CHECK_VALUE(pages >= 1 && slots % pages == 0, slots, " slots do not divide into ", pages, " pages");
  return kvx_pool{size32(pages), size32(slots / pages), max_pages};
}

void* stream_of(PyObject* raw, const at::Tensor& t) {
  if (raw != Py_None) return PyLong_AsVoidPtr(raw);
  PyObject* device = PyLong_FromLong(t.get_device());
  PyObject* handle = device == nullptr ? nullptr : PyObject_CallOneArg(current_stream, device);
  Py_XDECREF(device);
  if (handle == nullptr) throw python_error();
  void* s = PyLong_AsVoidPtr(handle);
  Py_DECREF(handle);
  return s;
}

// On the operands' device: a launch on its default stream, whose handle is 0, would go to the
// current device else.
template <typename F, typename... A>
void call(const Place& place, F entry, A... a) {
  const c10::DeviceGuard guard(place.device);
  kvx_status status;
  Py_BEGIN_ALLOW_THREADS
  status = entry(a...);
  Py_END_ALLOW_THREADS
  if (status == KVX_OK) return;
  PyObject* r = PyObject_CallFunction(check_status, "i", (int)status);
  Py_XDECREF(r);
  if (r == nullptr) throw python_error();
}

void arguments(Py_ssize_t got, Py_ssize_t want) {
  TORCH_CHECK_TYPE(got == want, got, " arguments instead of ", want);
  TORCH_CHECK(attend_cache8_entry != nullptr, "bind has not been called");
}

// An int32 vector of `n` elements from `first` on in the storage of `all`.
at::Tensor part(const at::Tensor& all, int64_t first, int64_t n) {
  at::Tensor t = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(all.storage()), all.key_set(), all.dtype());
  t.unsafeGetTensorImpl()->set_storage_offset(first);
  t.unsafeGetTensorImpl()->set_sizes_contiguous({n});
  return t;
}

// plan_pages(lens, add, block_tables, free_ring, free, T, page_size, out or None, stream or None)
PyObject* plan_pages(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  arguments(nargs, 9);
  const at::Tensor &lens = tensor(args[0], "lens"), &add = tensor(args[1], "add");
  const at::Tensor &tables = tensor(args[2], "block_tables"), &ring = tensor(args[3], "free_ring");
  const at::Tensor& free = tensor(args[4], "free");
  TORCH_CHECK_VALUE(tables.dim() == 2 && ring.dim() == 1, "block_tables must be [B, max_pages], free_ring [num_pages]");
  TORCH_CHECK_VALUE(free.scalar_type() == at::kInt && free.dim() == 1 && free.size(0) >= 2,
                    "free must be int32 with the ring's first place and count");
  const int64_t T = PyLong_AsLongLong(args[5]), page_size = PyLong_AsLongLong(args[6]);
  if (PyErr_Occurred()) throw python_error();
  const int64_t B = tables.size(0), M = tables.size(1), N = ring.size(0);
  const kvx_pool pool{size32(N), size32(page_size), size32(M)};
  const int32_t rows32 = size32(T);
  const Place place{lens.device()};
  const int32_t *lens_at = int32_at(place, lens, "lens", {B}), *add_at = int32_at(place, add, "add", {B});
  int32_t *tables_at = int32_at(place, tables, "block_tables", {B, M}), *ring_at = int32_at(place, ring, "free_ring", {N});
  const int32_t* free_at = static_cast<const int32_t*>(address(place, free, "free"));
  int32_t* outs[5];   // lens, cu, positions, slots, free
  const int64_t shape[5] = {B, B + 1, T, T, 4};
  PyObject* result = nullptr;
  if (args[7] == Py_None) {   // one allocation; positions and slots start on 16 bytes
    const int64_t rows = T < 0 ? 0 : (T + 3) / 4 * 4, first[5] = {2 * rows, 2 * rows + B, 0, rows, 2 * rows + 2 * B + 1};
    const at::Tensor all = at::empty({2 * rows + 2 * B + 5}, lens.options());
    PyObject* items = PyTuple_New(5);
    if (items == nullptr) throw python_error();
    for (int i = 0; i < 5; ++i) {
      at::Tensor t = part(all, first[i], shape[i] < 0 ? 0 : shape[i]);
      outs[i] = static_cast<int32_t*>(t.data_ptr());
      PyTuple_SET_ITEM(items, i, THPVariable_Wrap(std::move(t)));
    }
    PyObject* one = PyTuple_Pack(1, items);
    Py_DECREF(items);
    if (one == nullptr) throw python_error();
    result = PyTuple_Type.tp_new(reinterpret_cast<PyTypeObject*>(plan_type), one, nullptr);
    Py_DECREF(one);
    if (result == nullptr) throw python_error();
  } else {
    static const char* const names[5] = {"lens", "cu", "positions", "slots", "free"};
    TORCH_CHECK_TYPE(PyTuple_Check(args[7]) && PyTuple_GET_SIZE(args[7]) == 5, "out must be a PagePlan");
    for (int i = 0; i < 5; ++i) outs[i] = int32_at(place, tensor(PyTuple_GET_ITEM(args[7], i), names[i]), names[i], {shape[i]});
    result = args[7];
    Py_INCREF(result);
  }
  try {
    call(place, plan_pages_entry, &pool, size32(B), rows32, lens_at, add_at, tables_at, ring_at, free_at, outs[0], outs[1],
         outs[2], outs[3], outs[4], stream_of(args[8], lens));
  } catch (...) {
    Py_DECREF(result);
    throw;
  }
  return result;
  END_HANDLE_TH_ERRORS
}

// store_cache8(k, v, slot_mapping, pool, scales, stream or None)
PyObject* store_cache8(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  arguments(nargs, 6);
  const at::Tensor &k = tensor(args[0], "k"), &v = tensor(args[1], "v"), &slots = tensor(args[2], "slot_mapping");
  const at::Tensor &codes = tensor(args[3], "pool"), &scales = tensor(args[4], "scales");
  TORCH_CHECK_VALUE(k.dim() == 4 && v.sizes() == k.sizes() && v.scalar_type() == k.scalar_type(),
                    "k and v must be [L, H, T, d] of one dtype");
  const int64_t L = k.size(0), H = k.size(1), T = k.size(2), d = k.size(3);
  const kvx_pool pool = pool_of(codes, scales, {L, 2, H}, 1);
  TORCH_CHECK_VALUE(codes.size(4) == d, "pool rows have ", codes.size(4), " channels, k and v ", d);
  const Place place{k.device()};
  const int64_t ks[3] = {k.stride(0), k.stride(1), k.stride(2)}, vs[3] = {v.stride(0), v.stride(1), v.stride(2)};
  const kvx_dtype dtype = dtype_of(k);
  const void *k_at = rows_address(place, k, "k"), *v_at = rows_address(place, v, "v");
  const int32_t* slots_at = int32_at(place, slots, "slot_mapping", {T});
  uint8_t* codes_at = static_cast<uint8_t*>(address(place, codes, "pool"));
  float* scales_at = static_cast<float*>(address(place, scales, "scales"));
  call(place, store_cache8_entry, &pool, dtype, size32(L), size32(H), size32(T), size32(d), k_at, ks, v_at, vs, slots_at,
       codes_at, scales_at, stream_of(args[5], k));
  Py_INCREF(args[3]);
  return args[3];
  END_HANDLE_TH_ERRORS
}

// What both attention calls have: operands, sizes, outputs.
struct Attention {
  const at::Tensor &q, &codes, &scales, &tables;
  const int64_t T, heads, d, H, B, M;
  const kvx_pool pool;
  const kvx_attend_dims dims;
  const kvx_dtype dtype;
  const Place place;
  const void* q_at;
  const int64_t strides[2];
  const uint8_t* codes_at;
  const float* scales_at;
  const int32_t *tables_at, *lens_at, *cu_at;
  float scale;
  int with_lse;
  at::Tensor out, lse;

  static const at::Tensor& shaped(const at::Tensor& q, const at::Tensor& codes, const at::Tensor& tables) {
    TORCH_CHECK_VALUE(q.dim() == 3 && codes.dim() == 4 && tables.dim() == 2,
                      "q must be [T, H*G, d], pool [2, H, num_slots, d], block_tables [B, max_pages]");
    TORCH_CHECK_VALUE(codes.size(1) >= 1 && q.size(1) % codes.size(1) == 0 && codes.size(3) == q.size(2), q.size(1),
                      " query heads of ", q.size(2), " channels on a pool of ", codes.size(1), " heads of ", codes.size(3));
    return q;
  }
  Attention(PyObject* q_, PyObject* codes_, PyObject* scales_, PyObject* tables_, PyObject* lens, PyObject* cu,
            PyObject* scale_, PyObject* lse_, PyObject* longest)
      : q(shaped(tensor(q_, "q"), tensor(codes_, "pool"), tensor(tables_, "block_tables"))), codes(tensor(codes_, "pool")),
        scales(tensor(scales_, "scales")), tables(tensor(tables_, "block_tables")), T(q.size(0)), heads(q.size(1)),
        d(q.size(2)), H(codes.size(1)), B(tables.size(0)), M(tables.size(1)), pool(pool_of(codes, scales, {2, H}, size32(M))),
        dims{size32(B), size32(H), size32(heads / H), size32(T), size32(d), size32(PyLong_AsLongLong(longest))},
        dtype(dtype_of(q)), place{q.device()}, q_at(rows_address(place, q, "q")), strides{q.stride(0), q.stride(1)},
        codes_at(static_cast<const uint8_t*>(address(place, codes, "pool"))),
        scales_at(static_cast<const float*>(address(place, scales, "scales"))),
        tables_at(int32_at(place, tables, "block_tables", {B, M})), lens_at(int32_at(place, tensor(lens, "lens"), "lens", {B})),
        cu_at(int32_at(place, tensor(cu, "cu"), "cu", {B + 1})),
        scale((float)(scale_ == Py_None ? 1.0 / std::sqrt((double)d) : PyFloat_AsDouble(scale_))),
        with_lse(PyObject_IsTrue(lse_)) {
    if (PyErr_Occurred()) throw python_error();
  }
  // The workspace given, or one of `need` bytes whose counters are cleared.
  at::Tensor workspace(PyObject* given, size_t need) const {
    if (given != Py_None) return tensor(given, "workspace");
    const at::Tensor w = at::empty({need > 0 ? (int64_t)need : 1}, q.options().dtype(at::kByte));
    if (need > 0) w.narrow(0, 0, KVX_ATTEND_COUNTER_BYTES).zero_();
    return w;
  }
  void outputs(PyObject* given) {
    if (given == Py_None) {
      out = at::empty(q.sizes(), q.options());
    } else {
      out = tensor(given, "out");
      TORCH_CHECK_VALUE(out.sizes() == q.sizes() && out.scalar_type() == q.scalar_type(), "out must have q's shape and dtype");
    }
    if (with_lse) lse = at::empty({T, heads}, q.options().dtype(at::kFloat));
  }
  float* lse_at() const { return with_lse ? static_cast<float*>(lse.data_ptr()) : nullptr; }
  PyObject* result(PyObject* given) {
    PyObject* first = given;
    if (given == Py_None) first = THPVariable_Wrap(std::move(out));
    else Py_INCREF(given);
    if (!with_lse || first == nullptr) return first;
    PyObject* second = THPVariable_Wrap(std::move(lse));
    PyObject* both = second == nullptr ? nullptr : PyTuple_Pack(2, first, second);
    Py_DECREF(first);
    Py_XDECREF(second);
    return both;
  }
};

// attend_cache8(q, pool, scales, block_tables, lens, cu, scale or None, out or None, with_lse,
//               workspace or None, stream or None, longest)
PyObject* attend_cache8(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  arguments(nargs, 12);
  Attention x(args[0], args[1], args[2], args[3], args[4], args[5], args[6], args[8], args[11]);
  const at::Tensor workspace = x.workspace(args[9], args[9] == Py_None ? attend_workspace_bytes_entry(&x.dims, x.dtype) : 0);
  x.outputs(args[7]);
  call(x.place, attend_cache8_entry, &x.dims, &x.pool, x.dtype, x.q_at, x.strides, x.codes_at, x.scales_at, x.tables_at,
       x.lens_at, x.cu_at, x.scale, address(x.place, x.out, "out"), x.lse_at(), address(x.place, workspace, "workspace"),
       (size_t)workspace.numel(), stream_of(args[10], x.q));
  return x.result(args[7]);
  END_HANDLE_TH_ERRORS
}

// attend_prefix8(q, pool, scales, prefix_tables, prefix_lens, prefix_cu, block_tables, lens, cu, scale or
//                None, out or None, with_lse, workspace or None, stream or None, longest, longest_prefix)
PyObject* attend_prefix8(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  arguments(nargs, 16);
  Attention x(args[0], args[1], args[2], args[6], args[7], args[8], args[9], args[11], args[14]);
  const at::Tensor& tables = tensor(args[3], "prefix_tables");
  TORCH_CHECK_VALUE(tables.dim() == 2, "prefix_tables must be [S, max_pages]");
  const int64_t S = tables.size(0), M = tables.size(1), longest = PyLong_AsLongLong(args[15]);
  if (PyErr_Occurred()) throw python_error();
  const kvx_prefix_dims prefix{size32(S), size32(M), size32(longest)};
  const int32_t *tables_at = int32_at(x.place, tables, "prefix_tables", {S, M}),
                *lens_at = int32_at(x.place, tensor(args[4], "prefix_lens"), "prefix_lens", {S}),
                *cu_at = int32_at(x.place, tensor(args[5], "prefix_cu"), "prefix_cu", {S + 1});
  const at::Tensor workspace =
      x.workspace(args[12], args[12] == Py_None ? prefix_workspace_bytes_entry(&x.dims, &prefix, x.dtype) : 0);
  x.outputs(args[10]);
  call(x.place, attend_prefix8_entry, &x.dims, &prefix, &x.pool, x.dtype, x.q_at, x.strides, x.codes_at, x.scales_at, tables_at,
       lens_at, cu_at, x.tables_at, x.lens_at, x.cu_at, x.scale, address(x.place, x.out, "out"), x.lse_at(),
       address(x.place, workspace, "workspace"), (size_t)workspace.numel(), stream_of(args[13], x.q));
  return x.result(args[10]);
  END_HANDLE_TH_ERRORS
}

// norm_rope(q, k or None, q_weight or None, k_weight or None, address of a kvx_rope, positions, eps,
//           (q_out, k_out or None) or None, stream or None)
PyObject* norm_rope(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  arguments(nargs, 9);
  const bool keys = args[1] != Py_None;
  const at::Tensor &q = tensor(args[0], "q"), &k = keys ? tensor(args[1], "k") : q;
  const at::Tensor& positions = tensor(args[5], "positions");
  TORCH_CHECK_VALUE(q.dim() == 3 && k.dim() == 3 && k.size(0) == q.size(0) && k.size(2) == q.size(2) &&
                        k.scalar_type() == q.scalar_type(),
                    "q must be [T, H*G, d] and k [T, H, d], of one dtype");
  TORCH_CHECK_VALUE(k.size(1) >= 1, "k has no heads");
  const int64_t T = q.size(0), d = q.size(2);
  const kvx_dtype dtype = dtype_of(q);
  const Place place{q.device()};
  const void *x[2] = {rows_address(place, q, "q"), keys ? rows_address(place, k, "k") : nullptr}, *weight[2] = {nullptr, nullptr};
  const int64_t qs[2] = {q.stride(0), q.stride(1)}, ks[2] = {k.stride(0), k.stride(1)};
  static const char* const names[2] = {"q_weight", "k_weight"};
  for (int i = 0; i < 2; ++i) {
    if (args[2 + i] == Py_None) continue;
    TORCH_CHECK_VALUE(i == 0 || keys, "k_weight without k");
    const at::Tensor& w = tensor(args[2 + i], names[i]);
    TORCH_CHECK_VALUE(w.sizes() == at::IntArrayRef{d} && w.scalar_type() == q.scalar_type(), names[i],
                      " must be [d] with q's dtype");
    weight[i] = address(place, w, names[i]);
  }
  const kvx_rope* rope = static_cast<const kvx_rope*>(PyLong_AsVoidPtr(args[4]));
  const double eps = PyFloat_AsDouble(args[6]);
  if (PyErr_Occurred()) throw python_error();
  const int32_t* positions_at = int32_at(place, positions, "positions", {T});
  at::Tensor out[2];
  if (args[7] == Py_None) {
    out[0] = at::empty(q.sizes(), q.options());
    if (keys) out[1] = at::empty(k.sizes(), k.options());
  } else {
    TORCH_CHECK_TYPE(PyTuple_Check(args[7]) && PyTuple_GET_SIZE(args[7]) == 2, "out must be a pair (q, k)");
    for (int i = 0; i <= (keys ? 1 : 0); ++i) {
      out[i] = tensor(PyTuple_GET_ITEM(args[7], i), i == 0 ? "out[0]" : "out[1]");
      const at::Tensor& like = i == 0 ? q : k;
      TORCH_CHECK_VALUE(out[i].sizes() == like.sizes() && out[i].scalar_type() == like.scalar_type(),
                        "out must have the shapes and dtype of q and k");
    }
  }
  call(place, norm_rope_entry, dtype, size32(T), size32(q.size(1)), keys ? size32(k.size(1)) : 0, size32(d), x[0], qs, x[1],
       ks, weight[0], weight[1], (float)eps, rope, positions_at, address(place, out[0], "out[0]"),
       keys ? address(place, out[1], "out[1]") : nullptr, stream_of(args[8], q));
  if (args[7] != Py_None) {
    Py_INCREF(args[7]);
    return args[7];
  }
  PyObject* pair = PyTuple_New(2);
  if (pair == nullptr) throw python_error();
  PyTuple_SET_ITEM(pair, 0, THPVariable_Wrap(std::move(out[0])));
  if (!keys) Py_INCREF(Py_None);
  PyTuple_SET_ITEM(pair, 1, keys ? THPVariable_Wrap(std::move(out[1])) : Py_None);
  return pair;
  END_HANDLE_TH_ERRORS
}

// sample_tokens(logits, u, temperature, top_k, top_p, min_p (or None), out or None, with_logprob,
//               workspace or None, stream or None)
PyObject* sample_tokens(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  arguments(nargs, 10);
  const at::Tensor& logits = tensor(args[0], "logits");
  TORCH_CHECK_VALUE(logits.dim() == 2, "logits must be [B, V]");
  const int64_t B = logits.size(0), V = logits.size(1);
  const kvx_dtype dtype = dtype_of(logits);
  const Place place{logits.device()};
  const void* logits_at = rows_address(place, logits, "logits");
  auto floats = [&](PyObject* o, const char* name) -> const float* {
    if (o == Py_None) return nullptr;
    const at::Tensor& t = tensor(o, name);
    TORCH_CHECK_VALUE(t.scalar_type() == at::kFloat && t.sizes() == at::IntArrayRef{B}, name, " must be float32 [B]");
    return static_cast<const float*>(address(place, t, name));
  };
  TORCH_CHECK_TYPE(THPVariable_Check(args[1]), "u must be a tensor");
  const float *u_at = floats(args[1], "u"), *temperature = floats(args[2], "temperature");
  const int32_t* top_k = args[3] == Py_None ? nullptr : int32_at(place, tensor(args[3], "top_k"), "top_k", {B});
  const float *top_p = floats(args[4], "top_p"), *min_p = floats(args[5], "min_p");
  const int with_logprob = PyObject_IsTrue(args[7]);
  if (PyErr_Occurred()) throw python_error();
  const int32_t B32 = size32(B), V32 = size32(V);
  at::Tensor out, logprob, workspace;
  if (args[8] == Py_None) {
    const int64_t need = (int64_t)sample_workspace_bytes_entry(dtype, B32, V32);
    if (need > 0) {
      workspace = at::empty({need}, logits.options().dtype(at::kByte));
      workspace.view({B, -1}).narrow(1, 0, KVX_SAMPLE_COUNTER_BYTES).zero_();
    }
  } else {
    workspace = tensor(args[8], "workspace");
  }
  if (args[6] == Py_None) out = at::empty({B}, logits.options().dtype(at::kInt));
  else out = tensor(args[6], "out");
  int32_t* tokens = int32_at(place, out, "out", {B});
  if (with_logprob) logprob = at::empty({B}, logits.options().dtype(at::kFloat));
  call(place, sample_tokens_entry, dtype, B32, V32, logits_at, logits.stride(0), u_at, temperature, top_k, top_p, min_p, tokens,
       with_logprob ? static_cast<float*>(logprob.data_ptr()) : nullptr,
       workspace.defined() ? address(place, workspace, "workspace") : nullptr,
       workspace.defined() ? (size_t)workspace.nbytes() : (size_t)0, stream_of(args[9], logits));
  PyObject* result = args[6];
  if (result == Py_None) result = THPVariable_Wrap(std::move(out));
  else Py_INCREF(result);
  if (!with_logprob || result == nullptr) return result;
  PyObject* second = THPVariable_Wrap(std::move(logprob));
  PyObject* both = second == nullptr ? nullptr : PyTuple_Pack(2, result, second);
  Py_DECREF(result);
  Py_XDECREF(second);
  return both;
  END_HANDLE_TH_ERRORS
}

template <typename F>
bool entry(PyObject* args, Py_ssize_t i, F* to) {
  void* p = PyLong_AsVoidPtr(PyTuple_GET_ITEM(args, i));
  if (PyErr_Occurred()) return false;
  *to = reinterpret_cast<F>(p);
  return true;
}

// bind(check_status, plan_type, current_stream, addresses of kvx_plan_pages, kvx_store_cache8,
//      kvx_attend_cache8, kvx_attend_workspace_bytes, kvx_norm_rope, kvx_sample_workspace_bytes,
//      kvx_sample_tokens, kvx_prefix_workspace_bytes, kvx_attend_prefix8)
PyObject* bind(PyObject*, PyObject* args) {
  if (PyTuple_GET_SIZE(args) != 12) {
    PyErr_SetString(PyExc_TypeError, "bind takes 12 arguments");
    return nullptr;
  }
  PyObject* type = PyTuple_GET_ITEM(args, 1);
  if (!PyType_Check(type) || !PyType_IsSubtype(reinterpret_cast<PyTypeObject*>(type), &PyTuple_Type)) {
    PyErr_SetString(PyExc_TypeError, "plan_type must be a tuple type");
    return nullptr;
  }
  if (!entry(args, 3, &plan_pages_entry) || !entry(args, 4, &store_cache8_entry) || !entry(args, 5, &attend_cache8_entry) ||
      !entry(args, 6, &attend_workspace_bytes_entry) || !entry(args, 7, &norm_rope_entry) ||
      !entry(args, 8, &sample_workspace_bytes_entry) || !entry(args, 9, &sample_tokens_entry) ||
      !entry(args, 10, &prefix_workspace_bytes_entry) || !entry(args, 11, &attend_prefix8_entry))
    return nullptr;
  check_status = PyTuple_GET_ITEM(args, 0);
  plan_type = type;
  current_stream = PyTuple_GET_ITEM(args, 2);
  Py_INCREF(check_status);
  Py_INCREF(plan_type);
  Py_INCREF(current_stream);
  Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"bind", bind, METH_VARARGS, nullptr},
    {"plan_pages", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(plan_pages)), METH_FASTCALL, nullptr},
    {"store_cache8", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(store_cache8)), METH_FASTCALL, nullptr},
    {"attend_cache8", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(attend_cache8)), METH_FASTCALL, nullptr},
    {"attend_prefix8", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(attend_prefix8)), METH_FASTCALL, nullptr},
    {"sample_tokens", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(sample_tokens)), METH_FASTCALL, nullptr},
    {"norm_rope", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(norm_rope)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_kvx_bind", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__kvx_bind() { return PyModule_Create(&module); }
