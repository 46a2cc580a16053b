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

// attend_cache8(q, pool, scales, block_tables, lens, cu, scale or None, out or None, with_lse,
//               workspace or None, stream or None, longest)
PyObject* attend_cache8(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  arguments(nargs, 12);
  const at::Tensor &q = tensor(args[0], "q"), &codes = tensor(args[1], "pool"), &scales = tensor(args[2], "scales");
  const at::Tensor &tables = tensor(args[3], "block_tables"), &lens = tensor(args[4], "lens"), &cu = tensor(args[5], "cu");
  TORCH_CHECK_VALUE(q.dim() == 3 && codes.dim() == 4 && tables.dim() == 2,
                    "q must be [T, H*G, d], pool [2, H, num_slots, d], block_tables [B, max_pages]");
  const int64_t T = q.size(0), heads = q.size(1), d = q.size(2), H = codes.size(1), B = tables.size(0), M = tables.size(1);
  TORCH_CHECK_VALUE(H >= 1 && heads % H == 0 && codes.size(3) == d, heads, " query heads of ", d,
                    " channels on a pool of ", H, " heads of ", codes.size(3));
  const kvx_pool pool = pool_of(codes, scales, {2, H}, size32(M));
  const kvx_attend_dims dims{size32(B), size32(H), size32(heads / H), size32(T), size32(d),
                             size32(PyLong_AsLongLong(args[11]))};
  const kvx_dtype dtype = dtype_of(q);
  const Place place{q.device()};
  const void* q_at = rows_address(place, q, "q");
  const int64_t strides[2] = {q.stride(0), q.stride(1)};
  const uint8_t* codes_at = static_cast<const uint8_t*>(address(place, codes, "pool"));
  const float* scales_at = static_cast<const float*>(address(place, scales, "scales"));
  const int32_t *tables_at = int32_at(place, tables, "block_tables", {B, M}), *lens_at = int32_at(place, lens, "lens", {B});
  const int32_t* cu_at = int32_at(place, cu, "cu", {B + 1});
  const double scale = args[6] == Py_None ? 1.0 / std::sqrt((double)d) : PyFloat_AsDouble(args[6]);
  const int with_lse = PyObject_IsTrue(args[8]);
  if (PyErr_Occurred()) throw python_error();
  at::Tensor out, lse, workspace;
  if (args[9] == Py_None) {
    const int64_t need = (int64_t)attend_workspace_bytes_entry(&dims, dtype);
    workspace = at::empty({need > 0 ? need : 1}, q.options().dtype(at::kByte));
    if (need > 0) workspace.narrow(0, 0, KVX_ATTEND_COUNTER_BYTES).zero_();
  } else {
    workspace = tensor(args[9], "workspace");
  }
  if (args[7] == Py_None) {
    out = at::empty(q.sizes(), q.options());
  } else {
    out = tensor(args[7], "out");
    TORCH_CHECK_VALUE(out.sizes() == q.sizes() && out.scalar_type() == q.scalar_type(), "out must have q's shape and dtype");
  }
  if (with_lse) lse = at::empty({T, heads}, q.options().dtype(at::kFloat));
  call(place, attend_cache8_entry, &dims, &pool, dtype, q_at, strides, codes_at, scales_at, tables_at, lens_at, cu_at,
       (float)scale, address(place, out, "out"), with_lse ? static_cast<float*>(lse.data_ptr()) : nullptr,
       address(place, workspace, "workspace"), (size_t)workspace.numel(), stream_of(args[10], q));
  PyObject* result = args[7];
  if (result == Py_None) result = THPVariable_Wrap(std::move(out));
  else Py_INCREF(result);
  if (!with_lse || result == nullptr) return result;
  PyObject* second = THPVariable_Wrap(std::move(lse));
  PyObject* both = second == nullptr ? nullptr : PyTuple_Pack(2, result, second);
  Py_DECREF(result);
  Py_XDECREF(second);
  return both;
  END_HANDLE_TH_ERRORS
}

// bind(addresses of kvx_plan_pages, kvx_store_cache8, kvx_attend_cache8 and
//      kvx_attend_workspace_bytes, check_status, plan_type, current_stream)
PyObject* bind(PyObject*, PyObject* args) {
  PyObject *plan, *store, *attend, *bytes, *check, *type, *stream;
  if (!PyArg_ParseTuple(args, "OOOOOO!O", &plan, &store, &attend, &bytes, &check, &PyType_Type, &type, &stream))
    return nullptr;
  void *p = PyLong_AsVoidPtr(plan), *s = PyLong_AsVoidPtr(store), *a = PyLong_AsVoidPtr(attend), *w = PyLong_AsVoidPtr(bytes);
  if (PyErr_Occurred()) return nullptr;
  if (!PyType_IsSubtype(reinterpret_cast<PyTypeObject*>(type), &PyTuple_Type)) {
    PyErr_SetString(PyExc_TypeError, "plan_type must be a tuple type");
    return nullptr;
  }
  Py_INCREF(check);
  Py_INCREF(type);
  Py_INCREF(stream);
  check_status = check;
  plan_type = type;
  current_stream = stream;
  plan_pages_entry = reinterpret_cast<decltype(plan_pages_entry)>(p);
  store_cache8_entry = reinterpret_cast<decltype(store_cache8_entry)>(s);
  attend_cache8_entry = reinterpret_cast<decltype(attend_cache8_entry)>(a);
  attend_workspace_bytes_entry = reinterpret_cast<decltype(attend_workspace_bytes_entry)>(w);
  Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"bind", bind, METH_VARARGS, nullptr},
    {"plan_pages", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(plan_pages)), METH_FASTCALL, nullptr},
    {"store_cache8", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(store_cache8)), METH_FASTCALL, nullptr},
    {"attend_cache8", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(attend_cache8)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_kvx_bind", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__kvx_bind() { return PyModule_Create(&module); }
