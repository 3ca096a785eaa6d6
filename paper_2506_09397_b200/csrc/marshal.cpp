// Python arguments of the short calls - a decoding step's operators over a caller's paged cache - into the C entry points of sled.h.
//
// What binding.py does for the other calls, compiled: the same checks and messages, read from the tensors directly.  A step's
// call takes the GPU 3 - 12 us; its arguments took Python 7 - 12 us, and take 1 - 2 us here.
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <initializer_list>
#include <string>

#include "../../include/sled.h"

namespace {

PyObject* g_error = nullptr;       // SledError(code, what)

struct Refused {
  int code;
  std::string what;
};
[[noreturn]] void refuse(const char* what, const std::string& why) { throw Refused{SLED_ERR_ARG, std::string(what) + " (" + why + ")"}; }
void check(int code, const char* what) {
  if (code != SLED_OK) throw Refused{code, what};
}
// The call itself, without the interpreter's lock: a launch may wait for room in its stream's queue, and the stream for a host
// function that needs the lock.  Nothing of Python is touched meanwhile: tensors are the caller's, addresses are known.
template <typename Call>
int unlocked(Call call) {
  struct Unlocked {
    PyThreadState* state = PyEval_SaveThread();
    ~Unlocked() { PyEval_RestoreThread(state); }
  } now;
  return call();
}
struct NotATensor {
  std::string name;
};

const at::Tensor& tensor(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) throw NotATensor{name};
  return THPVariable_Unpack(o);
}
bool given(PyObject* o) { return o != Py_None; }
std::string on(int64_t dev) { return "on cuda:" + std::to_string(dev); }
template <typename T>
T* address(const at::Tensor& t) { return static_cast<T*>(t.data_ptr()); }

int32_t in_32_bits(PyObject* o, const char* what, const char* name) {
  int overflow = 0;
  const long long x = PyLong_AsLongLongAndOverflow(o, &overflow);
  if (x == -1 && !overflow && PyErr_Occurred()) throw Refused{1, ""};
  if (overflow || x < INT32_MIN || x > INT32_MAX) refuse(what, std::string(name) + " must be below 2^31");
  return static_cast<int32_t>(x);
}

// an int32 tensor that is contiguous along its last dimension, if it has any
int32_t* ints(const at::Tensor& t, const char* what, const char* name, int64_t dev) {
  if (t.scalar_type() != at::kInt || t.get_device() != dev || (t.dim() && t.size(-1) > 1 && t.stride(-1) != 1))
    refuse(what, std::string(name) + " must be an int32 tensor " + on(dev) + ", contiguous along its last dimension");
  return address<int32_t>(t);
}
int32_t* status_of(PyObject* o, const char* what, int64_t dev) {
  if (!given(o)) return nullptr;
  const at::Tensor& t = tensor(o, "status");
  if (!t.numel()) refuse(what, "status must have an entry");
  return ints(t, what, "status", dev);
}
template <typename T>
T* vector_of(PyObject* o, const char* what, const char* name, int64_t dev, int64_t n, at::ScalarType type) {
  const at::Tensor& t = tensor(o, name);
  if (t.scalar_type() != type || t.get_device() != dev || t.dim() != 1 || t.numel() != n || !t.is_contiguous())
    refuse(what, std::string(name) + " must be a contiguous " + c10::toString(type) + " vector of " + std::to_string(n) + " " + on(dev));
  return address<T>(t);
}
float* floats(const at::Tensor& t, const char* what, const char* name, int64_t dev, std::initializer_list<int64_t> shape) {
  if (t.scalar_type() != at::kFloat || t.get_device() != dev || t.sizes() != at::IntArrayRef(shape) || !t.is_contiguous())
    refuse(what, std::string(name) + " must be a contiguous fp32 tensor of another shape, or " + on(dev));
  return address<float>(t);
}
void* stream_of(int64_t dev) { return c10::cuda::getCurrentCUDAStream(static_cast<c10::DeviceIndex>(dev)).stream(); }

int type_of(const at::Tensor& t, bool codes) {
  if (t.scalar_type() == at::kFloat) return SLED_F32;
  if (t.scalar_type() == at::kBFloat16) return SLED_BF16;
  return codes && t.scalar_type() == at::kFloat8_e4m3fn ? SLED_E4M3 : -1;
}

// the cache description of a call
sled_paged_kv paged(const char* what, const at::Tensor& k, const at::Tensor& v, const at::Tensor& table, const at::Tensor& n_kv) {
  if (!k.is_cuda()) throw Refused{SLED_ERR_NO_DEVICE, std::string(what) + " (tensors must be on a CUDA device)"};
  const int64_t dev = k.get_device();
  const int type = type_of(k, true);
  if (type < 0 || k.dim() != 4) refuse(what, "the cache must be fp32, bf16 or e4m3, [n_pages, n_kv_heads, page_size, head_dim]");
  if (!k.is_contiguous() || v.scalar_type() != k.scalar_type() || v.get_device() != dev || v.sizes() != k.sizes() || !v.is_contiguous())
    refuse(what, "k must be contiguous, and v like k");
  if (table.dim() != 2 || n_kv.dim() != 1 || n_kv.numel() != table.size(0)) refuse(what, "page_table [n_reqs, cols] and n_kv [n_reqs]");
  const int64_t n_reqs = table.size(0), cols = table.size(1), stride = n_reqs > 1 ? table.stride(0) : cols;
  if (stride < cols) refuse(what, "rows of page_table must not overlap");
  for (const int64_t x : {n_reqs, stride, k.size(0), k.size(1), k.size(2), k.size(3)})
    if (x > INT32_MAX) refuse(what, "sizes must be below 2^31");
  sled_paged_kv kv{};
  kv.k = k.data_ptr();
  kv.v = v.data_ptr();
  kv.dtype = type;
  kv.n_layers = 1;
  kv.n_pages = static_cast<int32_t>(k.size(0));
  kv.n_kv_heads = static_cast<int32_t>(k.size(1));
  kv.page_size = static_cast<int32_t>(k.size(2));
  kv.head_dim = static_cast<int32_t>(k.size(3));
  kv.page_table = ints(table, what, "page_table", dev);
  kv.table_stride = static_cast<int32_t>(stride);
  kv.table_cols = static_cast<int32_t>(cols);
  kv.n_kv = ints(n_kv, what, "n_kv", dev);
  kv.n_reqs = static_cast<int32_t>(n_reqs);
  return kv;
}

// elements between rows [rows, heads, h]; a row itself is contiguous
int64_t row_stride(const at::Tensor& t, const char* what, const char* name) {
  const int64_t rows = t.size(0), heads = t.size(1), h = t.size(2);
  if (t.is_contiguous()) return heads * h;
  if (t.stride(2) != 1 || (heads > 1 && t.stride(1) != h)) refuse(what, std::string("a row of ") + name + " must be contiguous");
  return rows > 1 ? t.stride(0) : heads * h;
}
int32_t rows_of(const at::Tensor& t, const char* what) {
  if (t.size(0) > INT32_MAX || t.size(1) > INT32_MAX) refuse(what, "sizes must be below 2^31");
  return static_cast<int32_t>(t.size(0));
}

void scales_of(const char* what, const at::Tensor& k, PyObject* k_scale, PyObject* v_scale, float** ks, float** vs) {
  if (k.scalar_type() != at::kFloat8_e4m3fn || !given(k_scale) || !given(v_scale))
    refuse(what, "an e4m3 cache comes with k_scale and v_scale, another without");
  const int64_t dev = k.get_device();
  *ks = floats(tensor(k_scale, "k_scale"), what, "k_scale", dev, {k.size(0), k.size(1), k.size(2) / SLED_SCALE_BLOCK});
  *vs = floats(tensor(v_scale, "v_scale"), what, "v_scale", dev, {k.size(0), k.size(1), k.size(2) / SLED_SCALE_BLOCK});
}

// ---- the calls; arguments in a fixed order, None where there is none
// q, k, v, page_table, n_kv, cu_q, parents, scale, out, lse, key_weights, status, k_scale, v_scale
PyObject* attention_scaled(PyObject* const* a) {
  const char* what = "sled_attention_scaled";
  const at::Tensor &q = tensor(a[0], "q"), &k = tensor(a[1], "k"), &v = tensor(a[2], "v"), &cu_q = tensor(a[5], "cu_q");
  const sled_paged_kv kv = paged(what, k, v, tensor(a[3], "page_table"), tensor(a[4], "n_kv"));
  const int64_t dev = k.get_device();
  if (given(a[10])) refuse(what, "weights of keys are formed over caches of 16 and 32 bits");
  float *ks, *vs;
  scales_of(what, k, a[12], a[13], &ks, &vs);
  if (q.dim() != 3 || q.scalar_type() != at::kBFloat16 || q.get_device() != dev || q.size(2) != kv.head_dim)
    refuse(what, "q must be [rows, n_q_heads, head_dim] bf16 on the cache's device");
  if (cu_q.dim() != 1 || cu_q.numel() != static_cast<int64_t>(kv.n_reqs) + 1) refuse(what, "cu_q must be [n_reqs + 1]");
  const int32_t rows = rows_of(q, what), heads = static_cast<int32_t>(q.size(1));
  const int64_t q_stride = row_stride(q, what, "q");
  at::Tensor made;
  if (!given(a[8])) made = at::empty(q.sizes(), q.options());
  const at::Tensor& out = given(a[8]) ? tensor(a[8], "out") : made;
  if (out.sizes() != q.sizes() || out.scalar_type() != q.scalar_type() || out.get_device() != dev) refuse(what, "out must be like q");
  if (out.data_ptr() == q.data_ptr() && q.numel()) refuse(what, "out must not be q: queries are read until the call has run");
  const int64_t out_stride = row_stride(out, what, "out");
  int32_t* parents = nullptr;
  if (given(a[6])) {
    const at::Tensor& p = tensor(a[6], "parents");
    if (p.dim() != 1 || p.numel() != rows) refuse(what, "parents must have an entry for each row");
    parents = ints(p, what, "parents", dev);
  }
  float* lse = given(a[9]) ? floats(tensor(a[9], "lse"), what, "lse", dev, {rows, heads}) : nullptr;
  const double scale = PyFloat_AsDouble(a[7]);
  if (scale == -1.0 && PyErr_Occurred()) throw Refused{1, ""};
  int64_t bytes = 0;
  check(sled_attention_scaled_workspace(&kv, rows, heads, &bytes), what);
  const at::Tensor ws = at::empty({bytes}, q.options().dtype(at::kByte));
  const void* const queries = q.data_ptr();
  void *const results = out.data_ptr(), *const space = ws.data_ptr(), *const stream = stream_of(dev);
  int32_t *const offsets = ints(cu_q, what, "cu_q", dev), *const status = status_of(a[11], what, dev);
  check(unlocked([&] {
    return sled_attention_scaled(&kv, ks, vs, queries, q_stride, offsets, parents, rows, heads, static_cast<float>(scale), results, out_stride, lse, status, space,
                                 bytes, stream);
  }), what);
  if (!given(a[8])) return THPVariable_Wrap(made);
  Py_INCREF(a[8]);
  return a[8];
}

// k, v, k_cache, v_cache, page_table, n_kv, cu_q, k_scale, v_scale, status
PyObject* append_keys(PyObject* const* a) {
  const char* what = "sled_append_keys";
  const at::Tensor &k = tensor(a[0], "k"), &v = tensor(a[1], "v"), &k_cache = tensor(a[2], "k_cache"), &cu_q = tensor(a[6], "cu_q");
  const sled_paged_kv kv = paged(what, k_cache, tensor(a[3], "v_cache"), tensor(a[4], "page_table"), tensor(a[5], "n_kv"));
  const int64_t dev = k_cache.get_device();
  const int type = type_of(k, false);
  if (k.dim() != 3 || type < 0 || k.get_device() != dev || k.size(1) != kv.n_kv_heads || k.size(2) != kv.head_dim)
    refuse(what, "k must be [rows, n_kv_heads, head_dim], fp32 or bf16, " + on(dev));
  if (v.sizes() != k.sizes() || v.scalar_type() != k.scalar_type() || v.get_device() != dev) refuse(what, "v must be like k");
  if (kv.dtype != SLED_E4M3 && k.scalar_type() != k_cache.scalar_type()) refuse(what, "rows of another type go into a cache of 8 bits only");
  float *ks = nullptr, *vs = nullptr;
  if (kv.dtype == SLED_E4M3 || given(a[7]) || given(a[8])) scales_of(what, k_cache, a[7], a[8], &ks, &vs);
  if (cu_q.dim() != 1 || cu_q.numel() != static_cast<int64_t>(kv.n_reqs) + 1) refuse(what, "cu_q must be [n_reqs + 1]");
  const void *const keys = k.data_ptr(), *const values = v.data_ptr();
  const int64_t k_stride = row_stride(k, what, "k"), v_stride = row_stride(v, what, "v");
  const int32_t rows = rows_of(k, what);
  int32_t *const offsets = ints(cu_q, what, "cu_q", dev), *const status = status_of(a[9], what, dev);
  void* const stream = stream_of(dev);
  check(unlocked([&] { return sled_append_keys(&kv, ks, vs, keys, k_stride, values, v_stride, type, offsets, rows, status, stream); }), what);
  Py_RETURN_NONE;
}

sled_heads heads_of(const at::Tensor& t, const at::Tensor& out, const char* what, const char* name, const at::Tensor& q) {
  if (t.dim() != 3 || t.scalar_type() != q.scalar_type() || t.get_device() != q.get_device() || t.size(0) != q.size(0) || t.size(2) != q.size(2) ||
      (t.stride(2) != 1 && t.numel()))
    refuse(what, std::string(name) + " must be [rows, heads, head_dim] of q's type and device, heads contiguous");
  if (out.sizes() != t.sizes() || out.scalar_type() != t.scalar_type() || out.get_device() != t.get_device() || (out.stride(2) != 1 && out.numel()))
    refuse(what, std::string(name) + "_out must be like " + name);
  rows_of(t, what);
  return sled_heads{t.data_ptr(), t.stride(0), t.stride(1), out.data_ptr(), out.stride(0), out.stride(1), static_cast<int32_t>(t.size(1))};
}

// q, k, positions, frequencies, pairs, amplitude, transpose, q_out, k_out
PyObject* rotary(PyObject* const* a) {
  const char* what = "sled_rotary";
  const at::Tensor& q = tensor(a[0], "q");
  if (!q.is_cuda()) throw Refused{SLED_ERR_NO_DEVICE, std::string(what) + " (tensors must be on a CUDA device)"};
  const int64_t dev = q.get_device();
  const int type = type_of(q, false);
  const int32_t pairs = in_32_bits(a[4], what, "style");
  if (type < 0 || q.dim() != 3 || pairs < 0) refuse(what, "q must be [rows, heads, head_dim], fp32 or bf16; style pairs or halves");
  if (q.size(2) > INT32_MAX) refuse(what, "sizes must be below 2^31");
  at::Tensor q_made, k_made;
  if (!given(a[7])) q_made = at::empty(q.sizes(), q.options());
  const sled_heads qh = heads_of(q, given(a[7]) ? tensor(a[7], "q_out") : q_made, what, "q", q);
  sled_heads kh{};
  if (given(a[1])) {
    const at::Tensor& k = tensor(a[1], "k");
    if (!given(a[8])) k_made = at::empty(k.sizes(), k.options());
    kh = heads_of(k, given(a[8]) ? tensor(a[8], "k_out") : k_made, what, "k", q);
  }
  const double amplitude = PyFloat_AsDouble(a[5]);
  if (amplitude == -1.0 && PyErr_Occurred()) throw Refused{1, ""};
  const int transpose = PyObject_IsTrue(a[6]);
  if (transpose < 0) throw Refused{1, ""};
  const int64_t rows = q.size(0), half = tensor(a[3], "frequencies").numel();
  if (half > 256) refuse(what, "head_dim is at most 512");
  const int32_t head_dim = static_cast<int32_t>(q.size(2));
  const int32_t* const positions = vector_of<int32_t>(a[2], what, "positions", dev, rows, at::kInt);
  const double* const frequencies = vector_of<double>(a[3], what, "frequencies", dev, half, at::kDouble);
  const sled_heads* const keys = given(a[1]) ? &kh : nullptr;
  void* const stream = stream_of(dev);
  check(unlocked([&] {
    return sled_rotary(&qh, keys, static_cast<int32_t>(rows), head_dim, type, positions, frequencies, static_cast<int32_t>(2 * half), pairs,
                       static_cast<float>(amplitude), transpose, stream);
  }), what);
  PyObject* q_out = given(a[7]) ? Py_NewRef(a[7]) : THPVariable_Wrap(q_made);
  PyObject* k_out = !given(a[1]) ? Py_NewRef(Py_None) : given(a[8]) ? Py_NewRef(a[8]) : THPVariable_Wrap(k_made);
  PyObject* both = PyTuple_Pack(2, q_out, k_out);
  Py_DECREF(q_out);
  Py_DECREF(k_out);
  return both;
}

// n_kv, n_new, page_table, free_pages, n_free, page_size, n_rows, n_keep, out, status; returns the five tensors of out
PyObject* page_slots(PyObject* const* a) {
  const char* what = "sled_page_slots";
  const int32_t page_size = in_32_bits(a[5], what, "page_size"), n_rows = in_32_bits(a[6], what, "n_rows");
  const at::Tensor &n_kv = tensor(a[0], "n_kv"), &table = tensor(a[2], "page_table"), &free_pages = tensor(a[3], "free_pages");
  if (!n_kv.is_cuda()) throw Refused{SLED_ERR_NO_DEVICE, std::string(what) + " (tensors must be on a CUDA device)"};
  const int64_t dev = n_kv.get_device(), n = n_kv.numel();
  if (n_rows < 0 || table.dim() != 2 || table.size(0) != n || free_pages.dim() != 1)
    refuse(what, "page_table [n_reqs, cols], free_pages [cap], n_rows not negative");
  const int64_t cols = table.size(1), stride = n > 1 ? table.stride(0) : cols, cap = free_pages.numel();
  if (n > INT32_MAX || stride > INT32_MAX || cols > INT32_MAX || cap > INT32_MAX || stride < cols) refuse(what, "rows of page_table must not overlap, sizes be below 2^31");
  PyObject* out[5];
  at::Tensor made[5];
  if (!given(a[8])) {
    const auto i32 = n_kv.options().dtype(at::kInt);
    const at::Tensor all = at::empty({2 * n + n_rows + 2}, i32);
    made[0] = all.narrow(0, 0, n);
    made[1] = all.narrow(0, n, n + 1);
    made[2] = all.narrow(0, 2 * n + 1, n_rows);
    made[3] = at::empty({n_rows}, i32.dtype(at::kLong));
    made[4] = all.narrow(0, 2 * n + 1 + n_rows, 1);
  } else if (!PyTuple_Check(a[8]) || PyTuple_GET_SIZE(a[8]) != 5) {
    refuse(what, "out must be five tensors, as the call returns them");
  }
  for (int i = 0; i < 5; ++i) out[i] = given(a[8]) ? Py_NewRef(PyTuple_GET_ITEM(a[8], i)) : THPVariable_Wrap(made[i]);
  struct Hold {
    PyObject** p;
    ~Hold() { for (int i = 0; i < 5; ++i) Py_DECREF(p[i]); }
  } hold{out};
  const int32_t n_reqs = static_cast<int32_t>(n);
  const int32_t* const have = vector_of<int32_t>(a[0], what, "n_kv", dev, n, at::kInt);
  const int32_t* const keep = given(a[7]) ? vector_of<int32_t>(a[7], what, "n_keep", dev, n, at::kInt) : nullptr;
  const int32_t* const fresh = vector_of<int32_t>(a[1], what, "n_new", dev, n, at::kInt);
  int32_t *const pages = ints(table, what, "page_table", dev), *const stack = vector_of<int32_t>(a[3], what, "free_pages", dev, cap, at::kInt);
  const int32_t* const n_free = vector_of<int32_t>(a[4], what, "n_free", dev, 1, at::kInt);
  int32_t *const n_kv_out = vector_of<int32_t>(out[0], what, "out.n_kv", dev, n, at::kInt), *const n_free_out = vector_of<int32_t>(out[4], what, "out.n_free", dev, 1, at::kInt);
  int32_t* const cu_q = vector_of<int32_t>(out[1], what, "out.cu_q", dev, n + 1, at::kInt);
  int32_t* const positions = vector_of<int32_t>(out[2], what, "out.positions", dev, n_rows, at::kInt);
  int64_t* const slots = vector_of<int64_t>(out[3], what, "out.slots", dev, n_rows, at::kLong);
  int32_t* const status = status_of(a[9], what, dev);
  void* const stream = stream_of(dev);
  check(unlocked([&] {
    return sled_page_slots(have, keep, fresh, n_reqs, page_size, pages, static_cast<int32_t>(stride), static_cast<int32_t>(cols), stack, static_cast<int32_t>(cap),
                           n_free, n_kv_out, n_free_out, cu_q, positions, slots, n_rows, status, stream);
  }), what);
  return PyTuple_Pack(5, out[0], out[1], out[2], out[3], out[4]);
}

template <PyObject* (*kCall)(PyObject* const*), int kArgs>
PyObject* guarded(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != kArgs) {
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
    return nullptr;
  }
  try {
    return kCall(args);
  } catch (const Refused& r) {
    if (r.code <= 0) {
      PyObject* e = PyObject_CallFunction(g_error, "is", r.code, r.what.c_str());
      if (e) {
        PyErr_SetObject(g_error, e);
        Py_DECREF(e);
      }
    }                        // otherwise Python has an error of its own
  } catch (const NotATensor& t) {
    PyErr_Format(PyExc_TypeError, "%s must be a tensor", t.name.c_str());
  } catch (...) {            // torch's own: no memory left, among others
    torch::translate_exception_to_python(std::current_exception());
  }
  return nullptr;
}

PyObject* set_error(PyObject*, PyObject* type) {
  Py_XDECREF(g_error);
  g_error = Py_NewRef(type);
  Py_RETURN_NONE;
}

template <PyObject* (*kCall)(PyObject* const*), int kArgs>
PyMethodDef method(const char* name) {
  return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(guarded<kCall, kArgs>)), METH_FASTCALL, nullptr};
}
PyMethodDef g_methods[] = {method<attention_scaled, 14>("attention_scaled"),
                           method<append_keys, 10>("append_keys"),
                           method<rotary, 9>("rotary"),
                           method<page_slots, 10>("page_slots"),
                           {"set_error", set_error, METH_O, nullptr},
                           {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() {
  PyObject* m = PyModule_Create(&g_module);
  if (m && PyModule_AddStringConstant(m, "built_for", SLED_BUILT_FOR)) {      // the torch and Python that it is tied to
    Py_DECREF(m);
    return nullptr;
  }
  return m;
}
