// Native half of the ctypes binding: the calls of the decode/evict path from Python with torch tensors.
//
// A decode step of a few units is 5 us of GPU time; through ctypes the call itself took as long: 1.2 us for
// nine is_contiguous() / data_ptr() pairs, 0.5 us of argument conversion, 0.4 us for the stream handle, 0.4 us
// of Python around them, and 2.6 us in the library (the launch).  Here the first four take 0.3 us.
//
// Each function is the C entry point of the same name without its last argument, the stream, which is the
// current device's current one.  Arguments that are not exactly what the path passes (a torch.Tensor, contiguous, or
// None; an int of 32 bits; a float) are not converted here: the function returns None without having called
// anything, and the caller goes through ctypes, which converts or refuses them as it always has.
#include <torch/csrc/autograd/python_variable.h>

#include <c10/hip/HIPStream.h>

#include <cstring>
#include <initializer_list>
#include <tuple>
#include <utility>

#include "gkv.h"

namespace {

struct NotForUs {};

void* pointer(PyObject* o) {
  if (o == Py_None) return nullptr;
  if (!THPVariable_CheckExact(o)) throw NotForUs();
  const at::Tensor& t = THPVariable_Unpack(o);
  if (t.layout() != at::kStrided || !t.is_cuda() || !t.is_contiguous() || !t.has_storage()) throw NotForUs();
  return t.data_ptr();
}
void convert(PyObject* o, void*& out) { out = pointer(o); }
void convert(PyObject* o, const void*& out) { out = pointer(o); }
void convert(PyObject* o, int32_t*& out) { out = (int32_t*)pointer(o); }
void convert(PyObject* o, const int32_t*& out) { out = (const int32_t*)pointer(o); }
void convert(PyObject* o, float*& out) { out = (float*)pointer(o); }
void convert(PyObject* o, const float*& out) { out = (const float*)pointer(o); }
void convert(PyObject* o, gkv_ctx*& out) {
  if (!PyLong_CheckExact(o)) throw NotForUs();
  out = (gkv_ctx*)PyLong_AsVoidPtr(o);
  if (!out) { PyErr_Clear(); throw NotForUs(); }
}
void convert(PyObject* o, int32_t& out) {
  if (!PyLong_CheckExact(o)) throw NotForUs();
  int overflow = 0;
  const long v = PyLong_AsLongAndOverflow(o, &overflow);
  if (overflow || v < INT32_MIN || v > INT32_MAX) throw NotForUs();
  out = (int32_t)v;
}
void convert(PyObject* o, float& out) {
  if (!PyFloat_CheckExact(o)) throw NotForUs();
  out = (float)PyFloat_AS_DOUBLE(o);
}

// One type per entry point, with the signature that the header declares and the address that bind() was given
// (the library is loaded through ctypes).
#define GKV_CALLS(X)                                                                                 \
  X(gkv_attend_decode) X(gkv_score_window) X(gkv_global_update) X(gkv_select_topk) X(gkv_compact)    \
  X(gkv_evict) X(gkv_redundancy_combine) X(gkv_evicted_positions)                                   \
  X(gkv_q8_attend_decode) X(gkv_q8_score_window) X(gkv_q8_compact) X(gkv_q8_evict)                   \
  X(gkv_prefix_attend) X(gkv_attend_decode_prefix)
#define GKV_TYPE(name) struct call_##name { static inline decltype(&::name) address = nullptr; };
GKV_CALLS(GKV_TYPE)


template <typename Call, typename... A, size_t... I>
PyObject* call(gkv_status (*f)(A...), PyObject* const* args, Py_ssize_t n, std::index_sequence<I...>) {
  try {
    if (!f || n != (Py_ssize_t)sizeof...(I)) throw NotForUs();
    std::tuple<A...> v;
    (convert(args[I], std::get<I>(v)), ...);
    std::get<sizeof...(I)>(v) = (void*)c10::hip::getCurrentHIPStream().stream();
    gkv_status st;
    Py_BEGIN_ALLOW_THREADS
    st = std::apply(f, v);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(st);
  } catch (const NotForUs&) {
    Py_RETURN_NONE;
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}
template <typename... A> constexpr size_t arguments(gkv_status (*)(A...)) { return sizeof...(A); }

template <typename Call>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
  constexpr size_t N = arguments(decltype(Call::address){nullptr}) - 1;   // without the stream
  return call<Call>(Call::address, args, n, std::make_index_sequence<N>());
}

// ---- rotary positions and paged caches --------------------------------------------------------------
// Their sizes come from the tensors, so shapes, types and devices are looked at here: what is not as the header wants it is left to the Python
// half, which says what is wrong.  `spec` is the address of the context's configuration.
#define GKV_CHECKED_CALLS(X) X(gkv_rotate) X(gkv_paged_append) X(gkv_paged_attend_decode) X(gkv_paged_advance)
GKV_CHECKED_CALLS(GKV_TYPE)

struct Arguments {
  PyObject* const* args;
  Py_ssize_t n, at = 0;
  const gkv_config* cfg = nullptr;
  c10::DeviceIndex here = -1;                                // the current device, once there is a tensor of one
  PyObject* next() {
    if (at >= n) throw NotForUs();
    return args[at++];
  }
  template <typename T> T value() { T x; convert(next(), x); return x; }
  gkv_ctx* context() {
    gkv_ctx* ctx = value<gkv_ctx*>();
    PyObject* o = next();
    if (!PyLong_CheckExact(o)) throw NotForUs();
    cfg = (const gkv_config*)PyLong_AsVoidPtr(o);
    if (!cfg) { PyErr_Clear(); throw NotForUs(); }
    return ctx;
  }
  // The next one as a tensor of this device; null if it is None, which `may` allow.
  const at::Tensor* tensor(at::ScalarType type, bool may = false) {
    PyObject* o = next();
    if (may && o == Py_None) return nullptr;
    if (!THPVariable_CheckExact(o)) throw NotForUs();
    const at::Tensor& t = THPVariable_Unpack(o);
    if (t.layout() != at::kStrided || !t.is_cuda() || !t.has_storage() || t.scalar_type() != type) throw NotForUs();
    if (here < 0) here = c10::hip::current_device();
    if (t.get_device() != here) throw NotForUs();
    return &t;
  }
  at::ScalarType type() const { return cfg->dtype == GKV_F32 ? at::kFloat : at::kBFloat16; }
  void* shaped(at::ScalarType type, std::initializer_list<int64_t> shape, bool may = false) {
    const at::Tensor* t = tensor(type, may);
    if (!t) return nullptr;
    if (!t->is_contiguous() || t->sizes() != at::IntArrayRef(shape)) throw NotForUs();
    return t->data_ptr();
  }
  // Rows [n_layers, tokens, heads, d] that may lie apart; tokens < 0: as many as the tensor has.
  void* heads(int32_t n_heads, int64_t& tokens, int32_t& stride) {
    stride = 0;
    const at::Tensor* t = tensor(type(), true);
    if (!t) return nullptr;
    if (t->dim() != 4) throw NotForUs();
    if (tokens < 0) tokens = t->size(1);
    const int64_t L = cfg->n_layers, d = cfg->head_dim, own = n_heads * d;
    if (t->size(0) != L || t->size(1) != tokens || t->size(2) != n_heads || t->size(3) != d || tokens < 1 || tokens > INT32_MAX) throw NotForUs();
    if (!t->is_contiguous()) {
      const int64_t s = tokens > 1 ? t->stride(1) : t->stride(0);
      if ((d > 1 && t->stride(3) != 1) || (n_heads > 1 && t->stride(2) != d) || (L > 1 && t->stride(0) != s * tokens) || s < own || s > INT32_MAX)
        throw NotForUs();
      stride = (int32_t)s;
    }
    return t->data_ptr();
  }
  struct Rotary { const double* freq; int32_t dim, layout; float amplitude; };
  Rotary rotary() {                                          // freq, dim, layout, amplitude
    const at::Tensor* f = tensor(at::kDouble, true);
    Rotary r{f ? (const double*)f->data_ptr() : nullptr, value<int32_t>(), value<int32_t>(), value<float>()};
    if (f && (!f->is_contiguous() || r.dim < 0 || f->numel() < r.dim / 2)) throw NotForUs();
    return r;
  }
  struct Pages { const int32_t* table; int32_t width, rows, n; void *K, *V; const int32_t* len; };
  Pages pages() {                                            // d_len, page_table, K, V
    Pages p;
    p.len = (const int32_t*)shaped(at::kInt, {cfg->batch});
    const at::Tensor* table = tensor(at::kInt);
    if (table->dim() != 2 || table->size(0) != cfg->batch || !table->is_contiguous() || table->size(1) > INT32_MAX) throw NotForUs();
    const at::Tensor* K = tensor(type());
    if (K->dim() != 5 || !K->is_contiguous() || K->size(0) != cfg->n_layers || K->size(2) != cfg->n_kv_heads || K->size(4) != cfg->head_dim ||
        K->size(1) > INT32_MAX || K->size(3) > INT32_MAX) throw NotForUs();
    const at::Tensor* V = tensor(type());
    if (!V->is_contiguous() || V->sizes() != K->sizes()) throw NotForUs();
    p.table = (const int32_t*)table->data_ptr(); p.width = (int32_t)table->size(1);
    p.n = (int32_t)K->size(1); p.rows = (int32_t)K->size(3); p.K = K->data_ptr(); p.V = V->data_ptr();
    return p;
  }
};

template <typename F, typename... A>
gkv_status without_gil(F f, A... a) {
  if (!f) throw NotForUs();
  void* stream = (void*)c10::hip::getCurrentHIPStream().stream();
  gkv_status st;
  Py_BEGIN_ALLOW_THREADS
  st = f(a..., stream);
  Py_END_ALLOW_THREADS
  return st;
}

// ctx, spec, q, k, positions, step, freq, dim, layout, amplitude, transposed, q_out, k_out
gkv_status rotate(Arguments& x) {
  gkv_ctx* ctx = x.context();
  int64_t tokens = -1;
  int32_t qs, ks;
  void* q = x.heads(x.cfg->n_q_heads, tokens, qs);
  void* k = x.heads(x.cfg->n_kv_heads, tokens, ks);
  if (tokens < 0) throw NotForUs();
  auto* positions = (const int32_t*)x.shaped(at::kInt, {tokens}, true);
  const int32_t step = x.value<int32_t>();
  const auto r = x.rotary();
  const int32_t transposed = x.value<int32_t>();
  void* q_out = x.shaped(x.type(), {x.cfg->n_layers, tokens, x.cfg->n_q_heads, x.cfg->head_dim}, true);
  void* k_out = x.shaped(x.type(), {x.cfg->n_layers, tokens, x.cfg->n_kv_heads, x.cfg->head_dim}, true);
  return without_gil(call_gkv_rotate::address, ctx, q, qs, k, ks, (int32_t)tokens, positions, step, r.freq, r.dim, r.layout, r.amplitude, transposed,
                     q_out, k_out);
}

// ctx, spec, q, k, v, d_start, positions, freq, dim, layout, amplitude, d_len, page_table, K, V, q_out
gkv_status paged_append(Arguments& x) {
  gkv_ctx* ctx = x.context();
  int64_t tokens = -1;
  int32_t qs, ks, vs;
  void* q = x.heads(x.cfg->n_q_heads, tokens, qs);
  void* k = x.heads(x.cfg->n_kv_heads, tokens, ks);
  void* v = x.heads(x.cfg->n_kv_heads, tokens, vs);
  if (tokens < 0) throw NotForUs();
  auto* start = (const int32_t*)x.shaped(at::kInt, {x.cfg->batch + 1}, true);
  auto* positions = (const int32_t*)x.shaped(at::kInt, {tokens}, true);
  const auto r = x.rotary();
  const auto p = x.pages();
  void* q_out = x.shaped(x.type(), {x.cfg->n_layers, tokens, x.cfg->n_q_heads, x.cfg->head_dim}, true);
  return without_gil(call_gkv_paged_append::address, ctx, q, qs, k, ks, v, vs, (int32_t)tokens, start, p.len, positions, r.freq, r.dim, r.layout,
                     r.amplitude, p.table, p.width, p.rows, p.n, p.K, p.V, q_out);
}

// ctx, spec, q, d_len, page_table, K, V, len_max_host, out, workspace, bytes the workspace has at least
gkv_status paged_attend_decode(Arguments& x) {
  gkv_ctx* ctx = x.context();
  const auto shape = {(int64_t)x.cfg->n_layers, (int64_t)x.cfg->batch, (int64_t)x.cfg->n_q_heads, (int64_t)x.cfg->head_dim};
  void* q = x.shaped(x.type(), shape);
  const auto p = x.pages();
  const int32_t len_max = x.value<int32_t>();
  void* out = x.shaped(x.type(), shape);
  const at::Tensor* workspace = x.tensor(at::kByte);
  PyObject* bytes = x.next();
  if (!PyLong_CheckExact(bytes) || !workspace->is_contiguous() || workspace->numel() < PyLong_AsLongLong(bytes)) throw NotForUs();
  return without_gil(call_gkv_paged_attend_decode::address, ctx, q, p.K, p.V, p.table, p.width, p.rows, p.n, p.len, len_max, out, workspace->data_ptr());
}

// ctx, spec, d_len, d_start
gkv_status paged_advance(Arguments& x) {
  gkv_ctx* ctx = x.context();
  auto* len = (int32_t*)x.shaped(at::kInt, {x.cfg->batch});
  auto* start = (const int32_t*)x.shaped(at::kInt, {x.cfg->batch + 1}, true);
  return without_gil(call_gkv_paged_advance::address, ctx, len, start);
}

template <gkv_status (*f)(Arguments&)>
PyObject* checked(PyObject*, PyObject* const* args, Py_ssize_t n) {
  try {
    Arguments x{args, n};
    return PyLong_FromLong(f(x));
  } catch (const NotForUs&) {
    Py_RETURN_NONE;
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

PyObject* bind(PyObject*, PyObject* args) {
  const char* name;
  PyObject* address;
  if (!PyArg_ParseTuple(args, "sO!", &name, &PyLong_Type, &address)) return nullptr;
  void* p = PyLong_AsVoidPtr(address);
  if (PyErr_Occurred()) return nullptr;
#define GKV_BIND(call) if (!strcmp(name, #call)) { call_##call::address = (decltype(&::call))p; Py_RETURN_NONE; }
  GKV_CALLS(GKV_BIND)
  GKV_CHECKED_CALLS(GKV_BIND)
  PyErr_SetString(PyExc_KeyError, name);
  return nullptr;
}

#define GKV_METHOD(name) {#name, (PyCFunction)(void (*)(void))entry<call_##name>, METH_FASTCALL, nullptr},
#define GKV_CHECKED(name) {#name, (PyCFunction)(void (*)(void))checked<name>, METH_FASTCALL, nullptr},
PyMethodDef methods[] = {GKV_CALLS(GKV_METHOD) GKV_CHECKED(rotate) GKV_CHECKED(paged_append) GKV_CHECKED(paged_attend_decode)
                         GKV_CHECKED(paged_advance) {"bind", bind, METH_VARARGS, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_gkv_call", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__gkv_call() { return PyModule_Create(&module); }
