// The calls of the Python binding for the arguments that they are made with in earnest: checks, extents and pointers in
// native code, then the entry point.  Host time is what bounds a small call: a lookup of two tables spent 7.9 us in Python
// attribute accesses around a kernel of 3.9.
//
// Every function returns the entry point's status, or -1 for whatever it does not know to be right -- a wrong type, dtype,
// shape or layout, a tensor subclass or wrapper, more than 8 layers or tables --, without having called anything: the binding
// then takes its general path, which decides and raises.  Nothing is kept between calls.
#include <torch/csrc/autograd/python_variable.h>

#include <c10/hip/HIPStream.h>

#include <cstdint>

namespace {

typedef int (*tbmm_t)(const float*, const float*, float*, int64_t, int64_t, int64_t, int64_t, void*);
typedef int (*tbmm_ws_t)(const float*, const float*, float*, int64_t, int64_t, int64_t, int64_t, void*, size_t, void*);
typedef int (*mlp_t)(const float*, int64_t, int32_t, const int64_t*, const float* const*, const float* const*, float* const*, void*, size_t, void*);
typedef int (*gconv_t)(const float*, const float*, const float*, float*, int64_t, int64_t, int64_t, int64_t, int64_t, int64_t, int64_t, int64_t, void*);
typedef int (*kron_t)(const float*, const float*, const float*, float*, int64_t, int64_t, int64_t, int64_t, int64_t, void*);
typedef int (*sconv_t)(const float*, const float*, const float*, float*, int64_t, int64_t, int64_t, int64_t, int64_t, int64_t, int64_t, int64_t, int64_t,
                       void*);
typedef int (*embed_t)(const void*, const int32_t*, void*, int64_t, int64_t, int64_t, float, int, void*);
typedef int (*embed_grad_t)(const void*, const int32_t*, void*, int64_t, int64_t, int64_t, float, int64_t, int32_t, int, int, void*, size_t, void*);
typedef int (*route_t)(const void*, float*, int32_t*, int32_t*, int32_t*, int32_t*, int64_t, int64_t, int64_t, int32_t, int, void*, size_t, void*);
typedef int (*route_grad_t)(const void*, const int32_t*, const float*, void*, int64_t, int64_t, int64_t, int32_t, int, void*);
typedef int (*expert_mm_t)(const void*, const void*, const int32_t*, const int32_t*, void*, int64_t, int64_t, int64_t, int64_t, int64_t, int32_t, int, void*);
typedef int (*expert_mm_grad_x_t)(const void*, const void*, const int32_t*, const void*, void*, int64_t, int64_t, int64_t, int64_t, int, void*);
typedef int (*expert_mm_grad_w_t)(const void*, const void*, const int32_t*, const int32_t*, void*, int64_t, int64_t, int64_t, int64_t, int64_t, int32_t, int, int,
                                  void*, size_t, void*);
typedef int (*expert_sum_t)(const void*, const float*, const int32_t*, void*, int64_t, int64_t, int64_t, int64_t, int, void*);
typedef int (*expert_sum_grad_t)(const void*, const void*, const float*, const int32_t*, void*, float*, int64_t, int64_t, int64_t, int64_t, int, void*);
typedef int (*lut_t)(int32_t, const float* const*, const int32_t* const*, float* const*, const int64_t*, const int64_t*, int64_t, int64_t, void*);

constexpr int kMost = 8;  // layers, tables

// A dense contiguous GPU tensor of `dims` dimensions, exactly torch's own (or a Parameter), behind no wrapper.
struct Arg {
  const int64_t* size = nullptr;
  void* data = nullptr;
};

bool take(PyObject* o, c10::ScalarType type, int64_t dims, Arg* a) {
  if (!THPVariable_CheckExact(o)) return false;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.defined() || !t.is_cuda() || t.scalar_type() != type || t.layout() != c10::kStrided) return false;
  const c10::TensorImpl* impl = t.unsafeGetTensorImpl();
  if (impl->has_symbolic_sizes_strides() || !impl->has_storage()) return false;
  using K = c10::DispatchKey;
  if (impl->key_set().has_any(c10::DispatchKeySet({K::FuncTorchBatched, K::FuncTorchGradWrapper, K::Functionalize, K::Python, K::Batched})))
    return false;
  if (t.dim() != dims || !t.is_contiguous()) return false;
  a->size = t.sizes().data();
  a->data = t.data_ptr();
  return true;
}
bool take(PyObject* o, int64_t dims, Arg* a) { return take(o, c10::kFloat, dims, a); }

bool stream_of(PyObject* o, void** s) {
  if (o == Py_None) {
    *s = c10::hip::getCurrentHIPStream().stream();
    return true;
  }
  if (!PyLong_CheckExact(o)) return false;
  *s = PyLong_AsVoidPtr(o);
  if (!*s && PyErr_Occurred()) {
    PyErr_Clear();
    return false;
  }
  return true;
}

// Items of a list or tuple of n objects.
PyObject** items(PyObject* o, Py_ssize_t n) {
  if (!PyList_CheckExact(o) && !PyTuple_CheckExact(o)) return nullptr;
  return PySequence_Fast_GET_SIZE(o) == n ? PySequence_Fast_ITEMS(o) : nullptr;
}

// An entry point from its address.
template <typename T>
bool entry_of(PyObject* o, T* entry) {
  if (!PyLong_CheckExact(o)) return false;
  *entry = reinterpret_cast<T>(PyLong_AsVoidPtr(o));
  return *entry || !PyErr_Occurred();
}

// Runs `body`, which returns a status or -1; what throws (a tensor without memory, for one) is left to the general path.
template <typename F>
PyObject* guarded(F body) {
  int st = -1;
  try {
    st = body();
  } catch (...) {
    st = -1;
  }
  if (PyErr_Occurred()) PyErr_Clear();
  return PyLong_FromLong(st);
}

// The call itself, without the interpreter's lock; its arguments are evaluated with it.
struct Unlocked {
  PyThreadState* const state = PyEval_SaveThread();
  ~Unlocked() { PyEval_RestoreThread(state); }
};
template <typename... P, typename... A>
int call(int (*entry)(P...), A... args) {
  Unlocked u;
  return entry(args...);
}

inline const float* f(const Arg& a) { return static_cast<const float*>(a.data); }
inline float* out(const Arg& a) { return static_cast<float*>(a.data); }

// (entry, X, Y, Z, stream)
PyObject* call_tbmm(PyObject*, PyObject* const* v, Py_ssize_t n) {
  return guarded([&]() -> int {
    Arg X, Y, Z;
    void* s;
    if (n != 5 || !take(v[1], 3, &X) || !take(v[2], 3, &Y) || !take(v[3], 3, &Z) || !stream_of(v[4], &s)) return -1;
    const int64_t B = X.size[0], N = X.size[1], K = X.size[2], M = Y.size[1];
    if (Y.size[0] != B || Y.size[2] != K || Z.size[0] != B || Z.size[1] != N || Z.size[2] != M) return -1;
    tbmm_t entry;
    if (!entry_of(v[0], &entry)) return -1;
    return call(entry, f(X), f(Y), out(Z), B, N, M, K, s);
  });
}

// (entry, X, Y, Z, workspace, stream)
PyObject* call_tbmm_ws(PyObject*, PyObject* const* v, Py_ssize_t n) {
  return guarded([&]() -> int {
    Arg X, Y, Z, W;
    void* s;
    if (n != 6 || !take(v[1], 3, &X) || !take(v[2], 3, &Y) || !take(v[3], 3, &Z) || !take(v[4], c10::kByte, 1, &W) || !stream_of(v[5], &s)) return -1;
    const int64_t B = X.size[0], N = X.size[1], K = X.size[2], M = Y.size[1];
    if (Y.size[0] != B || Y.size[2] != K || Z.size[0] != B || Z.size[1] != N || Z.size[2] != M) return -1;
    tbmm_ws_t entry;
    if (!entry_of(v[0], &entry)) return -1;
    return call(entry, f(X), f(Y), out(Z), B, N, M, K, W.data, (size_t)W.size[0], s);
  });
}

// (entry, I, W, bias, O, workspace or None, stream)
PyObject* call_mlp(PyObject*, PyObject* const* v, Py_ssize_t n) {
  return guarded([&]() -> int {
    Arg I, ws;
    void* s;
    if (n != 7 || !take(v[1], 2, &I) || !(PyList_CheckExact(v[2]) || PyTuple_CheckExact(v[2]))) return -1;
    const Py_ssize_t layers = PySequence_Fast_GET_SIZE(v[2]);
    if (layers < 1 || layers > kMost) return -1;
    PyObject **W = items(v[2], layers), **b = items(v[3], layers), **O = items(v[4], layers);
    if (!W || !b || !O) return -1;
    const int64_t batch = I.size[0];
    int64_t dims[kMost + 1] = {I.size[1]};
    const float *Wp[kMost], *bp[kMost];
    float* Op[kMost];
    for (Py_ssize_t l = 0; l < layers; l++) {
      Arg w, c, o;
      if (!take(W[l], 2, &w) || !take(b[l], 1, &c) || w.size[1] != dims[l] || c.size[0] != w.size[0]) return -1;
      dims[l + 1] = w.size[0];
      if (O[l] != Py_None && (!take(O[l], 2, &o) || o.size[0] != batch || o.size[1] != dims[l + 1])) return -1;
      Wp[l] = f(w);
      bp[l] = f(c);
      Op[l] = out(o);
    }
    if ((v[5] != Py_None && !take(v[5], c10::kByte, 1, &ws)) || !stream_of(v[6], &s)) return -1;
    const size_t bytes = ws.size ? (size_t)ws.size[0] : 0;
    mlp_t entry;
    if (!entry_of(v[0], &entry)) return -1;
    return call(entry, f(I), batch, (int32_t)layers, dims, Wp, bp, Op, ws.data, bytes, s);
  });
}

// (entry, I, W1, bias or None, O, stream)
PyObject* call_gconv(PyObject*, PyObject* const* v, Py_ssize_t n) {
  return guarded([&]() -> int {
    Arg I, W, b, O;
    void* s;
    if (n != 6 || !take(v[1], 5, &I) || !take(v[2], 5, &W) || (v[3] != Py_None && !take(v[3], 1, &b)) || !take(v[4], 5, &O) || !stream_of(v[5], &s))
      return -1;
    const int64_t N = I.size[0], G = I.size[1], C = I.size[2], H = I.size[3], Wd = I.size[4], F = W.size[1], KH = W.size[3], KW = W.size[4];
    if (W.size[0] != G || W.size[2] != C || (b.size && b.size[0] != G * F)) return -1;
    if (O.size[0] != N || O.size[1] != G || O.size[2] != F || O.size[3] != H - KH + 1 || O.size[4] != Wd - KW + 1) return -1;
    gconv_t entry;
    if (!entry_of(v[0], &entry)) return -1;
    return call(entry, f(I), f(W), f(b), out(O), N, G, C, F, H, Wd, KH, KW, s);
  });
}

// (entry, W1, W2, X, Y, stream)
PyObject* call_kron(PyObject*, PyObject* const* v, Py_ssize_t n) {
  return guarded([&]() -> int {
    Arg W1, W2, X, Y;
    void* s;
    if (n != 6 || !take(v[1], 2, &W1) || !take(v[2], 2, &W2) || !take(v[3], 3, &X) || !take(v[4], 3, &Y) || !stream_of(v[5], &s)) return -1;
    const int64_t I = W1.size[0], K = W1.size[1], J = W2.size[0], L = W2.size[1], B = X.size[0];
    if (X.size[1] != K || X.size[2] != L || Y.size[0] != B || Y.size[1] != I || Y.size[2] != J) return -1;
    kron_t entry;
    if (!entry_of(v[0], &entry)) return -1;
    return call(entry, f(W1), f(W2), f(X), out(Y), B, I, K, J, L, s);
  });
}

// (entry, I, Wt, bias or None, O, sh, sw, stream)
PyObject* call_sconv(PyObject*, PyObject* const* v, Py_ssize_t n) {
  return guarded([&]() -> int {
    Arg I, W, b, O;
    void* s;
    if (n != 8 || !take(v[1], 4, &I) || !take(v[2], 4, &W) || (v[3] != Py_None && !take(v[3], 1, &b)) || !take(v[4], 4, &O) || !stream_of(v[7], &s))
      return -1;
    if (!PyLong_CheckExact(v[5]) || !PyLong_CheckExact(v[6])) return -1;
    const int64_t sh = PyLong_AsLongLong(v[5]), sw = PyLong_AsLongLong(v[6]);
    const int64_t N = I.size[0], C = I.size[1], H = I.size[2], Wd = I.size[3], F = W.size[0], KH = W.size[2], KW = W.size[3];
    if (W.size[1] != C || (b.size && b.size[0] != F) || sh < 1 || sw < 1 || KH < 1 || KH > H || KW < 1 || KW > Wd) return -1;
    if (O.size[0] != N || O.size[1] != F || O.size[2] != (H - KH) / sh + 1 || O.size[3] != (Wd - KW) / sw + 1) return -1;
    sconv_t entry;
    if (!entry_of(v[0], &entry)) return -1;
    return call(entry, f(I), f(W), f(b), out(O), N, C, F, H, Wd, KH, KW, sh, sw, s);
  });
}

// (entry, LUT, Idx, O, stream)
PyObject* call_lut(PyObject*, PyObject* const* v, Py_ssize_t n) {
  return guarded([&]() -> int {
    void* s;
    if (n != 5 || !(PyList_CheckExact(v[1]) || PyTuple_CheckExact(v[1]))) return -1;
    const Py_ssize_t tables = PySequence_Fast_GET_SIZE(v[1]);
    if (tables < 1 || tables > kMost) return -1;
    PyObject **T = items(v[1], tables), **X = items(v[2], tables), **O = items(v[3], tables);
    if (!T || !X || !O) return -1;
    const float* Tp[kMost];
    const int32_t* Xp[kMost];
    float* Op[kMost];
    int64_t E[kMost], L[kMost], B = 0, D = 0;
    for (Py_ssize_t t = 0; t < tables; t++) {
      Arg a, x, o;
      if (!take(T[t], 2, &a) || !take(X[t], c10::kInt, 2, &x) || !take(O[t], 2, &o)) return -1;
      if (t == 0) {
        B = o.size[0];
        D = o.size[1];
      }
      if (o.size[0] != B || o.size[1] != D || a.size[1] != D || x.size[0] != B) return -1;
      Tp[t] = f(a);
      Xp[t] = static_cast<const int32_t*>(x.data);
      Op[t] = out(o);
      E[t] = a.size[0];
      L[t] = x.size[1];
    }
    if (!stream_of(v[4], &s)) return -1;
    lut_t entry;
    if (!entry_of(v[0], &entry)) return -1;
    return call(entry, (int32_t)tables, Tp, Xp, Op, E, L, D, B, s);
  });
}

// ---- operators around experts: tensors of one of three storage types (tc_type in include/tc355.h) ----

struct Kind {
  c10::ScalarType type = c10::kFloat;
  int code = -1;
};
bool kind_of(PyObject* o, Kind* k) {
  if (!THPVariable_CheckExact(o)) return false;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.defined()) return false;
  k->type = t.scalar_type();
  k->code = k->type == c10::kFloat ? 0 : k->type == c10::kBFloat16 ? 1 : k->type == c10::kHalf ? 2 : -1;
  return k->code >= 0;
}
bool take(PyObject* o, const Kind& k, int64_t dims, Arg* a) { return take(o, k.type, dims, a); }
bool take_ints(PyObject* o, int64_t dims, Arg* a) { return take(o, c10::kInt, dims, a); }
bool take_or_none(PyObject* o, const Kind& k, int64_t dims, Arg* a) { return o == Py_None || take(o, k.type, dims, a); }
bool take_ints_or_none(PyObject* o, int64_t dims, Arg* a) { return o == Py_None || take(o, c10::kInt, dims, a); }
bool is(const Arg& a, int64_t rows, int64_t cols) { return a.size[0] == rows && a.size[1] == cols; }

bool number(PyObject* o, float* x) {
  if (PyFloat_CheckExact(o)) *x = (float)PyFloat_AS_DOUBLE(o);
  else if (PyLong_CheckExact(o)) *x = (float)PyLong_AsDouble(o);
  else return false;
  return !PyErr_Occurred();
}
bool whole_number(PyObject* o, int64_t* x) {
  if (!PyLong_CheckExact(o)) return false;
  *x = PyLong_AsLongLong(o);
  return !PyErr_Occurred();
}
bool truth(PyObject* o, int32_t* x) {
  *x = o == Py_True;
  return o == Py_True || o == Py_False;
}
bool workspace_of(PyObject* o, void** p, size_t* n) {
  Arg a;
  *p = nullptr;
  *n = 0;
  if (o == Py_None) return true;
  if (!take(o, c10::kByte, 1, &a)) return false;
  *p = a.data;
  *n = (size_t)a.size[0];
  return true;
}
inline const int32_t* ints(const Arg& a) { return static_cast<const int32_t*>(a.data); }

// (entry, LUT, Idx, O, scale, stream)
PyObject* call_embed(PyObject*, PyObject* const* v, Py_ssize_t n) {
  return guarded([&]() -> int {
    Kind k;
    Arg L, I, O;
    void* s;
    float scale;
    if (n != 6 || !kind_of(v[1], &k) || !take(v[1], k, 2, &L) || !take_ints(v[2], 1, &I) || !take(v[3], k, 2, &O) || !number(v[4], &scale) || !stream_of(v[5], &s)) return -1;
    const int64_t E = L.size[0], D = L.size[1], T = I.size[0];
    embed_t entry;
    if (!is(O, T, D) || !entry_of(v[0], &entry)) return -1;
    return call(entry, (const void*)L.data, ints(I), O.data, E, D, T, scale, k.code, s);
  });
}

// (entry, dO, Idx, dLUT, workspace or None, scale, pad, add, stream)
PyObject* call_embed_grad(PyObject*, PyObject* const* v, Py_ssize_t n) {
  return guarded([&]() -> int {
    Kind k, g;
    Arg d, I, G;
    void *s, *ws;
    size_t bytes;
    float scale;
    int64_t pad;
    int32_t add;
    if (n != 9 || !kind_of(v[1], &k) || !kind_of(v[3], &g) || (g.code != k.code && g.code != 0) || !take(v[1], k, 2, &d) || !take_ints(v[2], 1, &I) ||
        !take(v[3], g, 2, &G) || !workspace_of(v[4], &ws, &bytes) || !number(v[5], &scale) || !whole_number(v[6], &pad) || !truth(v[7], &add) || !stream_of(v[8], &s))
      return -1;
    const int64_t T = d.size[0], D = d.size[1], E = G.size[0];
    embed_grad_t entry;
    if (G.size[1] != D || I.size[0] != T || !entry_of(v[0], &entry)) return -1;
    return call(entry, (const void*)d.data, ints(I), G.data, E, D, T, scale, pad, add, k.code, g.code, ws, bytes, s);
  });
}

// (entry, L, Wt, Id, Off, Row, Place, workspace or None, norm, stream)
PyObject* call_route(PyObject*, PyObject* const* v, Py_ssize_t n) {
  return guarded([&]() -> int {
    Kind k;
    Arg L, W, I, F, R, P;
    void *s, *ws;
    size_t bytes;
    int32_t norm;
    if (n != 10 || !kind_of(v[1], &k) || !take(v[1], k, 2, &L) || !take(v[2], 2, &W) || !take_ints(v[3], 2, &I) || !take_ints(v[4], 1, &F) || !take_ints(v[5], 1, &R) ||
        !take_ints(v[6], 2, &P) || !workspace_of(v[7], &ws, &bytes) || !truth(v[8], &norm) || !stream_of(v[9], &s))
      return -1;
    const int64_t T = L.size[0], E = L.size[1], top = I.size[1];
    route_t entry;
    if (!is(I, T, top) || !is(W, T, top) || !is(P, T, top) || F.size[0] != E + 1 || R.size[0] != T * top || !entry_of(v[0], &entry)) return -1;
    return call(entry, (const void*)L.data, out(W), (int32_t*)I.data, (int32_t*)F.data, (int32_t*)R.data, (int32_t*)P.data, T, E, top, norm, k.code, ws, bytes, s);
  });
}

// (entry, L, Id, dWt, dL, norm, stream)
PyObject* call_route_grad(PyObject*, PyObject* const* v, Py_ssize_t n) {
  return guarded([&]() -> int {
    Kind k;
    Arg L, I, W, G;
    void* s;
    int32_t norm;
    if (n != 7 || !kind_of(v[1], &k) || !take(v[1], k, 2, &L) || !take_ints(v[2], 2, &I) || !take(v[3], 2, &W) || !take(v[4], k, 2, &G) || !truth(v[5], &norm) ||
        !stream_of(v[6], &s))
      return -1;
    const int64_t T = L.size[0], E = L.size[1], top = I.size[1];
    route_grad_t entry;
    if (!is(I, T, top) || !is(W, T, top) || !is(G, T, E) || !entry_of(v[0], &entry)) return -1;
    return call(entry, (const void*)L.data, ints(I), f(W), G.data, T, E, top, norm, k.code, s);
  });
}

// (entry, X, W, Off, Row or None, Y, relu, stream)
PyObject* call_expert_mm(PyObject*, PyObject* const* v, Py_ssize_t n) {
  return guarded([&]() -> int {
    Kind k;
    Arg X, W, F, Row, Y;
    void* s;
    int32_t relu;
    if (n != 8 || !kind_of(v[1], &k) || !take(v[1], k, 2, &X) || !take(v[2], k, 3, &W) || !take_ints(v[3], 1, &F) || !take_ints_or_none(v[4], 1, &Row) ||
        !take(v[5], k, 2, &Y) || !truth(v[6], &relu) || !stream_of(v[7], &s))
      return -1;
    const int64_t T = X.size[0], K = X.size[1], E = W.size[0], N = W.size[1], R = Y.size[0];
    expert_mm_t entry;
    if (W.size[2] != K || F.size[0] != E + 1 || Y.size[1] != N || (Row.size ? Row.size[0] : T) != R || !entry_of(v[0], &entry)) return -1;
    return call(entry, (const void*)X.data, (const void*)W.data, ints(F), ints(Row), Y.data, T, R, E, N, K, relu, k.code, s);
  });
}

// (entry, dY, W, Off, gate or None, dX, stream)
PyObject* call_expert_mm_grad_x(PyObject*, PyObject* const* v, Py_ssize_t n) {
  return guarded([&]() -> int {
    Kind k;
    Arg d, W, F, g, X;
    void* s;
    if (n != 7 || !kind_of(v[1], &k) || !take(v[1], k, 2, &d) || !take(v[2], k, 3, &W) || !take_ints(v[3], 1, &F) || !take_or_none(v[4], k, 2, &g) ||
        !take(v[5], k, 2, &X) || !stream_of(v[6], &s))
      return -1;
    const int64_t R = d.size[0], N = d.size[1], E = W.size[0], K = W.size[2];
    expert_mm_grad_x_t entry;
    if (W.size[1] != N || F.size[0] != E + 1 || !is(X, R, K) || (g.size && !is(g, R, K)) || !entry_of(v[0], &entry)) return -1;
    return call(entry, (const void*)d.data, (const void*)W.data, ints(F), (const void*)g.data, X.data, R, E, N, K, k.code, s);
  });
}

// (entry, dY, X, Off, Row or None, dW, workspace or None, add, stream)
PyObject* call_expert_mm_grad_w(PyObject*, PyObject* const* v, Py_ssize_t n) {
  return guarded([&]() -> int {
    Kind k, g;
    Arg d, X, F, Row, W;
    void *s, *ws;
    size_t bytes;
    int32_t add;
    if (n != 9 || !kind_of(v[1], &k) || !kind_of(v[5], &g) || (g.code != k.code && g.code != 0) || !take(v[1], k, 2, &d) || !take(v[2], k, 2, &X) ||
        !take_ints(v[3], 1, &F) || !take_ints_or_none(v[4], 1, &Row) || !take(v[5], g, 3, &W) || !workspace_of(v[6], &ws, &bytes) || !truth(v[7], &add) ||
        !stream_of(v[8], &s))
      return -1;
    const int64_t R = d.size[0], N = d.size[1], T = X.size[0], K = X.size[1], E = W.size[0];
    expert_mm_grad_w_t entry;
    if (W.size[1] != N || W.size[2] != K || F.size[0] != E + 1 || (Row.size ? Row.size[0] : T) != R || !entry_of(v[0], &entry)) return -1;
    return call(entry, (const void*)d.data, (const void*)X.data, ints(F), ints(Row), W.data, T, R, E, N, K, add, k.code, g.code, ws, bytes, s);
  });
}

// (entry, Y, Wt or None, Place, O, stream)
PyObject* call_expert_sum(PyObject*, PyObject* const* v, Py_ssize_t n) {
  return guarded([&]() -> int {
    Kind k;
    Arg Y, W, P, O;
    void* s;
    if (n != 6 || !kind_of(v[1], &k) || !take(v[1], k, 2, &Y) || (v[2] != Py_None && !take(v[2], 2, &W)) || !take_ints(v[3], 2, &P) || !take(v[4], k, 2, &O) ||
        !stream_of(v[5], &s))
      return -1;
    const int64_t R = Y.size[0], N = Y.size[1], T = P.size[0], top = P.size[1];
    expert_sum_t entry;
    if (!is(O, T, N) || (W.size && !is(W, T, top)) || !entry_of(v[0], &entry)) return -1;
    return call(entry, (const void*)Y.data, f(W), ints(P), O.data, T, R, top, N, k.code, s);
  });
}

// (entry, dO, Y, Wt, Place, dY, dWt, stream)
PyObject* call_expert_sum_grad(PyObject*, PyObject* const* v, Py_ssize_t n) {
  return guarded([&]() -> int {
    Kind k;
    Arg d, Y, W, P, dY, dW;
    void* s;
    if (n != 8 || !kind_of(v[1], &k) || !take(v[1], k, 2, &d) || !take(v[2], k, 2, &Y) || !take(v[3], 2, &W) || !take_ints(v[4], 2, &P) || !take(v[5], k, 2, &dY) ||
        !take(v[6], 2, &dW) || !stream_of(v[7], &s))
      return -1;
    const int64_t R = Y.size[0], N = Y.size[1], T = P.size[0], top = P.size[1];
    expert_sum_grad_t entry;
    if (!is(d, T, N) || !is(W, T, top) || !is(dW, T, top) || !is(dY, R, N) || !entry_of(v[0], &entry)) return -1;
    return call(entry, (const void*)d.data, (const void*)Y.data, f(W), ints(P), dY.data, out(dW), T, R, top, N, k.code, s);
  });
}

template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyMethodDef method(const char* name) {
  return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(F)), METH_FASTCALL, nullptr};
}

PyMethodDef methods[] = {method<call_tbmm>("tbmm"),   method<call_tbmm_ws>("tbmm_ws"), method<call_mlp>("mlp"),
                         method<call_gconv>("gconv"), method<call_kron>("kron"),       method<call_sconv>("sconv"),
                         method<call_lut>("lut"),     method<call_embed>("embed"),     method<call_embed_grad>("embed_grad"),
                         method<call_route>("route"), method<call_route_grad>("route_grad"), method<call_expert_mm>("expert_mm"),
                         method<call_expert_mm_grad_x>("expert_mm_grad_x"), method<call_expert_mm_grad_w>("expert_mm_grad_w"),
                         method<call_expert_sum>("expert_sum"), method<call_expert_sum_grad>("expert_sum_grad"),
                         {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fast", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__fast(void) { return PyModule_Create(&module); }
