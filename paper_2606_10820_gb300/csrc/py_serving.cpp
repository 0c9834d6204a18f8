// The Python binding of the serving operators (serving.py): argument checks and
// marshalling of torch tensors, and nothing else.  A call of the library enqueues in 3 to
// 4 us; its checks and outputs took 8 to 11 us through ctypes and Python attributes, more than
// a small operator runs.
//
// Shapes, types, strides and devices that a call does not take raise ValueError; what
// the library refuses raises the binding's KfError (set_check).  Work goes to the current
// torch stream of the tensors' device, outputs and scratch come from torch's allocator.
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/cuda/EmptyTensor.h>
#include <c10/core/GradMode.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>

#include <algorithm>
#include <cmath>
#include <optional>
#include <string>

#include "../../include/kforcing.h"
#include "../../include/kforcing_serving.h"

namespace {

PyObject* g_check = nullptr;      // called with a status other than KF_OK; raises

struct Refused { std::string what; };      // a ValueError
void need(bool ok, const char* what) {
  if (!ok) throw Refused{what};
}
const at::Tensor& tensor(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) throw Refused{std::string(name) + ": a torch tensor is wanted"};
  return THPVariable_Unpack(o);
}
bool none(PyObject* o) { return o == Py_None; }
int64_t integer(PyObject* o, const char* name, int64_t lo, int64_t hi) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) {
    PyErr_Clear();
    throw Refused{std::string(name) + ": a whole number is wanted"};
  }
  if (v < lo || v > hi) throw Refused{std::string(name) + ": out of range"};
  return v;
}
int32_t int32(PyObject* o, const char* name) { return (int32_t)integer(o, name, INT32_MIN, INT32_MAX); }
double real(PyObject* o, const char* name) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) {
    PyErr_Clear();
    throw Refused{std::string(name) + ": a number is wanted"};
  }
  return v;
}
float number(PyObject* o, const char* name) { return (float)real(o, name); }
int32_t narrow(int64_t v, const char* name) {
  if (v > INT32_MAX) throw Refused{std::string(name) + ": too long"};
  return (int32_t)v;
}
int32_t type_of(const at::Tensor& t, bool fp32, const char* what) {
  const auto s = t.scalar_type();
  if (s == at::kBFloat16) return KF_TYPE_BF16;
  if (s == at::kHalf) return KF_TYPE_FP16;
  if (fp32 && s == at::kFloat) return KF_TYPE_FP32;
  throw Refused{what};
}
void* addr(const at::Tensor& t) { return t.data_ptr(); }
// the operators have no backward pass: what would need one is refused, not dropped
bool wants_gradient(const at::Tensor& t) { return t.requires_grad() && at::GradMode::is_enabled(); }
void plain(const at::Tensor& t, const char* name) {
  if (wants_gradient(t))
    throw Refused{std::string(name) + ": requires a gradient, which this call does not pass on (detach it, or call under torch.no_grad())"};
}
// a call has written the tensor: autograd is to see it
void changed(const at::Tensor& t) {
  if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}
// a contiguous tensor of this type and shape on the device
void* on(const at::Tensor& t, c10::Device dev, at::ScalarType type, at::IntArrayRef shape, const char* name) {
  if (t.device() != dev || t.scalar_type() != type || t.sizes() != shape || !t.is_contiguous())
    throw Refused{std::string(name) + ": a contiguous tensor of the type, shape and device that the call asks for is wanted"};
  return t.data_ptr();
}
int32_t* ints(PyObject* o, c10::Device dev, at::IntArrayRef shape, const char* name) {
  return static_cast<int32_t*>(on(tensor(o, name), dev, at::kInt, shape, name));
}
// a list of int32 on the device; its length
int32_t length(PyObject* o, const char* name) {
  const at::Tensor& t = tensor(o, name);
  if (t.dim() != 1) throw Refused{std::string(name) + ": a list of int32 on the GPU is wanted"};
  return narrow(t.size(0), name);
}
// the stride of a dimension; of one of a single element any will do, whatever the tensor says
int64_t step(const at::Tensor& t, int64_t d) { return t.size(d) == 1 ? t.size(-1) : t.stride(d); }
at::Tensor make(at::IntArrayRef shape, at::ScalarType type, c10::Device dev) {
  return at::Tensor(at::detail::empty_cuda(shape, type, dev, std::nullopt));      // (at::empty without the dispatcher)
}
// scratch of one call (calls on several streams may overlap): none where 0 bytes are enough
struct Scratch {
  at::Tensor t;
  Scratch(int64_t bytes, c10::Device dev) {
    if (bytes > 0) t = make({bytes}, at::kByte, dev);
  }
  void* ptr() const { return t.defined() ? t.data_ptr() : nullptr; }
};
// the device made current, and its current stream
struct On {
  c10::cuda::CUDAGuard guard;
  void* stream;
  explicit On(c10::Device dev) : guard(dev), stream(c10::cuda::getCurrentCUDAStream(dev.index()).stream()) {}
};
// raises through the binding's check; true: an exception is set
bool failed(int rc) {
  if (rc == KF_OK) return false;
  PyObject* r = g_check ? PyObject_CallFunction(g_check, "i", rc) : nullptr;
  if (r) {
    Py_DECREF(r);
    PyErr_SetString(PyExc_RuntimeError, "kforcing: a call failed");
  } else if (!PyErr_Occurred()) {
    PyErr_SetString(PyExc_RuntimeError, "kforcing: a call failed, and no check is set");
  }
  return true;
}
PyObject* done() { Py_RETURN_NONE; }
void put(PyObject* dict, const char* key, const at::Tensor& t) {
  PyObject* v = THPVariable_Wrap(t);
  const int rc = v ? PyDict_SetItemString(dict, key, v) : -1;
  Py_XDECREF(v);
  if (rc) throw python_error();
}

// a function of `n` positional arguments; C++ exceptions become Python ones
#define KF_PY(name, n)                                                                      \
  PyObject* name##_(PyObject* const* a);                                                    \
  PyObject* name(PyObject*, PyObject* const* a, Py_ssize_t count) {                         \
    HANDLE_TH_ERRORS                                                                        \
    if (count != n) {                                                                       \
      PyErr_SetString(PyExc_TypeError, #name ": wrong number of arguments");                \
      return nullptr;                                                                       \
    }                                                                                       \
    try {                                                                                   \
      return name##_(a);                                                                    \
    } catch (const Refused& r) {                                                            \
      PyErr_SetString(PyExc_ValueError, (std::string(#name) + ": " + r.what).c_str());      \
      return nullptr;                                                                       \
    }                                                                                       \
    END_HANDLE_TH_ERRORS                                                                    \
  }                                                                                         \
  PyObject* name##_(PyObject* const* a)

KF_PY(set_check, 1) {
  Py_INCREF(a[0]);
  Py_XDECREF(g_check);
  g_check = a[0];
  return done();
}

// ------------------------------------------------------ rotary positions
// heads [T, H, hd] of contiguous elements; `like`: of its tokens, head size, type and device
void heads(const at::Tensor& t, const at::Tensor* like, const char* name, const char* want) {
  need(t.is_cuda() && t.dim() == 3 && t.stride(2) == 1, want);
  if (like)
    need(t.size(0) == like->size(0) && t.size(2) == like->size(2) && t.scalar_type() == like->scalar_type() && t.device() == like->device(), want);
  plain(t, name);
}
// q, k, freq, q_weight | None, k_weight | None, eps | None, neighbours
struct Turn {
  const at::Tensor &q, &k;
  c10::Device dev;
  int64_t T;
  int32_t type, Hq, Hkv, hd, n, neighbours;
  const double* freq;
  float eps;
  const void* w[2];
  Turn(PyObject* q_, PyObject* k_, PyObject* f, PyObject* wq, PyObject* wk, PyObject* e, PyObject* nb) : q(tensor(q_, "q")), k(tensor(k_, "k")), dev(q.device()) {
    heads(q, nullptr, "q", "q: [T, Hq, hd] on a GPU, heads of contiguous elements");
    type = type_of(q, false, "q and k: bf16 or fp16");
    heads(k, &q, "k", "k: [T, Hkv, hd] of q's type and device, heads of contiguous elements");
    T = q.size(0);
    Hq = narrow(q.size(1), "q");
    Hkv = narrow(k.size(1), "k");
    hd = narrow(q.size(2), "q");
    const at::Tensor& ft = tensor(f, "freq");
    need(ft.dim() == 1, "freq: a list of fp64 on the GPU");
    n = narrow(ft.size(0), "freq");
    freq = static_cast<const double*>(on(ft, dev, at::kDouble, {(int64_t)n}, "freq"));
    plain(ft, "freq");
    int i = 0;
    for (PyObject* o : {wq, wk}) {
      const char* name = i ? "k_weight" : "q_weight";
      w[i] = none(o) ? nullptr : on(tensor(o, name), dev, q.scalar_type(), {(int64_t)hd}, name);
      if (w[i++]) plain(THPVariable_Unpack(o), name);
    }
    eps = none(e) ? -1.f : number(e, "eps");
    need(none(e) || eps >= 0.f, "eps: 0 or more (None: no norms)");
    neighbours = PyObject_IsTrue(nb);
    if (neighbours < 0) throw python_error();
  }
  const int32_t* positions(PyObject* o) const { return ints(o, dev, {T}, "pos"); }
};
at::Tensor heads_out(PyObject* o, const at::Tensor& like, const char* name) {
  if (none(o)) return make({like.size(0), like.size(1), like.size(2)}, like.scalar_type(), like.device());
  const at::Tensor& t = tensor(o, name);
  if (t.sizes() != like.sizes() || t.scalar_type() != like.scalar_type() || t.device() != like.device() || t.stride(2) != 1)
    throw Refused{std::string(name) + ": a tensor like its input"};
  plain(t, name);
  return t;
}
// q, k, pos, freq, q_weight, k_weight, eps, neighbours, q_out | None, k_out | None
KF_PY(rotate_heads, 10) {
  const Turn x(a[0], a[1], a[3], a[4], a[5], a[6], a[7]);
  const int32_t* pos = x.positions(a[2]);
  const On at(x.dev);
  const at::Tensor oq = heads_out(a[8], x.q, "q_out"), ok = heads_out(a[9], x.k, "k_out");
  if (failed(kf_op_rotate_heads(x.type, x.T, x.Hq, x.Hkv, x.hd, addr(x.q), step(x.q, 0), step(x.q, 1), addr(x.k), step(x.k, 0), step(x.k, 1),
                                pos, x.freq, x.n, x.neighbours, x.eps, x.w[0], x.w[1], addr(oq), step(oq, 0), step(oq, 1), addr(ok),
                                step(ok, 0), step(ok, 1), at.stream)))
    return nullptr;
  if (!none(a[8])) changed(oq);
  if (!none(a[9])) changed(ok);
  PyObject *pq = THPVariable_Wrap(oq), *pk = THPVariable_Wrap(ok), *both = pq && pk ? PyTuple_Pack(2, pq, pk) : nullptr;
  Py_XDECREF(pq);
  Py_XDECREF(pk);
  return both;
}
// q, k, v, pool, starts, table, lens, slots, freq, q_weight, k_weight, eps, neighbours
KF_PY(rotate_append, 13) {
  const Turn x(a[0], a[1], a[8], a[9], a[10], a[11], a[12]);
  const at::Tensor &v = tensor(a[2], "v"), &pool = tensor(a[3], "pool"), &table = tensor(a[5], "table");
  heads(v, &x.q, "v", "v: [T, Hkv, hd] of q's type and device, heads of contiguous elements");
  need(v.size(1) == x.Hkv, "v: k's heads");
  need(pool.dim() == 5 && pool.size(1) == 2 && table.dim() == 2, "pool: [pages, 2, Hkv, page, hd], table: [slots, width]");
  void* pp = on(pool, x.dev, x.q.scalar_type(), {pool.size(0), 2, x.Hkv, pool.size(3), x.hd}, "pool");
  plain(pool, "pool");
  const int32_t n = length(a[7], "slots"), slots = narrow(table.size(0), "table"), width = narrow(table.size(1), "table");
  const int32_t *which = ints(a[7], x.dev, {(int64_t)n}, "slots"), *starts = ints(a[4], x.dev, {(int64_t)n + 1}, "starts");
  const int32_t *tp = ints(a[5], x.dev, {(int64_t)slots, (int64_t)width}, "table"), *lens = ints(a[6], x.dev, {(int64_t)slots}, "lens");
  const On at(x.dev);
  const at::Tensor oq = make({x.T, x.Hq, x.hd}, x.q.scalar_type(), x.dev);
  if (failed(kf_op_rotate_append(x.type, n, which, starts, x.T, x.Hq, x.Hkv, x.hd, addr(x.q), step(x.q, 0), step(x.q, 1), addr(x.k),
                                 step(x.k, 0), step(x.k, 1), addr(v), step(v, 0), step(v, 1), x.freq, x.n, x.neighbours, x.eps, x.w[0],
                                 x.w[1], addr(oq), pp, narrow(pool.size(0), "pool"), narrow(pool.size(3), "pool"), tp, slots, width, lens,
                                 at.stream)))
    return nullptr;
  changed(pool);
  return THPVariable_Wrap(oq);
}
// dq, dk, q, k, pos, freq, q_weight, k_weight, eps, neighbours
KF_PY(rotate_heads_grad, 10) {
  const Turn x(a[2], a[3], a[5], a[6], a[7], a[8], a[9]);
  const at::Tensor &dq = tensor(a[0], "dq"), &dk = tensor(a[1], "dk");
  heads(dq, &x.q, "dq", "dq: a tensor like q");
  heads(dk, &x.q, "dk", "dk: a tensor like k");
  need(dq.size(1) == x.Hq && dk.size(1) == x.Hkv, "dq and dk: the heads of q and k");
  const int32_t* pos = x.positions(a[4]);
  const On at(x.dev);
  const at::Tensor gq = make({x.T, x.Hq, x.hd}, x.q.scalar_type(), x.dev), gk = make({x.T, x.Hkv, x.hd}, x.q.scalar_type(), x.dev);
  at::Tensor gw[2];
  for (int i = 0; i < 2; ++i)
    if (x.w[i]) gw[i] = make({x.hd}, at::kFloat, x.dev);
  auto p = [&](int i) { return x.w[i] ? static_cast<float*>(gw[i].data_ptr()) : nullptr; };
  const Scratch work(x.w[0] || x.w[1] ? kf_op_rotate_heads_grad_work(x.T, x.Hq, x.Hkv, x.hd) : 0, x.dev);
  if (failed(kf_op_rotate_heads_grad(x.type, x.T, x.Hq, x.Hkv, x.hd, addr(dq), step(dq, 0), step(dq, 1), addr(dk), step(dk, 0), step(dk, 1),
                                     addr(x.q), step(x.q, 0), step(x.q, 1), addr(x.k), step(x.k, 0), step(x.k, 1), pos, x.freq, x.n,
                                     x.neighbours, x.eps, x.w[0], x.w[1], addr(gq), addr(gk), p(0), p(1), work.ptr(), at.stream)))
    return nullptr;
  PyObject* d = PyDict_New();
  if (!d) throw python_error();
  put(d, "q", gq);
  put(d, "k", gk);
  if (x.w[0]) put(d, "q_weight", gw[0]);
  if (x.w[1]) put(d, "k_weight", gw[1]);
  return d;
}

// --------------------------------------------------------------- attention
float scale_of(PyObject* o, int64_t hd) { return none(o) ? (float)(1.0 / std::sqrt((double)hd)) : number(o, "scale"); }

// q, k, v, starts, longest, scale | None, out | None
KF_PY(prompt_attention, 7) {
  const at::Tensor &q = tensor(a[0], "q"), &k = tensor(a[1], "k"), &v = tensor(a[2], "v");
  need(q.is_cuda() && q.dim() == 3 && k.dim() == 3, "q: [T, Hq, hd], k and v: [T, Hkv, hd], on a GPU");
  const int32_t type = type_of(q, false, "q, k and v: bf16 or fp16");
  const int64_t T = q.size(0), Hq = q.size(1), hd = q.size(2), Hkv = k.size(1);
  const c10::Device dev = q.device();
  need(k.size(0) == T && k.size(2) == hd && v.sizes() == k.sizes() && k.scalar_type() == q.scalar_type() &&
           v.scalar_type() == q.scalar_type() && k.device() == dev && v.device() == dev,
       "k and v: [T, Hkv, hd] of q's type and device");
  need(q.stride(2) == 1 && k.stride(2) == 1 && v.stride(2) == 1, "q, k and v: heads of contiguous elements");
  plain(q, "q");
  plain(k, "k");
  plain(v, "v");
  const at::Tensor& st = tensor(a[3], "starts");
  need(st.dim() == 1 && st.size(0) >= 1, "starts: [n + 1]");
  const int32_t n = narrow(st.size(0) - 1, "starts"), longest = int32(a[4], "longest");
  const int32_t* starts = ints(a[3], dev, {(int64_t)n + 1}, "starts");
  const float scale = scale_of(a[5], hd);
  const On at(dev);
  at::Tensor out;
  if (none(a[6])) {
    out = make({T, Hq, hd}, q.scalar_type(), dev);
  } else {
    out = tensor(a[6], "out");
    need(out.sizes() == q.sizes() && out.scalar_type() == q.scalar_type() && out.device() == dev && out.stride(2) == 1,
         "out: a tensor like q");
    plain(out, "out");
  }
  const Scratch work(kf_op_prompt_attention_work(n, T), dev);
  if (failed(kf_op_prompt_attention(type, n, T, longest, narrow(Hq, "q"), narrow(Hkv, "k"), narrow(hd, "q"), addr(q), step(q, 0), step(q, 1),
                                    addr(k), step(k, 0), step(k, 1), addr(v), step(v, 0), step(v, 1), addr(out), step(out, 0),
                                    step(out, 1), starts, scale, work.ptr(), at.stream)))
    return nullptr;
  if (!none(a[6])) changed(out);
  return THPVariable_Wrap(out);
}

// q, pool, table, lens, scale | None, out | None: what both attentions over a cache take
struct Paged {
  const at::Tensor &q, &pool, &table;
  c10::Device dev;
  int32_t type, B, rows, Hq, Hkv, hd, page, width;
  int64_t n_pages;
  void *pp;
  const int32_t *tp, *lp;
  float scale;
  Paged(PyObject* q_, PyObject* p, PyObject* t, PyObject* l, PyObject* s)
      : q(tensor(q_, "q")), pool(tensor(p, "pool")), table(tensor(t, "table")), dev(q.device()) {
    need(q.is_cuda() && q.dim() == 4 && pool.dim() == 5 && table.dim() == 2,
         "q: [B, rows, Hq, hd], pool: [pages, 2, Hkv, page, hd], table: [B, width], on a GPU");
    type = type_of(q, false, "q and pool: bf16 or fp16");
    n_pages = pool.size(0);
    need(pool.size(1) == 2 && q.stride(3) == 1, "pool: K and V of each page; q: heads of contiguous elements");
    pp = on(pool, dev, q.scalar_type(), {n_pages, 2, pool.size(2), pool.size(3), q.size(3)}, "pool");
    tp = ints(t, dev, {q.size(0), table.size(1)}, "table");
    lp = ints(l, dev, {q.size(0)}, "lens");
    scale = scale_of(s, q.size(3));
    plain(q, "q");
    plain(pool, "pool");
    B = narrow(q.size(0), "q");
    rows = narrow(q.size(1), "q");
    Hq = narrow(q.size(2), "q");
    Hkv = narrow(pool.size(2), "pool");
    hd = narrow(q.size(3), "q");
    page = narrow(pool.size(3), "pool");
    width = narrow(table.size(1), "table");
  }
  at::Tensor output(PyObject* o) const {
    at::Tensor out = none(o) ? make({B, rows, Hq, hd}, q.scalar_type(), dev) : tensor(o, "out");
    on(out, dev, q.scalar_type(), q.sizes(), "out");
    plain(out, "out");
    return out;
  }
};
KF_PY(paged_attention, 6) {
  const Paged x(a[0], a[1], a[2], a[3], a[4]);
  const On at(x.dev);
  const at::Tensor out = x.output(a[5]);
  const Scratch work(kf_op_paged_attention_work(x.B, x.rows, x.Hq, x.Hkv, x.hd, x.page, x.width), x.dev);
  if (failed(kf_op_paged_attention(x.type, x.B, x.rows, x.Hq, x.Hkv, x.hd, addr(x.q), step(x.q, 0), step(x.q, 1), step(x.q, 2), x.pp, x.n_pages,
                                   x.page, x.tp, x.width, x.lp, x.scale, addr(out), work.ptr(), at.stream)))
    return nullptr;
  if (!none(a[5])) changed(out);
  return THPVariable_Wrap(out);
}
// q, pool, table, lens, groups, shared, scale | None, out | None
KF_PY(shared_attention, 8) {
  const Paged x(a[0], a[1], a[2], a[3], a[6]);
  const int32_t n = length(a[5], "shared");
  const int32_t *groups = ints(a[4], x.dev, {(int64_t)n + 1}, "groups"), *shared = ints(a[5], x.dev, {(int64_t)n}, "shared");
  const On at(x.dev);
  const at::Tensor out = x.output(a[7]);
  const Scratch work(kf_op_shared_attention_work(x.B, x.rows, x.Hq, x.Hkv, x.hd, x.n_pages, x.page, x.width, n), x.dev);
  if (failed(kf_op_shared_attention(x.type, x.B, x.rows, x.Hq, x.Hkv, x.hd, addr(x.q), step(x.q, 0), step(x.q, 1), step(x.q, 2), x.pp, x.n_pages,
                                    x.page, x.tp, x.width, x.lp, n, groups, shared, x.scale, addr(out), work.ptr(), at.stream)))
    return nullptr;
  if (!none(a[7])) changed(out);
  return THPVariable_Wrap(out);
}

// ------------------------------------------------------------------- pages
struct Book {
  c10::Device dev;
  int32_t n_pages, slots, width;
  int32_t *ref, *table, *lens;
  PyObject* parts[3];
  Book(PyObject* r, PyObject* t, PyObject* l) : dev(c10::kCPU), parts{r, t, l} {
    const at::Tensor &rt = tensor(r, "ref"), &tt = tensor(t, "table");
    need(rt.is_cuda() && rt.dim() == 1 && tt.dim() == 2, "ref: [pages], table: [slots, width], int32 on a GPU");
    dev = rt.device();
    n_pages = narrow(rt.size(0), "ref");
    slots = narrow(tt.size(0), "table");
    width = narrow(tt.size(1), "table");
    ref = ints(r, dev, {(int64_t)n_pages}, "ref");
    table = ints(t, dev, {(int64_t)slots, (int64_t)width}, "table");
    lens = l ? ints(l, dev, {(int64_t)slots}, "lens") : nullptr;
  }
  void written() const {
    for (PyObject* o : parts)
      if (o) changed(THPVariable_Unpack(o));
  }
};
struct Pool {
  const at::Tensor& t;
  void* p;
  int32_t layers, n_pages;
  int64_t page_bytes;
  Pool(const at::Tensor& t_, c10::Device dev, int64_t pages) : t(t_) {
    need(t.dim() >= 3 && t.device() == dev && t.is_contiguous() && t.size(1) == pages,
         "pool: a contiguous [layers, pages, ...] tensor on the book's device");
    plain(t, "pool");
    p = addr(t);
    layers = narrow(t.size(0), "pool");
    n_pages = narrow(pages, "pool");
    // (not t.stride(1): a dimension of one page may have any)
    page_bytes = layers && n_pages ? t.numel() / layers / n_pages * (int64_t)t.element_size() : 0;
  }
};

// ref, table, lens, slots, new_lens, page
KF_PY(pages_grow, 6) {
  const Book b(a[0], a[1], a[2]);
  const int32_t n = length(a[3], "slots");
  const int32_t *which = ints(a[3], b.dev, {(int64_t)n}, "slots"), *lens = ints(a[4], b.dev, {(int64_t)n}, "new_lens");
  const On at(b.dev);
  const Scratch work(kf_op_pages_work(b.n_pages, b.slots, n), b.dev);
  if (failed(kf_op_pages_grow(n, which, lens, b.ref, b.n_pages, b.table, b.slots, b.width, b.lens, int32(a[5], "page"), work.ptr(),
                                 at.stream)))
    return nullptr;
  b.written();
  return done();
}
// ref, table, lens, slots, page
KF_PY(pages_free, 5) {
  const Book b(a[0], a[1], a[2]);
  const int32_t n = length(a[3], "slots");
  const int32_t* which = ints(a[3], b.dev, {(int64_t)n}, "slots");
  const On at(b.dev);
  const Scratch work(kf_op_pages_work(b.n_pages, b.slots, n), b.dev);
  if (failed(kf_op_pages_free(n, which, b.ref, b.n_pages, b.table, b.slots, b.width, b.lens, int32(a[4], "page"), work.ptr(), at.stream)))
    return nullptr;
  b.written();
  return done();
}
// pool, ref, table, lens, src, dst
KF_PY(pages_fork, 6) {
  const Book b(a[1], a[2], a[3]);
  const at::Tensor& t = tensor(a[0], "pool");
  need(t.dim() == 6, "pool: [layers, pages, 2, Hkv, page, hd]");
  const Pool p(t, b.dev, b.n_pages);
  const int32_t n = length(a[4], "src");
  const int32_t *src = ints(a[4], b.dev, {(int64_t)n}, "src"), *dst = ints(a[5], b.dev, {(int64_t)n}, "dst");
  const On at(b.dev);
  const Scratch work(kf_op_pages_work(b.n_pages, b.slots, n), b.dev);
  if (failed(kf_op_pages_fork(n, src, dst, b.ref, b.n_pages, b.table, b.slots, b.width, b.lens, narrow(t.size(4), "pool"), p.p, p.layers,
                                 p.page_bytes, work.ptr(), at.stream)))
    return nullptr;
  b.written();
  changed(p.t);
  return done();
}
// pool, ref, table, live | None
KF_PY(pages_compact, 4) {
  const Book b(a[1], a[2], nullptr);
  const Pool p(tensor(a[0], "pool"), b.dev, b.n_pages);
  int32_t* live = none(a[3]) ? nullptr : ints(a[3], b.dev, {1}, "live");
  const On at(b.dev);
  const Scratch work(kf_op_pages_work(b.n_pages, b.slots, 0), b.dev);
  if (failed(kf_op_pages_compact(b.ref, b.n_pages, b.table, b.slots, b.width, p.p, p.layers, p.page_bytes, live, work.ptr(), at.stream)))
    return nullptr;
  b.written();
  changed(p.t);
  if (!none(a[3])) changed(THPVariable_Unpack(a[3]));
  return done();
}
// pool, src, dst
KF_PY(pages_copy, 3) {
  const at::Tensor& t = tensor(a[0], "pool");
  need(t.is_cuda() && t.dim() >= 3, "pool: [layers, pages, ...] on a GPU");
  const Pool p(t, t.device(), t.size(1));
  const int32_t n = length(a[1], "src");
  const int32_t *src = ints(a[1], t.device(), {(int64_t)n}, "src"), *dst = ints(a[2], t.device(), {(int64_t)n}, "dst");
  const On at(t.device());
  if (failed(kf_op_pages_copy(n, src, dst, p.p, p.layers, p.n_pages, p.page_bytes, at.stream))) return nullptr;
  changed(t);
  return done();
}
// pool, k, v, starts, table, lens, slots
KF_PY(pages_append, 7) {
  const at::Tensor &pool = tensor(a[0], "pool"), &k = tensor(a[1], "k"), &v = tensor(a[2], "v"), &table = tensor(a[4], "table");
  need(pool.is_cuda() && pool.dim() == 5 && pool.size(1) == 2 && pool.element_size() == 2 && pool.is_contiguous() && k.dim() == 3 &&
           table.dim() == 2,
       "pool: [pages, 2, Hkv, page, hd], k and v: [T, Hkv, hd], 16-bit elements on a GPU");
  const c10::Device dev = pool.device();
  const int64_t T = k.size(0), Hkv = pool.size(2), hd = pool.size(4);
  need(k.size(1) == Hkv && k.size(2) == hd && v.sizes() == k.sizes() && k.scalar_type() == pool.scalar_type() &&
           v.scalar_type() == pool.scalar_type() && k.device() == dev && v.device() == dev && k.stride(2) == 1 && v.stride(2) == 1,
       "k and v: rows of the pool's heads, type and device");
  plain(pool, "pool");
  plain(k, "k");
  plain(v, "v");
  const int32_t n = length(a[6], "slots"), slots = narrow(table.size(0), "table"), width = narrow(table.size(1), "table");
  const int32_t *which = ints(a[6], dev, {(int64_t)n}, "slots"), *starts = ints(a[3], dev, {(int64_t)n + 1}, "starts");
  const int32_t *tp = ints(a[4], dev, {(int64_t)slots, (int64_t)width}, "table"), *lens = ints(a[5], dev, {(int64_t)slots}, "lens");
  const On at(dev);
  if (failed(kf_op_pages_append(n, which, starts, T, narrow(Hkv, "pool"), narrow(hd, "pool"), addr(k), step(k, 0), step(k, 1), addr(v),
                                   step(v, 0), step(v, 1), addr(pool), narrow(pool.size(0), "pool"), narrow(pool.size(3), "pool"), tp,
                                   slots, width, lens, at.stream)))
    return nullptr;
  changed(pool);
  return done();
}

// ------------------------------------------------------------------ scores
struct Logits {
  const at::Tensor& t;
  c10::Device dev;
  int32_t type, V;
  int64_t R, stride;
  const int64_t* tokens;
  at::Tensor logp, entropy, lse;
  Logits(PyObject* l, PyObject* tok) : t(tensor(l, "logits")), dev(t.device()) {
    need(t.is_cuda() && t.dim() == 2, "logits: [R, V] on a GPU");
    type = type_of(t, true, "logits: fp32, bf16 or fp16");
    R = t.size(0);
    V = narrow(t.size(1), "logits");
    need(V > 0 && (t.stride(1) == 1 || V == 1), "logits: rows of contiguous elements");
    stride = R > 1 ? t.stride(0) : V;
    need(stride >= V, "logits: rows that do not overlap");
    tokens = static_cast<const int64_t*>(on(tensor(tok, "tokens"), dev, at::kLong, {R}, "tokens"));
  }
  void outputs(bool with_lse = true) {
    logp = make({R}, at::kFloat, dev);
    entropy = make({R}, at::kFloat, dev);
    if (with_lse) lse = make({R}, at::kFloat, dev);
  }
  float* p(const at::Tensor& x) const { return static_cast<float*>(x.data_ptr()); }
  PyObject* dict() const {
    PyObject* d = PyDict_New();
    if (!d) throw python_error();
    put(d, "logp", logp);
    put(d, "entropy", entropy);
    put(d, "lse", lse);
    return d;
  }
};
// logits, tokens, top, tau
KF_PY(token_scores, 4) {
  Logits x(a[0], a[1]);
  plain(x.t, "logits");
  const int32_t top = (int32_t)integer(a[2], "top: 0 to 64, and at most the vocabulary", 0, std::min(64, x.V));
  const float tau = number(a[3], "tau");
  const On at(x.dev);
  x.outputs();
  at::Tensor ids, lps;
  if (top) {
    ids = make({x.R, top}, at::kInt, x.dev);
    lps = make({x.R, top}, at::kFloat, x.dev);
  }
  if (failed(kf_op_token_scores(x.type, x.R, x.V, addr(x.t), x.stride, x.tokens, tau, top, x.p(x.logp), x.p(x.entropy), x.p(x.lse),
                                top ? static_cast<int32_t*>(ids.data_ptr()) : nullptr, top ? x.p(lps) : nullptr, at.stream)))
    return nullptr;
  PyObject* d = x.dict();
  if (top) {
    put(d, "top_ids", ids);
    put(d, "top_logp", lps);
  }
  return d;
}
// the gradient's tensor: `o`, or a new one
at::Tensor grad_like(const Logits& x, PyObject* o) {
  if (none(o)) return make({x.R, x.V}, x.t.scalar_type(), x.dev);
  const at::Tensor& grad = tensor(o, "out");
  need(grad.scalar_type() == x.t.scalar_type() && grad.device() == x.dev && grad.sizes() == x.t.sizes() && (grad.stride(1) == 1 || x.V == 1),
       "out: a tensor like the logits");
  need(!wants_gradient(grad) || !grad.is_leaf(), "out: a leaf that requires a gradient cannot be written (detach it, or call under torch.no_grad())");
  return grad;
}
// logits, tokens, g_logp | None, g_entropy | None, tau, out | None
KF_PY(token_scores_grad, 6) {
  Logits x(a[0], a[1]);
  const float* g[2];
  for (int i = 0; i < 2; ++i) {
    g[i] = none(a[2 + i]) ? nullptr
                          : static_cast<const float*>(on(tensor(a[2 + i], "g_logp, g_entropy"), x.dev, at::kFloat, {x.R}, "g_logp, g_entropy"));
    if (g[i]) plain(THPVariable_Unpack(a[2 + i]), "g_logp, g_entropy");
  }
  const float tau = number(a[4], "tau");
  const On at(x.dev);
  const at::Tensor grad = grad_like(x, a[5]);
  x.outputs();
  if (failed(kf_op_token_scores_grad(x.type, x.R, x.V, addr(x.t), x.stride, x.tokens, tau, g[0], g[1], x.p(x.logp), x.p(x.entropy),
                                     x.p(x.lse), addr(grad), x.R > 1 ? grad.stride(0) : x.V, at.stream)))
    return nullptr;
  if (!none(a[5])) changed(grad);
  PyObject* d = x.dict();
  put(d, "grad", grad);
  return d;
}

// logits, tokens, old_logp, advantage, ref_logp | None, weight | None, clip below, above, kl_weight, entropy_weight, tau, out | None
KF_PY(policy_loss, 12) {
  Logits x(a[0], a[1]);
  const char* names[4] = {"old_logp", "advantage", "ref_logp", "weight"};
  const float* rows[4];
  for (int i = 0; i < 4; ++i) {
    rows[i] = i >= 2 && none(a[2 + i]) ? nullptr : static_cast<const float*>(on(tensor(a[2 + i], names[i]), x.dev, at::kFloat, {x.R}, names[i]));
    if (rows[i]) plain(THPVariable_Unpack(a[2 + i]), names[i]);
  }
  const float low = number(a[6], "clip"), high = number(a[7], "clip"), kl_weight = number(a[8], "kl_weight"), entropy_weight = number(a[9], "entropy_weight");
  const double tau = real(a[10], "tau");
  const On at(x.dev);
  const at::Tensor grad = grad_like(x, a[11]);
  x.outputs(false);
  const at::Tensor loss = make({x.R}, at::kFloat, x.dev), ratio = make({x.R}, at::kFloat, x.dev);
  at::Tensor kl;
  if (rows[2]) kl = make({x.R}, at::kFloat, x.dev);
  if (failed(kf_op_policy_loss(x.type, x.R, x.V, addr(x.t), x.stride, x.tokens, tau, rows[0], rows[1], rows[2], rows[3], low, high, kl_weight,
                               entropy_weight, x.p(loss), x.p(x.logp), x.p(x.entropy), x.p(ratio), rows[2] ? x.p(kl) : nullptr, addr(grad),
                               x.R > 1 ? grad.stride(0) : x.V, at.stream)))
    return nullptr;
  if (!none(a[11])) changed(grad);
  PyObject* d = PyDict_New();
  if (!d) throw python_error();
  put(d, "loss", loss);
  put(d, "logp", x.logp);
  put(d, "entropy", x.entropy);
  put(d, "ratio", ratio);
  if (rows[2]) put(d, "kl", kl);
  put(d, "grad", grad);
  return d;
}

#define KF_ENTRY(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(name)), METH_FASTCALL, nullptr}
PyMethodDef g_methods[] = {KF_ENTRY(set_check),     KF_ENTRY(rotate_heads),     KF_ENTRY(rotate_append),   KF_ENTRY(rotate_heads_grad),
                           KF_ENTRY(prompt_attention), KF_ENTRY(paged_attention), KF_ENTRY(shared_attention), KF_ENTRY(pages_grow),
                           KF_ENTRY(pages_free),    KF_ENTRY(pages_fork),       KF_ENTRY(pages_compact),   KF_ENTRY(pages_copy),
                           KF_ENTRY(pages_append),  KF_ENTRY(token_scores),     KF_ENTRY(token_scores_grad), KF_ENTRY(policy_loss), {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_serving", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__serving(void) { return PyModule_Create(&g_module); }
