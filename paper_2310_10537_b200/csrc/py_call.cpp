// Python calls of the norm, routing, row-moving, grouped-product and cache entry points, marshalled in C++.
//
// These calls stand in loops whose GPU time is a few microseconds, where checking the tensors, allocating the
// results and converting the arguments in Python costs several times that (norm of 16 x 4096: 15 us of host time
// for 2.6 us on the GPU).  Every function takes its arguments positionally from the wrapper of the same name in
// binding.py, checks them, allocates what it returns on the current stream of the current device and calls the
// C entry point; nothing is computed here.  A wrong tensor raises ValueError, a wrong type TypeError, a
// status of the library MxError.
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/ATen.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>

#include <cmath>
#include <initializer_list>
#include <string>

#include "mx.h"

namespace {

struct Raised {};  // a Python exception is set

PyObject* g_error_type = nullptr;  // MxError(status, where)

[[noreturn]] void fail(PyObject* type, const std::string& text) {
  PyErr_SetString(type, text.c_str());
  throw Raised();
}

void check(int status, const char* where) {
  if (status == MX_OK) return;
  PyObject* e = g_error_type ? PyObject_CallFunction(g_error_type, "is", status, where) : nullptr;
  if (e) {
    PyErr_SetObject(g_error_type, e);
    Py_DECREF(e);
  } else if (!PyErr_Occurred()) {
    PyErr_Format(PyExc_RuntimeError, "%s: status %d", where, status);
  }
  throw Raised();
}

std::string describe(c10::ScalarType dtype, at::IntArrayRef sizes) {
  std::string s = std::string(c10::toString(dtype)) + " [";
  for (size_t i = 0; i < sizes.size(); ++i) s += (i ? ", " : "") + std::to_string(sizes[i]);
  return s + "]";
}

// A tensor argument; None is a null pointer where that is allowed.
const at::Tensor* tensor(PyObject* o, const char* name, bool optional = false) {
  if (optional && o == Py_None) return nullptr;
  if (!THPVariable_Check(o)) fail(PyExc_TypeError, std::string(name) + " has to be a tensor");
  return &THPVariable_Unpack(o);
}
int64_t integer(PyObject* o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw Raised();
  return v;
}
int small(PyObject* o) {  // an enum or a flag: anything that does not fit is a value the library refuses
  const int64_t v = integer(o);
  return v < -1 || v > 1 << 20 ? -1 : (int)v;
}
float real(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Raised();
  return (float)v;
}

// The device of the call: that of its first tensor, which has to be the current one.
int call_device(const at::Tensor& t) {
  if (!t.is_cuda() || t.get_device() != c10::cuda::current_device())
    fail(PyExc_ValueError, "tensors have to be on the current CUDA device, not on " + t.device().str());
  return t.get_device();
}
void on_device(const at::Tensor& t, const char* name, int dev) {
  if (!t.is_cuda() || t.get_device() != dev || !t.is_contiguous())
    fail(PyExc_ValueError, std::string(name) + " has to be a contiguous tensor on the current CUDA device");
}
// The address of a tensor of exactly this type and shape; null stays null.
void* need(const at::Tensor* t, const char* name, int dev, c10::ScalarType dtype, std::initializer_list<int64_t> sizes) {
  if (!t) return nullptr;
  on_device(*t, name, dev);
  const at::IntArrayRef want(sizes.begin(), sizes.size());
  if (t->scalar_type() != dtype || t->sizes() != want)
    fail(PyExc_ValueError, std::string(name) + " has to be " + describe(dtype, want) + ", not " +
                               describe(t->scalar_type(), t->sizes()));
  return t->data_ptr();
}
// The address of a contiguous tensor of at least this many bytes.
void* holds(const at::Tensor& t, const char* name, int dev, int64_t bytes) {
  on_device(t, name, dev);
  if ((int64_t)t.nbytes() < bytes)
    fail(PyExc_ValueError, std::string(name) + " holds " + std::to_string(t.nbytes()) + " bytes, " +
                               std::to_string(bytes) + " are needed");
  return t.data_ptr();
}
void two_dims(const at::Tensor& t, const char* name, const char* what) {
  if (t.dim() != 2) fail(PyExc_ValueError, std::string(name) + " has to be " + what);
}
mx_dtype_t float_code(c10::ScalarType d) {
  if (d == at::kFloat) return MX_F32;
  if (d == at::kBFloat16) return MX_BF16;
  fail(PyExc_TypeError, std::string("unsupported float dtype ") + c10::toString(d));
}
mx_dtype_t float_code(const at::Tensor& t) { return float_code(t.scalar_type()); }

at::Tensor make(const at::Tensor& like, c10::ScalarType dtype, std::initializer_list<int64_t> sizes) {
  for (int64_t s : sizes)
    if (s < 0) fail(PyExc_ValueError, "negative extent");
  // Past the dispatcher, whose part is more than the allocation's: a norm of 16 x 4096 with its three results takes the
  // host 4.55 us, 5.4 with at::empty.
  return at::Tensor(at::detail::empty_cuda(at::IntArrayRef(sizes.begin(), sizes.size()), dtype, like.device(), std::nullopt));
}

mx_opts_t options(int dev, int dtype, int layout = MX_SCALES_SWIZZLED, bool check_status = false) {
  return {dtype, layout, (void*)c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)dev).stream(), check_status ? 1 : 0, 0};
}

// Bytes of the codes and scales of an MX tensor [rows, dim] (0 where the library refuses the shape).
int64_t code_bytes(int64_t rows, int64_t dim, int fmt) {
  const int64_t shape[2] = {rows, dim};
  return (int64_t)mx_elems_bytes(shape, 2, 1, (mx_fmt_t)fmt);
}
int64_t scale_bytes(int64_t rows, int64_t dim, int layout) {
  const int64_t shape[2] = {rows, dim};
  return (int64_t)mx_scales_bytes(shape, 2, 1, (mx_scale_layout_t)layout);
}

// The lock is not held while the library launches (or, with a status check, waits).
struct Unlocked {
  PyThreadState* state = PyEval_SaveThread();
  ~Unlocked() { PyEval_RestoreThread(state); }
};
template <typename F>
int unlocked(F f) {
  Unlocked u;
  return f();
}

PyObject* wrap(const at::Tensor& t) { return THPVariable_Wrap(t); }
PyObject* pair(PyObject* a, PyObject* b) {
  PyObject* r = a && b ? PyTuple_Pack(2, a, b) : nullptr;
  Py_XDECREF(a);
  Py_XDECREF(b);
  return r;
}
PyObject* given(PyObject* o) {
  Py_INCREF(o);
  return o;
}

using Args = PyObject* const*;

// x weight fmt eps residual rounding layout y_out h_out out_elems out_scales
PyObject* rmsnorm_quantize(Args a) {
  const at::Tensor &x = *tensor(a[0], "x"), &w = *tensor(a[1], "weight");
  two_dims(x, "x", "[rows, dim]");
  const at::Tensor *res = tensor(a[4], "residual", true), *y = tensor(a[7], "y_out", true), *h = tensor(a[8], "h_out", true);
  const at::Tensor *oe = tensor(a[9], "elems", true), *os = tensor(a[10], "scales", true);
  const int dev = call_device(x), fmt = small(a[2]), layout = small(a[6]);
  const int64_t rows = x.size(0), dim = x.size(1), ne = code_bytes(rows, dim, fmt), ns = scale_bytes(rows, dim, layout);
  const auto dt = x.scalar_type();
  void *px = need(&x, "x", dev, dt, {rows, dim}), *pr = need(res, "residual", dev, dt, {rows, dim});
  void *pw = need(&w, "weight", dev, w.scalar_type(), {dim}), *py = need(y, "y_out", dev, dt, {rows, dim});
  void* ph = need(h, "h_out", dev, dt, {rows, dim});
  const mx_dtype_t code = float_code(x), wcode = float_code(w);
  at::Tensor elems, scales, hn;
  void *pe = oe ? holds(*oe, "elems", dev, ne) : (elems = make(x, at::kByte, {ne})).data_ptr();
  void *ps = os ? holds(*os, "scales", dev, ns) : (scales = make(x, at::kByte, {ns})).data_ptr();
  if (res && !h) ph = (hn = make(x, dt, {rows, dim})).data_ptr();
  const mx_opts_t o = options(dev, code, layout);
  const float eps = real(a[3]);
  const int rounding = small(a[5]);
  check(unlocked([&] {
          return mx_rmsnorm_quantize(px, pr, pw, wcode, eps, rows, dim, ph, py, pe, (uint8_t*)ps, (mx_fmt_t)fmt,
                                     (mx_round_t)rounding, &o);
        }), "mx_rmsnorm_quantize");
  PyObject *re = oe ? given(a[9]) : wrap(elems), *rs = os ? given(a[10]) : wrap(scales);
  PyObject* rh = h ? given(a[8]) : hn.defined() ? wrap(hn) : given(Py_None);
  PyObject* r = re && rs && rh ? PyTuple_Pack(3, re, rs, rh) : nullptr;
  Py_XDECREF(re); Py_XDECREF(rs); Py_XDECREF(rh);
  return r;
}

// dy h weight eps dres out workspace
PyObject* rmsnorm_backward(Args a) {
  const at::Tensor &dy = *tensor(a[0], "dy"), &h = *tensor(a[1], "h"), &w = *tensor(a[2], "weight");
  two_dims(h, "h", "[rows, dim]");
  const at::Tensor *dres = tensor(a[4], "dres", true), *out = tensor(a[5], "out", true), *ws = tensor(a[6], "workspace", true);
  const int dev = call_device(h);
  const int64_t rows = h.size(0), dim = h.size(1);
  const auto dt = h.scalar_type();
  void *pd = need(&dy, "dy", dev, dt, {rows, dim}), *ph = need(&h, "h", dev, dt, {rows, dim});
  void *pw = need(&w, "weight", dev, w.scalar_type(), {dim}), *pr = need(dres, "dres", dev, dt, {rows, dim});
  const mx_dtype_t code = float_code(h), wcode = float_code(w);
  at::Tensor space, dh;
  int64_t bytes = (int64_t)mx_rmsnorm_backward_workspace_bytes(rows, dim);
  void* pws;
  if (ws) {
    pws = holds(*ws, "workspace", dev, 0);
    bytes = (int64_t)ws->nbytes();
  } else {
    pws = (space = make(h, at::kByte, {bytes})).data_ptr();
  }
  void* po = out ? need(out, "out", dev, dt, {rows, dim}) : (dh = make(h, dt, {rows, dim})).data_ptr();
  at::Tensor dw = make(h, at::kFloat, {dim});
  const mx_opts_t o = options(dev, code);
  const float eps = real(a[3]);
  float* pdw = (float*)dw.data_ptr();
  check(unlocked([&] {
          return mx_rmsnorm_backward(pd, ph, pw, wcode, eps, pr, rows, dim, po, pdw, &o, pws, (size_t)bytes);
        }), "mx_rmsnorm_backward");
  return pair(out ? given(a[5]) : wrap(dh), wrap(dw));
}

// logits topk score bias groups topk_groups group_score renormalize scale
PyObject* route(Args a) {
  const at::Tensor& x = *tensor(a[0], "logits");
  two_dims(x, "logits", "[tokens, experts]");
  const at::Tensor* bias = tensor(a[3], "bias", true);
  const int dev = call_device(x);
  const int64_t tokens = x.size(0), experts = x.size(1);
  const mx_route_t r = {small(a[1]), small(a[2]), small(a[4]), small(a[5]), small(a[6]), small(a[7]) ? 1 : 0, real(a[8])};
  void *px = need(&x, "logits", dev, x.scalar_type(), {tokens, experts}), *pb = need(bias, "bias", dev, at::kFloat, {experts});
  const int64_t width = r.topk > 0 && r.topk <= 1024 ? r.topk : 0;  // (the library refuses the rest)
  at::Tensor ids = make(x, at::kInt, {tokens, width}), weights = make(x, at::kFloat, {tokens, width});
  const mx_opts_t o = options(dev, float_code(x));
  int32_t* pi = (int32_t*)ids.data_ptr();
  float* pw = (float*)weights.data_ptr();
  check(unlocked([&] { return mx_route(px, (const float*)pb, tokens, experts, &r, pi, pw, &o); }), "mx_route");
  return pair(wrap(ids), wrap(weights));
}

// dweights logits ids score renormalize scale
PyObject* route_backward(Args a) {
  const at::Tensor &dw = *tensor(a[0], "dweights"), &x = *tensor(a[1], "logits"), &ids = *tensor(a[2], "ids");
  two_dims(x, "logits", "[tokens, experts]");
  two_dims(ids, "ids", "[tokens, topk]");
  const int dev = call_device(x);
  const int64_t tokens = x.size(0), experts = x.size(1), topk = ids.size(1);
  const mx_route_t r = {(int32_t)(topk < 1 << 20 ? topk : -1), small(a[3]), 1, 1, MX_GROUP_MAX, small(a[4]) ? 1 : 0, real(a[5])};
  void *pd = need(&dw, "dweights", dev, at::kFloat, {tokens, topk}), *px = need(&x, "logits", dev, x.scalar_type(), {tokens, experts});
  void* pi = need(&ids, "ids", dev, at::kInt, {tokens, topk});
  at::Tensor dx = make(x, x.scalar_type(), {tokens, experts});
  const mx_opts_t o = options(dev, float_code(x));
  void* po = dx.data_ptr();
  check(unlocked([&] {
          return mx_route_backward((const float*)pd, px, (const int32_t*)pi, tokens, experts, &r, po, &o);
        }), "mx_route_backward");
  return wrap(dx);
}

// ids experts align workspace -> offsets counts row_of rows src_of
PyObject* moe_plan(Args a) {
  const at::Tensor& ids = *tensor(a[0], "ids");
  two_dims(ids, "ids", "[tokens, topk]");
  const at::Tensor* ws = tensor(a[3], "workspace", true);
  const int dev = call_device(ids);
  const int64_t tokens = ids.size(0), topk = ids.size(1), experts = integer(a[1]), align = integer(a[2]);
  void* pi = need(&ids, "ids", dev, at::kInt, {tokens, topk});
  const int64_t rows = mx_moe_rows(tokens, topk, experts, align), e = experts > 0 && experts <= 1024 ? experts : 0;
  int64_t bytes = (int64_t)mx_moe_plan_workspace_bytes(tokens, topk, experts);
  at::Tensor space, offsets = make(ids, at::kInt, {e + 1}), counts = make(ids, at::kInt, {e});
  at::Tensor row_of = make(ids, at::kInt, {tokens, topk}), src_of = make(ids, at::kInt, {rows});
  void* pws;
  if (ws) {
    pws = holds(*ws, "workspace", dev, 0);
    bytes = (int64_t)ws->nbytes();
  } else {
    pws = (space = make(ids, at::kByte, {bytes > 0 ? bytes : 1})).data_ptr();
  }
  const mx_opts_t o = options(dev, MX_F32);
  int32_t *p0 = (int32_t*)offsets.data_ptr(), *p1 = (int32_t*)counts.data_ptr(), *p2 = (int32_t*)row_of.data_ptr();
  int32_t* p3 = (int32_t*)src_of.data_ptr();
  check(unlocked([&] {
          return mx_moe_plan((const int32_t*)pi, tokens, topk, experts, align, p0, p1, p2, p3, &o, pws, (size_t)bytes);
        }), "mx_moe_plan");
  PyObject* r = PyTuple_New(5);
  if (!r) return nullptr;
  PyTuple_SET_ITEM(r, 0, wrap(offsets));
  PyTuple_SET_ITEM(r, 1, wrap(counts));
  PyTuple_SET_ITEM(r, 2, wrap(row_of));
  PyTuple_SET_ITEM(r, 3, PyLong_FromLongLong(rows));
  PyTuple_SET_ITEM(r, 4, wrap(src_of));
  return r;
}

struct Plan {
  const int32_t *offsets, *counts, *row_of, *src_of;
  int64_t tokens, topk, experts, rows;
};
Plan plan(PyObject* t, int dev) {
  if (!PyTuple_Check(t) || PyTuple_GET_SIZE(t) != 5) fail(PyExc_TypeError, "plan has to be a MoePlan");
  const at::Tensor &off = *tensor(PyTuple_GET_ITEM(t, 0), "offsets"), &cnt = *tensor(PyTuple_GET_ITEM(t, 1), "counts");
  const at::Tensor &row = *tensor(PyTuple_GET_ITEM(t, 2), "row_of"), *src = tensor(PyTuple_GET_ITEM(t, 4), "src_of", true);
  two_dims(row, "row_of", "[tokens, topk]");
  Plan p;
  p.rows = integer(PyTuple_GET_ITEM(t, 3));
  p.tokens = row.size(0);
  p.topk = row.size(1);
  p.experts = cnt.numel();
  p.offsets = (const int32_t*)need(&off, "offsets", dev, at::kInt, {p.experts + 1});
  p.counts = (const int32_t*)need(&cnt, "counts", dev, at::kInt, {p.experts});
  p.row_of = (const int32_t*)need(&row, "row_of", dev, at::kInt, {p.tokens, p.topk});
  p.src_of = (const int32_t*)need(src, "src_of", dev, at::kInt, {p.rows});
  return p;
}

// elems scales dim fmt plan layout out_elems out_scales
PyObject* moe_gather(Args a) {
  const at::Tensor &e = *tensor(a[0], "elems"), &s = *tensor(a[1], "scales");
  const at::Tensor *oe = tensor(a[6], "out elems", true), *os = tensor(a[7], "out scales", true);
  const int dev = call_device(e), fmt = small(a[3]), layout = small(a[5]);
  const int64_t dim = integer(a[2]);
  const Plan p = plan(a[4], dev);
  if (PyTuple_GET_ITEM(a[4], 4) == Py_None) fail(PyExc_ValueError, "the plan has no src_of");
  void *pe = holds(e, "elems", dev, code_bytes(p.tokens, dim, fmt)), *ps = holds(s, "scales", dev, scale_bytes(p.tokens, dim, layout));
  const int64_t ne = code_bytes(p.rows, dim, fmt), ns = scale_bytes(p.rows, dim, layout);
  at::Tensor ge, gs;
  void* qe = oe ? holds(*oe, "out elems", dev, ne) : (ge = make(e, at::kByte, {ne})).data_ptr();
  void* qs = os ? holds(*os, "out scales", dev, ns) : (gs = make(e, at::kByte, {ns})).data_ptr();
  const mx_opts_t o = options(dev, MX_F32, layout);
  check(unlocked([&] {
          return mx_moe_gather(pe, (const uint8_t*)ps, p.tokens, p.topk, dim, (mx_fmt_t)fmt, p.offsets, p.counts, p.row_of,
                               p.src_of, p.experts, p.rows, qe, (uint8_t*)qs, &o);
        }), "mx_moe_gather");
  return pair(oe ? given(a[6]) : wrap(ge), os ? given(a[7]) : wrap(gs));
}

// y weights plan out
PyObject* moe_combine(Args a) {
  const at::Tensor& y = *tensor(a[0], "y");
  const at::Tensor *w = tensor(a[1], "weights", true), *out = tensor(a[3], "out", true);
  const int dev = call_device(y);
  const Plan p = plan(a[2], dev);
  two_dims(y, "y", "[plan.rows, dim]");
  const int64_t dim = y.size(1);
  const auto dt = y.scalar_type();
  void *py = need(&y, "y", dev, dt, {p.rows, dim}), *pw = need(w, "weights", dev, at::kFloat, {p.tokens, p.topk});
  at::Tensor made;
  void* po = out ? need(out, "out", dev, dt, {p.tokens, dim}) : (made = make(y, dt, {p.tokens, dim})).data_ptr();
  const mx_opts_t o = options(dev, float_code(y));
  check(unlocked([&] {
          return mx_moe_combine(py, (const float*)pw, p.row_of, p.tokens, p.topk, dim, p.rows, po, &o);
        }), "mx_moe_combine");
  return out ? given(a[3]) : wrap(made);
}

// dout y weights plan
PyObject* moe_combine_backward(Args a) {
  const at::Tensor &d = *tensor(a[0], "dout"), *y = tensor(a[1], "y", true), *w = tensor(a[2], "weights", true);
  const int dev = call_device(d);
  const Plan p = plan(a[3], dev);
  two_dims(d, "dout", "[tokens, dim]");
  const int64_t dim = d.size(1);
  const auto dt = d.scalar_type();
  void *pd = need(&d, "dout", dev, dt, {p.tokens, dim}), *py = need(y, "y", dev, dt, {p.rows, dim});
  void* pw = need(w, "weights", dev, at::kFloat, {p.tokens, p.topk});
  at::Tensor dy = make(d, dt, {p.rows, dim}), dw;
  if (y) dw = make(d, at::kFloat, {p.tokens, p.topk});
  const mx_opts_t o = options(dev, float_code(d));
  void* po = dy.data_ptr();
  float* pdw = y ? (float*)dw.data_ptr() : nullptr;
  check(unlocked([&] {
          return mx_moe_combine_backward(pd, py, (const float*)pw, p.offsets, p.counts, p.row_of, p.tokens, p.topk, dim,
                                         p.experts, p.rows, po, pdw, &o);
        }), "mx_moe_combine_backward");
  return pair(wrap(dy), y ? wrap(dw) : given(Py_None));
}

// A sA B sB offsets n0 n1 n2 fmtA fmtB out out_dtype check_status; n0 n1 n2 = rows N K, or M N rows
// EX: wait_cycles drop_fill
template <bool KG, bool EX>
PyObject* gemm_grouped(Args a) {
  const at::Tensor &A = *tensor(a[0], "A"), &sA = *tensor(a[1], "sA"), &B = *tensor(a[2], "B"), &sB = *tensor(a[3], "sB");
  const at::Tensor &off = *tensor(a[4], "offsets"), *out = tensor(a[10], "out", true);
  const int dev = call_device(A), fa = small(a[8]), fb = small(a[9]);
  const int64_t n0 = integer(a[5]), n1 = integer(a[6]), n2 = integer(a[7]), groups = off.numel() - 1;
  // A is [n0, n2]; B [groups * n1, n2], or [n1, n2]
  void *pa = holds(A, "A", dev, code_bytes(n0, n2, fa)), *psa = holds(sA, "sA", dev, scale_bytes(n0, n2, MX_SCALES_SWIZZLED));
  const int64_t brows = KG ? n1 : groups * n1;
  void *pb = holds(B, "B", dev, code_bytes(brows, n2, fb)), *psb = holds(sB, "sB", dev, scale_bytes(brows, n2, MX_SCALES_SWIZZLED));
  const int32_t* po = (const int32_t*)need(&off, "offsets", dev, at::kInt, {groups + 1});
  at::Tensor made;
  if (!out) {
    if (!THPDtype_Check(a[11])) fail(PyExc_TypeError, "out_dtype has to be a torch.dtype");
    const auto dt = reinterpret_cast<THPDtype*>(a[11])->scalar_type;
    float_code(dt);
    made = KG ? make(A, dt, {groups, n0, n1}) : make(A, dt, {n0, n1});
  }
  const at::Tensor& c = out ? *out : made;
  void* pc = KG ? need(&c, "out", dev, c.scalar_type(), {groups, n0, n1}) : need(&c, "out", dev, c.scalar_type(), {n0, n1});
  const mx_dtype_t code = float_code(c);
  const mx_opts_t o = options(dev, MX_F32, MX_SCALES_SWIZZLED, small(a[12]) != 0);
  const int64_t wait = EX ? integer(a[13]) : 0;
  const int64_t d = EX ? integer(a[14]) : -1;
  const int drop = d < -1 || d > 1 << 30 ? -2 : (int)d;  // (-2: the library refuses it)
  const auto call = KG ? mx_gemm_grouped_k_ex : mx_gemm_grouped_ex;
  check(unlocked([&] {
          return call(pa, (const uint8_t*)psa, pb, (const uint8_t*)psb, po, pc, code, groups, n0, n1, n2, (mx_fmt_t)fa,
                      (mx_fmt_t)fb, &o, wait, drop);
        }), KG ? (EX ? "mx_gemm_grouped_k_ex" : "mx_gemm_grouped_k") : (EX ? "mx_gemm_grouped_ex" : "mx_gemm_grouped"));
  return out ? given(a[10]) : wrap(made);
}

// A KvCache: the four tensors [pages, heads, page_size, row bytes], dim, fmt.
mx_kv_t kv_cache(PyObject* t, int* dev) {
  if (!PyTuple_Check(t) || PyTuple_GET_SIZE(t) != 6) fail(PyExc_TypeError, "cache has to be a KvCache");
  const at::Tensor &ke = *tensor(PyTuple_GET_ITEM(t, 0), "k_elems"), &ks = *tensor(PyTuple_GET_ITEM(t, 1), "k_scales");
  const at::Tensor &ve = *tensor(PyTuple_GET_ITEM(t, 2), "v_elems"), &vs = *tensor(PyTuple_GET_ITEM(t, 3), "v_scales");
  if (ke.dim() != 4) fail(PyExc_ValueError, "k_elems has to be [pages, heads, page_size, bytes]");
  *dev = call_device(ke);
  mx_kv_t kv = {};
  kv.pages = ke.size(0);
  kv.heads = ke.size(1);
  kv.page_size = ke.size(2);
  kv.dim = integer(PyTuple_GET_ITEM(t, 4));
  kv.fmt = small(PyTuple_GET_ITEM(t, 5));
  const int bits = mx_fmt_bits((mx_fmt_t)kv.fmt);
  const int64_t dim = kv.dim > 0 && kv.dim < 1 << 24 ? kv.dim : 0;  // (the library refuses the rest)
  const int64_t code = dim * bits / 8, scale = (dim + 127) / 128 * 4;
  kv.k_elems = need(&ke, "k_elems", *dev, at::kByte, {kv.pages, kv.heads, kv.page_size, code});
  kv.k_scales = (uint8_t*)need(&ks, "k_scales", *dev, at::kByte, {kv.pages, kv.heads, kv.page_size, scale});
  kv.v_elems = need(&ve, "v_elems", *dev, at::kByte, {kv.pages, kv.heads, kv.page_size, code});
  kv.v_scales = (uint8_t*)need(&vs, "v_scales", *dev, at::kByte, {kv.pages, kv.heads, kv.page_size, scale});
  return kv;
}
// Rows of heads of tokens that may lie inside a wider tensor: [.., heads, dim] contiguous within a token, the tokens (all
// leading axes in order) evenly spaced.  Their spacing in elements.
int64_t token_stride(const at::Tensor& t, const char* name, int dev, c10::ScalarType dtype, int64_t heads, int64_t dim) {
  const int64_t n = t.dim();
  if (!t.is_cuda() || t.get_device() != dev)
    fail(PyExc_ValueError, std::string(name) + " has to be a tensor on the current CUDA device");
  if (t.scalar_type() != dtype || t.size(n - 2) != heads || t.size(n - 1) != dim)
    fail(PyExc_ValueError, std::string(name) + " has to be " + c10::toString(dtype) + " [.., " + std::to_string(heads) + ", " +
                               std::to_string(dim) + "], not " + describe(t.scalar_type(), t.sizes()));
  const bool rows = (dim < 2 || t.stride(n - 1) == 1) && (heads < 2 || t.stride(n - 2) == dim);
  const bool lead = n < 4 || t.size(0) < 2 || t.size(1) < 2 || t.stride(0) == t.size(1) * t.stride(1);  // (of one token stride(1) says nothing)
  if (!rows || !lead) fail(PyExc_ValueError, std::string(name) + " has to have contiguous heads and evenly spaced tokens");
  if (n == 4 && t.size(1) < 2) return t.size(0) < 2 ? heads * dim : t.stride(0);
  return t.size(n - 3) < 2 ? heads * dim : t.stride(n - 3);
}

// cache k v slots rounding
PyObject* kv_append(Args a) {
  int dev;
  const mx_kv_t kv = kv_cache(a[0], &dev);
  const at::Tensor &k = *tensor(a[1], "k"), &v = *tensor(a[2], "v"), &slots = *tensor(a[3], "slots");
  if (k.dim() != 3 || v.dim() != 3) fail(PyExc_ValueError, "k and v have to be [tokens, heads, dim]");
  const int64_t tokens = k.size(0);
  const mx_dtype_t code = float_code(k);
  const int64_t ks = token_stride(k, "k", dev, k.scalar_type(), kv.heads, kv.dim), vs = token_stride(v, "v", dev, k.scalar_type(), kv.heads, kv.dim);
  if (v.size(0) != tokens) fail(PyExc_ValueError, "k and v have to have the same tokens");
  const int32_t* ps = (const int32_t*)need(&slots, "slots", dev, at::kInt, {tokens});
  const int rounding = small(a[4]);
  const mx_opts_t o = options(dev, code);
  const void *pk = k.data_ptr(), *pv = v.data_ptr();
  check(unlocked([&] { return mx_kv_append(&kv, pk, pv, ks, vs, ps, tokens, (mx_round_t)rounding, &o); }), "mx_kv_append");
  return given(Py_None);
}

// cache slots dtype out_k out_v
PyObject* kv_read(Args a) {
  int dev;
  const mx_kv_t kv = kv_cache(a[0], &dev);
  const at::Tensor &slots = *tensor(a[1], "slots"), *ok = tensor(a[3], "out k", true), *ov = tensor(a[4], "out v", true);
  if (slots.dim() != 1) fail(PyExc_ValueError, "slots has to be [tokens]");
  const int64_t tokens = slots.size(0);
  if (!THPDtype_Check(a[2])) fail(PyExc_TypeError, "dtype has to be a torch.dtype");
  const auto dt = reinterpret_cast<THPDtype*>(a[2])->scalar_type;
  const mx_dtype_t code = float_code(dt);
  const int32_t* ps = (const int32_t*)need(&slots, "slots", dev, at::kInt, {tokens});
  at::Tensor mk, mv;
  void* pk = ok ? need(ok, "out k", dev, dt, {tokens, kv.heads, kv.dim}) : (mk = make(slots, dt, {tokens, kv.heads, kv.dim})).data_ptr();
  void* pv = ov ? need(ov, "out v", dev, dt, {tokens, kv.heads, kv.dim}) : (mv = make(slots, dt, {tokens, kv.heads, kv.dim})).data_ptr();
  const mx_opts_t o = options(dev, code);
  check(unlocked([&] { return mx_kv_read(&kv, ps, tokens, pk, pv, &o); }), "mx_kv_read");
  return pair(ok ? given(a[3]) : wrap(mk), ov ? given(a[4]) : wrap(mv));
}

// q cache table lengths scale window return_lse out workspace
PyObject* kv_attention(Args a) {
  int dev;
  const mx_kv_t kv = kv_cache(a[1], &dev);
  const at::Tensor &q = *tensor(a[0], "q"), &table = *tensor(a[2], "table"), &len = *tensor(a[3], "lengths");
  const at::Tensor *out = tensor(a[7], "out", true), *ws = tensor(a[8], "workspace", true);
  const int64_t n = q.dim();
  if (n != 3 && n != 4) fail(PyExc_ValueError, "q has to be [batch, heads, dim] or [batch, new tokens, heads, dim]");
  two_dims(table, "table", "[batch, pages of a sequence]");
  mx_kv_attention_t t = {};
  t.batch = q.size(0);
  t.new_tokens = n == 4 ? q.size(1) : 1;
  t.q_heads = q.size(n - 2);
  t.max_pages = table.size(1);
  t.window = integer(a[5]);
  const auto dt = q.scalar_type();
  const mx_dtype_t code = float_code(q);
  t.q_stride = token_stride(q, "q", dev, dt, t.q_heads, kv.dim);
  const float natural = kv.dim > 0 ? 1.0f / sqrtf((float)kv.dim) : 0.0f;
  t.scale = a[4] == Py_None ? natural : real(a[4]);
  const int32_t* pt = (const int32_t*)need(&table, "table", dev, at::kInt, {t.batch, t.max_pages});
  const int32_t* pl = (const int32_t*)need(&len, "lengths", dev, at::kInt, {t.batch});
  const int with_lse = PyObject_IsTrue(a[6]);
  if (with_lse < 0) throw Raised();
  at::Tensor made, lse, space;
  if (out) {
    on_device(*out, "out", dev);
    if (out->scalar_type() != dt || out->sizes() != q.sizes())
      fail(PyExc_ValueError, "out has to be " + describe(dt, q.sizes()) + ", not " + describe(out->scalar_type(), out->sizes()));
    const int64_t tokens = t.batch * t.new_tokens, width = t.q_heads * kv.dim, esz = (int64_t)q.element_size();
    const char *qb = (const char*)q.data_ptr(), *ob = (const char*)out->data_ptr();
    if (tokens > 0 && width > 0 && qb < ob + tokens * width * esz && ob < qb + ((tokens - 1) * t.q_stride + width) * esz)
      fail(PyExc_ValueError, "out shares memory with q, which other blocks still read");
  } else {
    made = n == 4 ? make(q, dt, {t.batch, t.new_tokens, t.q_heads, kv.dim}) : make(q, dt, {t.batch, t.q_heads, kv.dim});
  }
  if (with_lse) lse = n == 4 ? make(q, at::kFloat, {t.batch, t.new_tokens, t.q_heads}) : make(q, at::kFloat, {t.batch, t.q_heads});
  int64_t bytes = (int64_t)mx_kv_attention_workspace_bytes(&kv, &t);
  void* pws;
  if (ws) {
    pws = holds(*ws, "workspace", dev, 0);
    bytes = (int64_t)ws->nbytes();
  } else {
    pws = (space = make(q, at::kByte, {bytes > 0 ? bytes : 1})).data_ptr();
  }
  const mx_opts_t o = options(dev, code);
  const void* pq = q.data_ptr();
  void* po = out ? out->data_ptr() : made.data_ptr();
  float* pe = with_lse ? (float*)lse.data_ptr() : nullptr;
  check(unlocked([&] { return mx_kv_attention(&kv, &t, pq, pt, pl, po, pe, &o, pws, (size_t)bytes); }), "mx_kv_attention");
  PyObject* r = out ? given(a[7]) : wrap(made);
  return with_lse ? pair(r, wrap(lse)) : r;
}

// One entry: the argument count, and no C++ exception leaves.
template <PyObject* (*F)(Args), int N>
PyObject* entry(PyObject*, Args args, Py_ssize_t n) {
  if (n != N) {
    PyErr_Format(PyExc_TypeError, "%d arguments, not %zd", N, n);
    return nullptr;
  }
  try {
    return F(args);
  } catch (const Raised&) {
    return nullptr;
  } catch (const c10::OutOfMemoryError& e) {
    PyObject* torch = PyImport_ImportModule("torch");
    PyObject* type = torch ? PyObject_GetAttrString(torch, "OutOfMemoryError") : nullptr;
    PyErr_Clear();
    PyErr_SetString(type ? type : PyExc_MemoryError, e.what());
    Py_XDECREF(type);
    Py_XDECREF(torch);
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}

PyObject* set_error_type(PyObject*, PyObject* type) {
  Py_INCREF(type);
  Py_XDECREF(g_error_type);
  g_error_type = type;
  Py_RETURN_NONE;
}

#define ENTRY(name, fn, n) {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&entry<fn, n>)), METH_FASTCALL, nullptr}
PyMethodDef g_methods[] = {
    ENTRY("rmsnorm_quantize", rmsnorm_quantize, 11), ENTRY("rmsnorm_backward", rmsnorm_backward, 7),
    ENTRY("route", route, 9), ENTRY("route_backward", route_backward, 6),
    ENTRY("moe_plan", moe_plan, 4), ENTRY("moe_gather", moe_gather, 8),
    ENTRY("moe_combine", moe_combine, 4), ENTRY("moe_combine_backward", moe_combine_backward, 4),
    ENTRY("gemm_grouped", (gemm_grouped<false, false>), 13), ENTRY("gemm_grouped_k", (gemm_grouped<true, false>), 13),
    ENTRY("gemm_grouped_ex", (gemm_grouped<false, true>), 15), ENTRY("gemm_grouped_k_ex", (gemm_grouped<true, true>), 15),
    ENTRY("kv_append", kv_append, 5), ENTRY("kv_read", kv_read, 5), ENTRY("kv_attention", kv_attention, 9),
    {"set_error_type", set_error_type, METH_O, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_py_call", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

#ifndef MX_PY_CALL_FOR
#define MX_PY_CALL_FOR ""
#endif
PyMODINIT_FUNC PyInit__py_call(void) {
  PyObject* m = PyModule_Create(&g_module);
  // the interpreter and torch whose C++ interfaces this was compiled against: binding.py compares them
  if (m && PyModule_AddStringConstant(m, "compiled_for", MX_PY_CALL_FOR) < 0) Py_CLEAR(m);
  return m;
}
