// Argument marshalling of the calls that small shapes make often, as a CPython module: output and workspace tensors, device
// pointers, sizes and the current stream, then the C ABI of lrboost.h.  No arithmetic and no state.
//
// Bound: host time.  A layer's forward and backward on a few hundred tokens are four launches of 3 us of host time each; the same
// marshalling through ctypes and torch's Python functions took another 18 us (1.7 us for each of seven tensors, 2-3 us for each
// call's twenty arguments), more than the GPU needs for the kernels.
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/ATen.h>
#include <c10/hip/HIPStream.h>

#include "lrboost.h"

namespace {

struct PyError {};   // a Python exception is set
PyObject* g_lr_error = nullptr;

[[noreturn]] void fail(PyObject* type, const char* what) {
  PyErr_SetString(type, what);
  throw PyError{};
}

// Positional arguments of a call.
struct Args {
  PyObject* const* v;
  Py_ssize_t n;
  Py_ssize_t at = 0;
  PyObject* next() {
    if (at >= n) fail(PyExc_TypeError, "too few arguments");
    return v[at++];
  }
  const at::Tensor& tensor() {
    PyObject* o = next();
    if (!THPVariable_Check(o)) fail(PyExc_TypeError, "tensor expected");
    return THPVariable_Unpack(o);
  }
  at::Tensor optional() { return at < n && v[at] == Py_None ? (at++, at::Tensor()) : tensor(); }
  int64_t integer() {
    PyObject* o = PyNumber_Index(next());
    if (!o) throw PyError{};
    const long long x = PyLong_AsLongLong(o);
    Py_DECREF(o);
    if (x == -1 && PyErr_Occurred()) throw PyError{};
    return x;
  }
  int enumerator() {
    const int64_t x = integer();
    if (x < INT_MIN || x > INT_MAX) fail(PyExc_OverflowError, "integer out of range");
    return (int)x;
  }
  float real() {
    const double x = PyFloat_AsDouble(next());
    if (x == -1.0 && PyErr_Occurred()) throw PyError{};
    return (float)x;
  }
};

int dt_of(const at::Tensor& t) {
  if (t.scalar_type() == at::kFloat) return LR_F32;
  if (t.scalar_type() == at::kBFloat16) return LR_BF16;
  fail(g_lr_error, "unsupported dtype");
}
at::ScalarType scalar(int dt) { return dt == LR_F32 ? at::kFloat : at::kBFloat16; }
int64_t rows_of(const at::Tensor& t, int dims = 2) {
  if (t.dim() != dims) fail(PyExc_ValueError, "unexpected number of dimensions");
  return t.size(0);
}
int64_t stride_of(const at::Tensor& t) {
  if (t.dim() != 2 || t.stride(1) != 1) fail(PyExc_AssertionError, "row-major 2-D tensor expected");
  return t.stride(0);
}
// The row stride of t, passed for the others too (of a single row any will do; beside a dense t, dense others of as many elements are the
// same rows in any shape).
int64_t stride_of_all(const at::Tensor& t, std::initializer_list<const at::Tensor*> others) {
  const int64_t ld = stride_of(t);
  for (const at::Tensor* o : others) {
    if ((ld == t.size(1) || t.size(0) <= 1) && o->is_contiguous() && o->numel() == t.numel()) continue;
    if (stride_of(*o) != ld && (t.size(0) > 1 || o->size(0) > 1)) fail(PyExc_AssertionError, "operands with the same row stride expected");
  }
  return ld;
}
int64_t size_of(const at::Tensor& t, int64_t i) {
  if (t.dim() <= i) fail(PyExc_IndexError, "tuple index out of range");
  return t.size(i);
}
void* ptr(const at::Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }
// of an operand that no stride is passed for
void* dense(const at::Tensor& t) {
  if (t.defined() && !t.is_contiguous()) fail(PyExc_AssertionError, "contiguous tensor expected");
  return ptr(t);
}
at::Tensor fresh(at::IntArrayRef sizes, at::ScalarType dt, const at::Tensor& like) {
  return at::empty(sizes, at::TensorOptions().dtype(dt).device(like.device()));
}
// an output that is written with the row stride of t
at::Tensor rows_like(const at::Tensor& t) { return at::empty_strided(t.sizes(), t.strides(), t.options()); }
at::Tensor workspace(size_t bytes, const at::Tensor& like) {
  return fresh({(int64_t)(bytes < 256 ? 256 : bytes)}, at::kByte, like);
}
void* stream() { return (void*)c10::hip::getCurrentHIPStream().stream(); }

// The call itself runs without the interpreter's lock.
template <class F>
void call(const char* what, F&& f) {
  int status;
  Py_BEGIN_ALLOW_THREADS
  status = f();
  Py_END_ALLOW_THREADS
  if (status == LR_OK) return;
  PyErr_Format(g_lr_error, "%s failed: %s", what, lr_status_string(status));
  throw PyError{};
}

template <class... T>
PyObject* tuple(const T&... t) {
  PyObject* out = PyTuple_New(sizeof...(t));
  if (!out) throw PyError{};
  Py_ssize_t i = 0;
  for (const at::Tensor* x : {&t...}) {
    PyObject* o = THPVariable_Wrap(*x);
    if (!o) {
      Py_DECREF(out);
      throw PyError{};
    }
    PyTuple_SET_ITEM(out, i++, o);
  }
  return out;
}
PyObject* wrap(const at::Tensor& t) { return THPVariable_Wrap(t); }

// ---- one bottleneck layer ------------------------------------------------------------------
PyObject* linear_fwd(Args& a) {
  const at::Tensor &x = a.tensor(), &wd = a.tensor(), &wu = a.tensor();
  const int act = a.enumerator(), dt = dt_of(x);
  const int64_t T = rows_of(x), d = x.size(1), r = size_of(wd, 0), n = size_of(wu, 0);
  const at::Tensor z = fresh({T, r}, x.scalar_type(), x), y = fresh({T, n}, x.scalar_type(), x);
  const size_t nb = lr_linear_workspace_bytes(T, d, r, n, dt, 0);
  const at::Tensor ws = workspace(nb, x);
  const int64_t ldx = stride_of(x);
  void *px = ptr(x), *pd = dense(wd), *pu = dense(wu), *pz = ptr(z), *py = ptr(y), *pw = ptr(ws), *st = stream();
  call("lr_linear_fwd", [&] { return lr_linear_fwd(px, ldx, pd, pu, pz, py, n, T, d, r, n, act, dt, pw, nb, st); });
  return tuple(z, y);
}

PyObject* linear_fwd_static(Args& a) {
  const at::Tensor &x = a.tensor(), &wd = a.tensor(), &wu = a.tensor(), &z = a.tensor(), &y = a.tensor();
  const int act = a.enumerator();
  const int64_t T = rows_of(x), d = x.size(1), r = size_of(wd, 0), n = size_of(wu, 0);
  const int64_t zs[] = {T, r}, ys[] = {T, n};
  if (z.sizes() != at::IntArrayRef(zs) || y.sizes() != at::IntArrayRef(ys) || !z.is_contiguous() || !y.is_contiguous())
    fail(PyExc_AssertionError, "contiguous z [T, r] and y [T, d_out] expected");
  const int64_t ldx = stride_of(x);
  const int dt = dt_of(x);
  void *px = ptr(x), *pd = dense(wd), *pu = dense(wu), *pz = ptr(z), *py = ptr(y), *st = stream();
  call("lr_linear_fwd_static", [&] { return lr_linear_fwd_static(px, ldx, pd, pu, pz, py, n, T, d, r, n, act, dt, st); });
  return tuple(z, y);
}

PyObject* linear_bwd(Args& a) {
  const at::Tensor &x = a.tensor(), &wd = a.tensor(), &wu = a.tensor(), &z = a.tensor(), &dy = a.tensor();
  const int act = a.enumerator();
  const int acc = a.enumerator();
  at::Tensor dwd = a.optional(), dwu = a.optional();     // acc: added to
  const int gdt = a.enumerator(), dt = dt_of(x);
  const int64_t T = rows_of(x), d = x.size(1), r = size_of(wd, 0), n = size_of(wu, 0);
  const at::Tensor dx = fresh({T, d}, x.scalar_type(), x);
  if (!acc) {
    dwd = at::empty_like(wd, at::TensorOptions().dtype(scalar(gdt)));
    dwu = at::empty_like(wu, at::TensorOptions().dtype(scalar(gdt)));
  }
  const size_t nb = lr_linear_workspace_bytes(T, d, r, n, dt, 1);
  const at::Tensor ws = workspace(nb, x);
  const int64_t ldx = stride_of(x), lddy = stride_of(dy);
  void *px = ptr(x), *pd = dense(wd), *pu = dense(wu), *pz = dense(z), *py = ptr(dy), *pdx = ptr(dx), *gd = dense(dwd), *gu = dense(dwu),
       *pw = ptr(ws), *st = stream();
  call("lr_linear_bwd", [&] { return lr_linear_bwd(px, ldx, pd, pu, pz, py, lddy, pdx, d, gd, gu, T, d, r, n, act, dt, gdt, acc, pw, nb, st); });
  return tuple(dx, dwd, dwu);
}

// ---- G projections sharing one input ---------------------------------------------------------
PyObject* group_fwd(Args& a) {
  const at::Tensor& x = a.tensor();
  const at::Tensor gamma = a.optional();
  const float eps = a.real();
  const int norm = a.enumerator();
  const at::Tensor &wd = a.tensor(), &wu = a.tensor();
  const int act = a.enumerator(), dt = dt_of(x);
  const int64_t T = rows_of(x), d = x.size(1), G = rows_of(wu, 3), n = wu.size(1), r = wu.size(2);
  const at::Tensor z = fresh({T, G * r}, x.scalar_type(), x), stat = fresh({T}, at::kFloat, x), y = fresh({G, T, n}, x.scalar_type(), x);
  const size_t nb = lr_group_workspace_bytes((int)G, T, d, r, n, dt, 0);
  const at::Tensor ws = workspace(nb, x);
  const int64_t ldx = stride_of(x);
  void *px = ptr(x), *pg = dense(gamma), *pd = dense(wd), *pu = dense(wu), *pz = ptr(z), *ps = dense(stat), *py = ptr(y), *pw = ptr(ws), *st = stream();
  call("lr_group_fwd", [&] {
    return lr_group_fwd(px, ldx, pg, eps, norm, pd, pu, pz, (float*)ps, py, n, T * n, (int)G, T, d, r, n, act, dt, pw, nb, st);
  });
  return tuple(z, stat, y);
}

PyObject* group_bwd(Args& a) {
  const at::Tensor& x = a.tensor();
  const at::Tensor gamma = a.optional();
  const float eps = a.real();
  const int norm = a.enumerator();
  const at::Tensor &wd = a.tensor(), &wu = a.tensor(), &z = a.tensor();
  const at::Tensor stat = a.optional();
  const at::Tensor& dy = a.tensor();
  const int act = a.enumerator();
  const int acc = a.enumerator();
  at::Tensor dgamma = a.optional(), dwd = a.optional(), dwu = a.optional();   // acc: added to
  const int gdt = a.enumerator(), dt = dt_of(x);
  const int64_t T = rows_of(x), d = x.size(1), G = rows_of(wu, 3), n = wu.size(1), r = wu.size(2);
  const at::Tensor dx = fresh({T, d}, x.scalar_type(), x);
  if (!acc) {
    dgamma = fresh({d}, scalar(gdt), x);
    dwd = at::empty_like(wd, at::TensorOptions().dtype(scalar(gdt)));
    dwu = at::empty_like(wu, at::TensorOptions().dtype(scalar(gdt)));
  }
  const size_t nb = lr_group_workspace_bytes((int)G, T, d, r, n, dt, 1);
  const at::Tensor ws = workspace(nb, x);
  const int64_t ldx = stride_of(x);
  void *px = ptr(x), *pg = dense(gamma), *pd = dense(wd), *pu = dense(wu), *pz = dense(z), *ps = dense(stat), *py = dense(dy), *pdx = ptr(dx),
       *gg = dense(dgamma), *gd = dense(dwd), *gu = dense(dwu), *pw = ptr(ws), *st = stream();
  call("lr_group_bwd", [&] {
    return lr_group_bwd(px, ldx, pg, eps, norm, pd, pu, pz, (const float*)ps, py, n, T * n, pdx, d, gg, gd, gu, (int)G, T, d, r, n, act, dt, gdt,
                        acc, pw, nb, st);
  });
  return tuple(dx, dgamma, dwd, dwu);
}

// ---- attention -----------------------------------------------------------------------------
int64_t stride_of_kv(const at::Tensor& k, const at::Tensor& v) {
  const int64_t ldkv = stride_of(k);
  if (ldkv != stride_of(v)) fail(PyExc_AssertionError, "k and v with the same row stride expected");
  return ldkv;
}

PyObject* attention_fwd(Args& a) {
  const at::Tensor &q = a.tensor(), &k = a.tensor(), &v = a.tensor();
  const int64_t B = a.integer(), S = a.integer(), H = a.integer(), Hkv = a.integer(), hd = a.integer();
  const int causal = a.enumerator();
  const int64_t ld = stride_of(q), ldkv = stride_of_kv(k, v);
  const int dt = dt_of(q);
  const at::Tensor o = rows_like(q), lse = fresh({B, H, S}, at::kFloat, q);
  void *pq = ptr(q), *pk = ptr(k), *pv = ptr(v), *po = ptr(o), *pl = dense(lse), *st = stream();
  call("lr_attention_gqa_fwd", [&] { return lr_attention_gqa_fwd(pq, pk, pv, po, (float*)pl, ld, ldkv, B, S, H, Hkv, hd, causal, dt, st); });
  return tuple(o, lse);
}

PyObject* attention_bwd(Args& a) {
  const at::Tensor &q = a.tensor(), &k = a.tensor(), &v = a.tensor(), &o = a.tensor(), &dout = a.tensor(), &lse = a.tensor();
  const int64_t B = a.integer(), S = a.integer(), H = a.integer(), Hkv = a.integer(), hd = a.integer();
  const int causal = a.enumerator();
  const int64_t ld = stride_of_all(q, {&o, &dout}), ldkv = stride_of_kv(k, v);
  const at::Tensor dq = rows_like(q), dk = rows_like(k), dv = rows_like(k);
  const at::Tensor ws = workspace(lr_attention_gqa_bwd_workspace_bytes(B, S, H, Hkv, hd), q);
  const size_t nb = (size_t)ws.numel();
  const int dt = dt_of(q);
  void *pq = ptr(q), *pk = ptr(k), *pv = ptr(v), *po = ptr(o), *pdo = ptr(dout), *pl = dense(lse), *gq = ptr(dq), *gk = ptr(dk), *gv = ptr(dv),
       *pw = ptr(ws), *st = stream();
  call("lr_attention_gqa_bwd", [&] {
    return lr_attention_gqa_bwd(pq, pk, pv, po, pdo, (const float*)pl, gq, gk, gv, ld, ldkv, B, S, H, Hkv, hd, causal, dt, pw, nb, st);
  });
  return tuple(dq, dk, dv);
}

// ---- standalone memory-bound kernels ---------------------------------------------------------
PyObject* rms_stat(Args& a) {
  const at::Tensor& x = a.tensor();
  const int64_t T = rows_of(x), d = x.size(1);
  const at::Tensor stat = fresh({T}, at::kFloat, x);
  const int64_t ldx = stride_of(x);
  const int dt = dt_of(x);
  void *px = ptr(x), *ps = dense(stat), *st = stream();
  call("lr_rms_stat", [&] { return lr_rms_stat(px, ldx, (float*)ps, T, d, dt, st); });
  return wrap(stat);
}

PyObject* rmsnorm_apply(Args& a) {
  const at::Tensor &x = a.tensor(), &gamma = a.tensor(), &stat = a.tensor();
  const float eps = a.real();
  const int64_t T = rows_of(x), d = x.size(1);
  const at::Tensor out = at::empty_like(x);
  const int64_t ldx = stride_of(x);
  const int dt = dt_of(x);
  void *px = ptr(x), *pg = dense(gamma), *ps = dense(stat), *po = ptr(out), *st = stream();
  call("lr_rmsnorm_apply", [&] { return lr_rmsnorm_apply(px, ldx, pg, (const float*)ps, eps, po, d, T, d, dt, st); });
  return wrap(out);
}

PyObject* rmsnorm_bwd(Args& a) {
  const at::Tensor &x = a.tensor(), &gamma = a.tensor(), &stat = a.tensor();
  const float eps = a.real();
  const at::Tensor& dxhat = a.tensor();
  const at::Tensor dres = a.optional();
  const int64_t T = rows_of(x), d = x.size(1);
  const at::Tensor dx = at::empty_like(x);
  const int64_t parts = lr_rmsnorm_bwd_parts(T);
  const at::Tensor part = fresh({parts < 1 ? 1 : parts, d}, at::kFloat, x);
  const int64_t ldx = stride_of(x), lddxh = stride_of(dxhat), lddres = dres.defined() ? stride_of(dres) : 0;
  const int dt = dt_of(x);
  void *px = ptr(x), *pg = dense(gamma), *ps = dense(stat), *ph = ptr(dxhat), *pr = ptr(dres), *pdx = ptr(dx), *pp = ptr(part), *st = stream();
  call("lr_rmsnorm_bwd", [&] { return lr_rmsnorm_bwd(px, ldx, pg, (const float*)ps, eps, ph, lddxh, pr, lddres, pdx, d, (float*)pp, T, d, dt, st); });
  return tuple(dx, part);
}

PyObject* swiglu_fwd(Args& a) {
  const at::Tensor &g = a.tensor(), &u = a.tensor();
  const int64_t T = rows_of(g), f = g.size(1);
  const int64_t ld = stride_of_all(g, {&u});
  const at::Tensor m = rows_like(g);
  const int dt = dt_of(g);
  void *pg = ptr(g), *pu = ptr(u), *pm = ptr(m), *st = stream();
  call("lr_swiglu_fwd", [&] { return lr_swiglu_fwd(pg, pu, pm, ld, T, f, dt, st); });
  return wrap(m);
}

PyObject* swiglu_bwd(Args& a) {
  const at::Tensor &g = a.tensor(), &u = a.tensor(), &dm = a.tensor();
  const int64_t T = rows_of(g), f = g.size(1);
  const int64_t ld = stride_of_all(g, {&u, &dm});
  const at::Tensor dg = rows_like(g), du = rows_like(u);
  const int dt = dt_of(g);
  void *pg = ptr(g), *pu = ptr(u), *pm = ptr(dm), *gg = ptr(dg), *gu = ptr(du), *st = stream();
  call("lr_swiglu_bwd", [&] { return lr_swiglu_bwd(pg, pu, pm, gg, gu, ld, T, f, dt, st); });
  return tuple(dg, du);
}

// ---- rotary positions, paged cache -----------------------------------------------------------
// Launches go to the current stream, which is one of the current device's: operands are there too.
void on_current_device(std::initializer_list<const at::Tensor*> ts) {
  for (const at::Tensor* t : ts)
    if (t->defined() && (!t->is_cuda() || t->get_device() != c10::hip::current_device())) fail(g_lr_error, "tensors on the current GPU expected");
}
const int32_t* indices(const at::Tensor& t, int64_t n) {
  if (t.defined() && t.scalar_type() != at::kInt) fail(g_lr_error, "int32 indices expected");
  if (t.defined() && (t.dim() != 1 || t.size(0) != n)) fail(PyExc_ValueError, "unexpected number of indices");
  return (const int32_t*)dense(t);
}
void same_type(const at::Tensor& a, std::initializer_list<const at::Tensor*> others) {
  for (const at::Tensor* t : others)
    if (t->defined() && t->scalar_type() != a.scalar_type()) fail(g_lr_error, "operands of one type expected");
}
// The row stride of T rows that are at least as wide (of a single row any will do).
int64_t rows_as_wide(const at::Tensor& t, int64_t T, int64_t width) {
  if (t.dim() != 2 || t.size(0) != T || t.size(1) < width) fail(PyExc_ValueError, "unexpected shape");
  const int64_t ld = stride_of(t);
  return T > 1 ? ld : width;
}
// rows and pairs of the tables
void tables_of(const at::Tensor& cos, const at::Tensor& sin, int64_t& rows, int64_t& half) {
  if (cos.scalar_type() != at::kFloat || sin.scalar_type() != at::kFloat) fail(g_lr_error, "fp32 tables expected");
  rows = rows_of(cos);
  half = cos.size(1);
  if (sin.sizes() != cos.sizes()) fail(PyExc_ValueError, "tables of the same shape expected");
}

PyObject* rope_table(Args& a) {
  const int64_t n = a.integer(), rot = a.integer(), first = a.integer();
  double x[6];
  for (double& v : x) {
    v = PyFloat_AsDouble(a.next());
    if (v == -1.0 && PyErr_Occurred()) throw PyError{};
  }
  const auto options = at::TensorOptions().dtype(at::kFloat).device(at::kCUDA, c10::hip::current_device());
  const int64_t sizes[] = {n < 0 ? 0 : n, rot < 0 ? 0 : rot / 2};
  const at::Tensor cos = at::empty(sizes, options), sin = at::empty(sizes, options);
  void *pc = ptr(cos), *ps = ptr(sin), *st = stream();
  call("lr_rope_table", [&] { return lr_rope_table((float*)pc, (float*)ps, n, rot, first, x[0], x[1], x[2], x[3], x[4], x[5], st); });
  return tuple(cos, sin);
}

PyObject* rope_at(Args& a) {
  const at::Tensor &x = a.tensor(), &cos = a.tensor(), &sin = a.tensor();
  const int64_t H = a.integer(), hd = a.integer();
  const at::Tensor pos = a.optional();
  const int inter = a.enumerator(), inverse = a.enumerator();
  at::Tensor out = a.optional();
  const int64_t T = rows_of(x);
  const int dt = dt_of(x);
  int64_t rows, half;
  tables_of(cos, sin, rows, half);
  const int32_t* pp = indices(pos, T);
  const int64_t ldx = rows_as_wide(x, T, H * hd);
  if (!out.defined()) out = fresh({T, H * hd}, x.scalar_type(), x);
  same_type(x, {&out});
  const int64_t ldo = rows_as_wide(out, T, H * hd);
  on_current_device({&x, &cos, &sin, &pos, &out});
  void *px = ptr(x), *pc = dense(cos), *ps = dense(sin), *po = ptr(out), *st = stream();
  call("lr_rope_at", [&] { return lr_rope_at(px, ldx, po, ldo, pp, (float*)pc, (float*)ps, rows, T, H, hd, 2 * half, inter, inverse, dt, st); });
  return wrap(out);
}

// k, v [pages, page size, heads, hd], page_table [batch, columns], cu_q [batch + 1], kv_len [batch]
struct CacheTensors {
  const at::Tensor &k, &v, &table, &cu, &len;
  explicit CacheTensors(Args& a) : k(a.tensor()), v(a.tensor()), table(a.tensor()), cu(a.tensor()), len(a.tensor()) {}
  lr_kv_cache view() const {
    if (k.dim() != 4 || v.sizes() != k.sizes() || table.dim() != 2) fail(PyExc_ValueError, "unexpected shape of the cache or its page table");
    if (k.scalar_type() != at::kBFloat16 || v.scalar_type() != at::kBFloat16) fail(g_lr_error, "a bf16 cache expected");
    bool alike = k.stride(3) == 1 && v.stride(3) == 1;
    for (int i = 0; i < 3; i++) alike &= k.size(i) <= 1 || v.stride(i) == k.stride(i);
    if (!alike) fail(PyExc_AssertionError, "caches with the same strides and contiguous heads expected");
    if (table.scalar_type() != at::kInt) fail(g_lr_error, "int32 indices expected");
    if (table.size(1) > 1 && table.stride(1) != 1) fail(PyExc_AssertionError, "row-major page table expected");
    const int64_t batch = table.size(0), cols = table.size(1);
    lr_kv_cache c;
    c.k = ptr(k); c.v = ptr(v);
    c.n_pages = k.size(0); c.page_size = k.size(1); c.n_kv_heads = k.size(2); c.head_dim = k.size(3);
    const auto stride = [&](int i) { return k.size(i) > 1 ? k.stride(i) : c.head_dim; };      // (of one page, token or head any will do)
    c.page_stride = stride(0); c.token_stride = stride(1); c.head_stride = stride(2);
    c.page_table = (const int32_t*)ptr(table);
    c.batch = batch; c.max_pages = cols;
    c.table_ld = batch > 1 ? table.stride(0) : cols;
    c.cu_q = indices(cu, batch + 1);
    c.kv_len = indices(len, batch);
    return c;
  }
};

PyObject* kv_append(Args& a) {
  const at::Tensor &k = a.tensor(), &v = a.tensor();
  const CacheTensors ct(a);
  const at::Tensor cos = a.optional(), sin = a.optional();
  const int inter = a.enumerator();
  const at::Tensor q = a.optional();
  const int64_t H = a.integer();
  at::Tensor q_out = a.optional();
  const lr_kv_cache c = ct.view();
  const int64_t T = rows_of(k);
  const int dt = dt_of(k);
  int64_t rows = 0, half = 0, ldq = 0, ldqo = 0;
  if (cos.defined() != sin.defined()) fail(PyExc_ValueError, "both tables or neither expected");
  if (cos.defined()) tables_of(cos, sin, rows, half);
  if (cos.defined() && half == 0) fail(PyExc_ValueError, "tables without columns");
  const int64_t ldk = rows_as_wide(k, T, c.n_kv_heads * c.head_dim), ldv = rows_as_wide(v, T, c.n_kv_heads * c.head_dim);
  if (q.defined()) {
    ldq = rows_as_wide(q, T, H * c.head_dim);
    if (!q_out.defined()) q_out = fresh({T, H * c.head_dim}, q.scalar_type(), q);
    ldqo = rows_as_wide(q_out, T, H * c.head_dim);
  }
  same_type(k, {&v, &q, &q_out});
  on_current_device({&k, &v, &ct.k, &ct.v, &ct.table, &ct.cu, &ct.len, &cos, &sin, &q, &q_out});
  void *pk = ptr(k), *pv = ptr(v), *pc = dense(cos), *ps = dense(sin), *pq = ptr(q), *po = ptr(q_out), *st = stream();
  call("lr_kv_append", [&] {
    return lr_kv_append(&c, pk, ldk, pv, ldv, pq, ldq, po, ldqo, T, H, (float*)pc, (float*)ps, rows, 2 * half, inter, dt, st);
  });
  if (!q_out.defined()) Py_RETURN_NONE;
  return wrap(q_out);
}

PyObject* attention_paged_fwd(Args& a) {
  const at::Tensor& q = a.tensor();
  const CacheTensors ct(a);
  const int64_t H = a.integer();
  const float scale = a.real();
  const int causal = a.enumerator();
  at::Tensor o = a.optional(), lse = a.optional(), ws = a.optional();
  const lr_kv_cache c = ct.view();
  const int64_t T = rows_of(q);
  const int dt = dt_of(q);
  const int64_t ldq = rows_as_wide(q, T, H * c.head_dim);
  if (!o.defined()) o = fresh({T, H * c.head_dim}, q.scalar_type(), q);
  const int64_t ldo = rows_as_wide(o, T, H * c.head_dim);
  same_type(q, {&o});
  if (!lse.defined()) lse = fresh({T, H}, at::kFloat, q);
  if (lse.scalar_type() != at::kFloat || lse.dim() != 2 || lse.size(0) != T || lse.size(1) != H) fail(PyExc_ValueError, "lse [T, H] fp32 expected");
  on_current_device({&q, &ct.k, &ct.v, &ct.table, &ct.cu, &ct.len, &o, &lse, &ws});
  if (!ws.defined()) ws = workspace(lr_attention_paged_workspace_bytes(&c, T, H), q);
  const size_t nb = ws.numel() * ws.element_size();
  void *pq = ptr(q), *po = ptr(o), *pl = dense(lse), *pw = dense(ws), *st = stream();
  call("lr_attention_paged_fwd", [&] { return lr_attention_paged_fwd(&c, pq, ldq, po, ldo, (float*)pl, T, H, scale, causal, dt, pw, nb, st); });
  return tuple(o, lse);
}

// No C++ exception leaves an entry; torch's own become the Python exceptions that they are elsewhere (out of memory, a device's error,
// an interpreter's exception that crossed torch).
template <PyObject* (*F)(Args&)>
PyObject* entry(PyObject*, PyObject* const* v, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  try {
    Args a{v, n};
    return F(a);
  } catch (const PyError&) {
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

PyObject* set_error(PyObject*, PyObject* type) {
  Py_INCREF(type);
  Py_XSETREF(g_lr_error, type);
  Py_RETURN_NONE;
}

#define ENTRY(f) {#f, (PyCFunction)(void (*)(void))(&entry<f>), METH_FASTCALL, nullptr}
PyMethodDef g_methods[] = {
    ENTRY(linear_fwd), ENTRY(linear_fwd_static), ENTRY(linear_bwd), ENTRY(group_fwd), ENTRY(group_bwd), ENTRY(attention_fwd), ENTRY(attention_bwd),
    ENTRY(rope_table), ENTRY(rope_at), ENTRY(kv_append), ENTRY(attention_paged_fwd), ENTRY(rms_stat), ENTRY(rmsnorm_apply), ENTRY(rmsnorm_bwd), ENTRY(swiglu_fwd), ENTRY(swiglu_bwd),
    {"set_error", set_error, METH_O, "the exception type of failed calls"}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal(void) {
  PyObject* m = PyModule_Create(&g_module);
  if (m) {
    Py_INCREF(PyExc_RuntimeError);
    g_lr_error = PyExc_RuntimeError;
  }
  return m;
}
