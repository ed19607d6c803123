// Python entry points of the sequence operators (the module _seq, which seq.py
// wraps): checks torch tensors against each other, allocates results and
// scratch from torch's allocator and makes the C ABI's call on the current
// stream of the tensors' device.  A call of the smallest sizes takes the GPU 3
// us; through ctypes its marshalling took the host 11 to 17, here 4 to 5.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <string>
#include <vector>

#include <ATen/core/LegacyTypeDispatch.h>
#include <ATen/core/Tensor.h>
#include <ATen/ops/empty_cuda_dispatch.h>
#include <c10/core/DeviceGuard.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "seq_ops.h"

namespace {

using at::IntArrayRef;
using at::ScalarType;
using at::Tensor;
using Sizes = std::initializer_list<int64_t>;

[[noreturn]] void raise(PyObject* type, const std::string& s) {
  PyErr_SetString(type, s.c_str());
  throw python_error();
}
[[noreturn]] void value_error(const std::string& s) { raise(PyExc_ValueError, s); }
[[noreturn]] void type_error(const std::string& s) { raise(PyExc_TypeError, s); }

std::string text(IntArrayRef v) {
  std::string s = "[";
  for (size_t i = 0; i < v.size(); ++i) s += (i ? ", " : "") + std::to_string(v[i]);
  return s + "]";
}
const char* type_name(ScalarType t) {
  return t == at::kFloat ? "float32" : t == at::kBFloat16 ? "bfloat16" : t == at::kInt ? "int32" : c10::toString(t);
}

// A status of the C ABI as the framework's exception.
[[noreturn]] void conv_error(int status, const char* call) {
  PyObject* mod = PyImport_ImportModule("paper_2101_09808_amd.conv");
  PyObject* cls = mod ? PyObject_GetAttrString(mod, "ConvError") : nullptr;
  PyObject* args = cls ? Py_BuildValue("(is)", status, call) : nullptr;
  if (args) PyErr_SetObject(cls, args);
  Py_XDECREF(args), Py_XDECREF(cls), Py_XDECREF(mod);
  throw python_error();
}

const Tensor& tensor(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) type_error(std::string(name) + " must be a torch tensor");
  return THPVariable_Unpack(o);
}

// The tensor that sets a call's type, extents and device.
const Tensor& lead(PyObject* o, const char* name, int64_t rank) {
  const Tensor& t = tensor(o, name);
  if (!t.is_cuda()) value_error(std::string(name) + " must be a GPU tensor (the library has no CPU path)");
  if (t.scalar_type() != at::kFloat && t.scalar_type() != at::kBFloat16)
    type_error(std::string(name) + " must be float32 or bfloat16, got " + type_name(t.scalar_type()));
  if (t.dim() != rank)
    value_error(std::string(name) + " must have " + std::to_string(rank) + " dimensions, got " + text(t.sizes()));
  if (t.numel() == 0) value_error(std::string(name) + " is empty: " + text(t.sizes()));
  for (const int64_t v : t.sizes())
    if (v > INT32_MAX) conv_error(CONV_ERANGE, name);
  return t;
}

// Whether a tensor has a byte in [lo, hi): its whole span first, then, if that
// meets it, slice by slice, since a slice of a larger tensor spans what is not its own.
bool meets(const char* p, const Tensor& t, int64_t dim, const char* lo, const char* hi) {
  const int64_t es = int64_t(t.element_size());
  int64_t span = 1, numel = 1;
  for (int64_t k = dim; k < t.dim(); ++k) span += (t.size(k) - 1) * t.stride(k), numel *= t.size(k);
  if (p >= hi || p + span * es <= lo) return false;
  if (numel >= span) return true;
  for (int64_t i = 0; i < t.size(dim); ++i)
    if (meets(p + i * t.stride(dim) * es, t, dim + 1, lo, hi)) return true;
  return false;
}
bool meets(const Tensor& t, const Tensor& dense) {
  if (t.numel() == 0 || dense.numel() == 0) return false;
  const char* lo = static_cast<const char*>(dense.data_ptr());
  return meets(static_cast<const char*>(t.data_ptr()), t, 0, lo, lo + dense.nbytes());
}

struct Call {
  struct Given {
    const Tensor* t;
    const char* name;
  };
  mutable Given given[16];  // the inputs (no call has more)
  mutable int inputs = 0;
  const Tensor& like;
  c10::OptionalDeviceGuard guard;
  at::AutoDispatchBelowADInplaceOrView below;  // (results are plain tensors)
  void* stream;

  Call(const Tensor& t, const char* name)
      : like(t), guard(t.device()), stream(c10::hip::getCurrentHIPStream(t.device().index()).stream()) {
    given[inputs++] = {&t, name};
  }

  ScalarType type() const { return like.scalar_type(); }

  const Tensor& fits(PyObject* o, const char* name, IntArrayRef sizes, ScalarType t) const {
    const Tensor& x = tensor(o, name);
    if (x.scalar_type() != t)
      type_error(std::string(name) + " must be " + type_name(t) + ", got " + type_name(x.scalar_type()));
    if (x.sizes() != sizes) value_error(std::string(name) + " must be " + text(sizes) + ", got " + text(x.sizes()));
    if (x.device() != like.device())
      value_error(std::string(name) + " must be on " + like.device().str() + ", is on " + x.device().str());
    return x;
  }
  const Tensor& check(PyObject* o, const char* name, IntArrayRef sizes, ScalarType t) const {
    const Tensor& x = fits(o, name, sizes, t);
    TORCH_INTERNAL_ASSERT(inputs < 16);
    given[inputs++] = {&x, name};
    return x;
  }
  // The length innermost, of stride 1.
  const Tensor& seq(PyObject* o, const char* name, IntArrayRef sizes, ScalarType t) const {
    const Tensor& x = check(o, name, sizes, t);
    if (x.stride(-1) != 1 && sizes.back() > 1)
      value_error(std::string(name) + " must have stride 1 along the length, has strides " + text(x.strides()));
    return x;
  }
  const Tensor& dense(PyObject* o, const char* name, IntArrayRef sizes, ScalarType t) const {
    const Tensor& x = check(o, name, sizes, t);
    if (!x.is_contiguous()) value_error(std::string(name) + " must be contiguous");
    return x;
  }
  template <typename P = const float>
  P* opt(PyObject* o, const char* name, Sizes sizes, ScalarType t = at::kFloat) const {
    return o == Py_None ? nullptr : static_cast<P*>(dense(o, name, sizes, t).data_ptr());
  }
  Tensor empty(IntArrayRef sizes, ScalarType t) const {
    // (at::empty without its way through the dispatcher: a backward scan has ten
    // results)
    return at::cuda::empty(sizes, at::TensorOptions().dtype(t).device(like.device()));
  }
  // A caller's tensor that the call writes, after all inputs have been checked: it
  // may share memory with none of them (`same`: but be that one).
  const Tensor& written(PyObject* o, const char* name, IntArrayRef sizes, ScalarType t,
                        const Tensor* same = nullptr) const {
    const Tensor& x = fits(o, name, sizes, t);
    if (!x.is_contiguous()) value_error(std::string(name) + " must be contiguous");
    apart(x, name, same);
    touch(x);
    return x;
  }
  // What autograd has saved of it is no longer what it was: a backward pass that
  // needs it raises.
  static void touch(const Tensor& x) {
    if (!x.is_inference()) x.unsafeGetTensorImpl()->bump_version();
  }
  void apart(const Tensor& x, const char* name, const Tensor* same) const {
    for (int i = 0; i < inputs; ++i) {
      const Tensor& in = *given[i].t;
      if (same && &in == same && in.data_ptr() == x.data_ptr()) continue;
      if (meets(in, x)) value_error(std::string(name) + " overlaps " + given[i].name);
    }
  }
  Tensor out(PyObject* o, IntArrayRef sizes, ScalarType t) const {
    return o == Py_None ? empty(sizes, t) : written(o, "out", sizes, t);
  }
  // The state after a token: `o`, or in the place of `state`; `out` is apart from it.
  void* new_state(PyObject* o, const Tensor& state, const Tensor& out) const {
    const Tensor* to = &state;
    if (o == Py_None)
      apart(state, "state", &state), touch(state);
    else
      to = &written(o, "new_state", state.sizes(), state.scalar_type(), &state);
    if (meets(out, *to)) value_error(std::string("out overlaps ") + (o == Py_None ? "state" : "new_state"));
    return to->data_ptr();
  }

  template <typename P>
  void run(const char* name, int (*f)(const P*, void*), const P& p) const {
    if (const int rc = f(&p, stream)) conv_error(rc, name);
  }
  template <typename P>
  void run(const char* name, int (*f)(const P*, void*), P& p, int64_t (*size)(const P*)) const {
    const int64_t bytes = size(&p);
    if (bytes < 0) conv_error(int(bytes), name);
    Tensor scratch;  // (freed on the call's stream: reused after it)
    if (bytes > 0) {
      scratch = empty({bytes}, at::kByte);
      p.workspace = scratch.data_ptr();
      p.workspace_bytes = bytes;
    }
    run(name, f, p);
  }
};

int32_t dtype_of(ScalarType t) { return t == at::kFloat ? CONV_DTYPE_F32 : CONV_DTYPE_BF16; }

PyObject* wrap(const Tensor& t) {
  if (!t.defined()) Py_RETURN_NONE;
  return THPVariable_Wrap(t);
}
PyObject* wrap(std::initializer_list<Tensor> ts) {
  PyObject* r = PyTuple_New(Py_ssize_t(ts.size()));
  if (!r) throw python_error();
  Py_ssize_t i = 0;
  for (const Tensor& t : ts) PyTuple_SET_ITEM(r, i++, wrap(t));
  return r;
}

bool flag(PyObject* o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw python_error();
  return v;
}

void need(Py_ssize_t n, Py_ssize_t want) {
  if (n != want) type_error("expected " + std::to_string(want) + " arguments");
}

// --------------------------------------------------------- causal convolution

int32_t activation(PyObject* o) {
  if (o == Py_None) return SEQ_ACT_NONE;
  if (PyUnicode_Check(o) && PyUnicode_CompareWithASCIIString(o, "silu") == 0) return SEQ_ACT_SILU;
  value_error("activation must be None or 'silu'");
}

// x, weight, bias, activation, initial_state, lengths
seq_conv_t conv_args(const Call& c, const Tensor& x, PyObject* weight, PyObject* bias, PyObject* act, PyObject* init,
                     PyObject* lengths, const char* init_name) {
  const int64_t N = x.size(0), D = x.size(1);
  const Tensor& w = tensor(weight, "weight");
  if (w.dim() != 2 || w.size(1) < 1 || w.size(1) > SEQ_CONV_MAX_TAPS)
    value_error("weight must be [D, R] with R of 1 to " + std::to_string(SEQ_CONV_MAX_TAPS) + ", got " +
                text(w.sizes()));
  const int64_t R = w.size(1);
  seq_conv_t p = {};
  p.N = int32_t(N), p.D = int32_t(D), p.L = x.dim() == 3 ? int32_t(x.size(2)) : 1, p.R = int32_t(R);
  p.dtype = dtype_of(c.type()), p.activation = activation(act);
  p.x = x.data_ptr(), p.x_n = x.stride(0), p.x_d = x.stride(1);
  p.weight = static_cast<const float*>(c.dense(weight, "weight", {D, R}, at::kFloat).data_ptr());
  p.bias = c.opt(bias, "bias", {D});
  p.initial_state = c.opt<const void>(init, init_name, {N, D, R - 1}, c.type());
  p.lengths = c.opt<const int32_t>(lengths, "lengths", {N}, at::kInt);
  return p;
}

// x, weight, bias, activation, initial_state, lengths, return_final_state, out
PyObject* conv_fwd(PyObject* const* a) {
  const Tensor& x = lead(a[0], "x", 3);
  const Call c(x, "x");
  c.seq(a[0], "x", x.sizes(), c.type());
  seq_conv_t p = conv_args(c, x, a[1], a[2], a[3], a[4], a[5], "initial_state");
  const Tensor out = c.out(a[7], x.sizes(), c.type());
  p.out = out.data_ptr();
  if (!flag(a[6])) {
    c.run("causal_conv_fwd", seq_causal_conv_fwd, p);
    return wrap(out);
  }
  const Tensor fin = c.empty({p.N, p.D, p.R - 1}, c.type());
  p.final_state = fin.data_ptr();
  c.run("causal_conv_fwd", seq_causal_conv_fwd, p);
  return wrap({out, fin});
}

// dout, x, weight, bias, activation, initial_state, lengths, dfinal_state
PyObject* conv_bwd(PyObject* const* a) {
  const Tensor& x = lead(a[1], "x", 3);
  const Call c(x, "x");
  c.seq(a[1], "x", x.sizes(), c.type());
  seq_conv_t p = conv_args(c, x, a[2], a[3], a[4], a[5], a[6], "initial_state");
  const Tensor& dout = c.seq(a[0], "dout", x.sizes(), c.type());
  p.dout = dout.data_ptr(), p.dout_n = dout.stride(0), p.dout_d = dout.stride(1);
  p.dfinal_state = c.opt<const void>(a[7], "dfinal_state", {p.N, p.D, p.R - 1}, c.type());
  const Tensor dx = c.empty(x.sizes(), c.type()), dw = c.empty({p.D, p.R}, at::kFloat);
  Tensor db, di;
  p.dx = dx.data_ptr(), p.dweight = static_cast<float*>(dw.data_ptr());
  if (p.bias) db = c.empty({p.D}, at::kFloat), p.dbias = static_cast<float*>(db.data_ptr());
  if (a[5] != Py_None) di = c.empty({p.N, p.D, p.R - 1}, c.type()), p.dinitial_state = di.data_ptr();
  c.run("causal_conv_bwd", seq_causal_conv_bwd, p, seq_causal_conv_bwd_workspace);
  return wrap({dx, dw, db, di});
}

// x, state, weight, bias, activation, new_state, out
PyObject* conv_step(PyObject* const* a) {
  const Tensor& x = lead(a[0], "x", 2);
  const Call c(x, "x");
  tensor(a[1], "state");
  seq_conv_t p = conv_args(c, x, a[2], a[3], a[4], a[1], Py_None, "state");
  const Tensor out = c.out(a[6], x.sizes(), c.type());
  p.out = out.data_ptr();
  p.final_state = c.new_state(a[5], tensor(a[1], "state"), out);
  c.run("causal_conv_step", seq_causal_conv_step, p);
  return wrap(out);
}

// -------------------------------------------------------------- selective scan

// u, delta, A, B, C, D, z, delta_bias, delta_softplus, lengths
seq_scan_t scan_args(const Call& c, const Tensor& u, PyObject* delta, PyObject* A, PyObject* B, PyObject* C,
                     PyObject* D, PyObject* z, PyObject* bias, PyObject* softplus, PyObject* lengths) {
  const int64_t N = u.size(0), Dn = u.size(1);
  const bool many = u.dim() == 3;
  const Tensor &At = tensor(A, "A"), &Bt = tensor(B, "B");
  if (At.dim() != 2 || At.size(1) < 1 || At.size(1) > SEQ_SCAN_MAX_STATE)
    value_error("A must be [D, S] with S of 1 to " + std::to_string(SEQ_SCAN_MAX_STATE) + ", got " + text(At.sizes()));
  const int64_t S = At.size(1);
  if (Bt.dim() != u.dim() + 1)
    value_error(std::string("B must be [N, G, S") + (many ? ", L]" : "]") + ", got " + text(Bt.sizes()));
  const int64_t G = Bt.size(1);
  if (G < 1 || Dn % G)
    value_error(std::to_string(Dn) + " channels do not divide into " + std::to_string(G) + " groups");
  const int64_t L = many ? u.size(2) : 1, bs[4] = {N, G, S, L};
  const IntArrayRef bsize(bs, many ? 4 : 3);
  const auto get = [&](PyObject* o, const char* name, IntArrayRef sizes) -> const Tensor& {
    return many ? c.seq(o, name, sizes, c.type()) : c.check(o, name, sizes, c.type());
  };
  seq_scan_t p = {};
  p.N = int32_t(N), p.D = int32_t(Dn), p.L = int32_t(L), p.S = int32_t(S), p.G = int32_t(G);
  p.dtype = dtype_of(c.type()), p.delta_softplus = flag(softplus);
  p.u = u.data_ptr(), p.u_n = u.stride(0), p.u_d = u.stride(1);
  const Tensor& dt = get(delta, "delta", u.sizes());
  p.delta = dt.data_ptr(), p.delta_n = dt.stride(0), p.delta_d = dt.stride(1);
  if (z != Py_None) {
    const Tensor& zt = get(z, "z", u.sizes());
    p.z = zt.data_ptr(), p.z_n = zt.stride(0), p.z_d = zt.stride(1);
  }
  p.A = static_cast<const float*>(c.dense(A, "A", {Dn, S}, at::kFloat).data_ptr());
  get(B, "B", bsize);
  p.B = Bt.data_ptr(), p.B_n = Bt.stride(0), p.B_g = Bt.stride(1), p.B_s = Bt.stride(2);
  const Tensor& Ct = get(C, "C", bsize);
  p.C = Ct.data_ptr(), p.C_n = Ct.stride(0), p.C_g = Ct.stride(1), p.C_s = Ct.stride(2);
  p.Dskip = c.opt(D, "D", {Dn});
  p.delta_bias = c.opt(bias, "delta_bias", {Dn});
  p.lengths = c.opt<const int32_t>(lengths, "lengths", {N}, at::kInt);
  return p;
}
int64_t chunks_of(const seq_scan_t& p) { return (int64_t(p.L) + SEQ_SCAN_CHUNK - 1) / SEQ_SCAN_CHUNK; }

// u, delta, A, B, C, D, z, delta_bias, delta_softplus, initial_state, lengths,
// return_final_state, return_checkpoints, out
PyObject* scan_fwd(PyObject* const* a) {
  const Tensor& u = lead(a[0], "u", 3);
  const Call c(u, "u");
  c.seq(a[0], "u", u.sizes(), c.type());
  seq_scan_t p = scan_args(c, u, a[1], a[2], a[3], a[4], a[5], a[6], a[7], a[8], a[10]);
  p.initial_state = c.opt(a[9], "initial_state", {p.N, p.D, p.S});
  const Tensor out = c.out(a[13], u.sizes(), c.type());
  p.out = out.data_ptr();
  Tensor fin, chk;
  if (flag(a[11])) fin = c.empty({p.N, p.D, p.S}, at::kFloat), p.final_state = static_cast<float*>(fin.data_ptr());
  if (flag(a[12]))
    chk = c.empty({p.N, chunks_of(p), p.D, p.S}, at::kFloat), p.checkpoints = static_cast<float*>(chk.data_ptr());
  c.run("selective_scan_fwd", seq_selective_scan_fwd, p, seq_selective_scan_fwd_workspace);
  if (fin.defined() && chk.defined()) return wrap({out, fin, chk});
  if (fin.defined() || chk.defined()) return wrap({out, fin.defined() ? fin : chk});
  return wrap(out);
}

// dout, u, delta, A, B, C, checkpoints, D, z, delta_bias, delta_softplus,
// lengths, dfinal_state
PyObject* scan_bwd(PyObject* const* a) {
  const Tensor& u = lead(a[1], "u", 3);
  const Call c(u, "u");
  c.seq(a[1], "u", u.sizes(), c.type());
  seq_scan_t p = scan_args(c, u, a[2], a[3], a[4], a[5], a[7], a[8], a[9], a[10], a[11]);
  const Tensor& dout = c.seq(a[0], "dout", u.sizes(), c.type());
  p.dout = dout.data_ptr(), p.dout_n = dout.stride(0), p.dout_d = dout.stride(1);
  p.checkpoints = static_cast<float*>(
      c.dense(a[6], "checkpoints", {p.N, chunks_of(p), p.D, p.S}, at::kFloat).data_ptr());
  p.dfinal_state = c.opt(a[12], "dfinal_state", {p.N, p.D, p.S});
  const auto ptr = [](const Tensor& t) { return static_cast<float*>(t.data_ptr()); };
  const Tensor du = c.empty(u.sizes(), c.type()), dd = c.empty(u.sizes(), c.type());
  const Tensor dA = c.empty({p.D, p.S}, at::kFloat), di = c.empty({p.N, p.D, p.S}, at::kFloat);
  const Tensor dB = c.empty({p.N, p.G, p.S, p.L}, c.type()), dC = c.empty({p.N, p.G, p.S, p.L}, c.type());
  Tensor dD, db, dz;
  p.du = du.data_ptr(), p.ddelta = dd.data_ptr(), p.dB = dB.data_ptr(), p.dC = dC.data_ptr();
  p.dA = ptr(dA), p.dinitial_state = ptr(di);
  if (p.Dskip) dD = c.empty({p.D}, at::kFloat), p.dDskip = ptr(dD);
  if (p.delta_bias) db = c.empty({p.D}, at::kFloat), p.ddelta_bias = ptr(db);
  if (p.z) dz = c.empty(u.sizes(), c.type()), p.dz = dz.data_ptr();
  c.run("selective_scan_bwd", seq_selective_scan_bwd, p, seq_selective_scan_bwd_workspace);
  return wrap({du, dd, dA, dB, dC, dD, db, dz, di});
}

// u, state, delta, A, B, C, D, z, delta_bias, delta_softplus, new_state, out
PyObject* scan_step(PyObject* const* a) {
  const Tensor& u = lead(a[0], "u", 2);
  const Call c(u, "u");
  seq_scan_t p = scan_args(c, u, a[2], a[3], a[4], a[5], a[6], a[7], a[8], a[9], Py_None);
  const Tensor& state = c.dense(a[1], "state", {p.N, p.D, p.S}, at::kFloat);
  p.initial_state = static_cast<const float*>(state.data_ptr());
  const Tensor out = c.out(a[11], u.sizes(), c.type());
  p.out = out.data_ptr();
  p.final_state = static_cast<float*>(c.new_state(a[10], state, out));
  c.run("selective_scan_step", seq_selective_scan_step, p);
  return wrap(out);
}

// ------------------------------------------------------------------------ norms

// x (or what has its type and extents), weight, scale, eps; the residual's type
seq_norm_t norm_args(const Call& c, PyObject* weight, PyObject* scale, PyObject* eps, ScalarType rt) {
  const Tensor& x = c.like;
  if (rt != c.type() && rt != at::kFloat)
    type_error(std::string("the residual's type must be ") + type_name(c.type()) + " or float32, got " +
               type_name(rt));
  seq_norm_t p = {};
  p.N = int32_t(x.size(0)), p.D = int32_t(x.size(1)), p.L = int32_t(x.size(2));
  p.dtype = dtype_of(c.type()), p.res_dtype = dtype_of(rt);
  const double e = PyFloat_AsDouble(eps);
  if (e == -1.0 && PyErr_Occurred()) throw python_error();
  if (!(e >= 0)) value_error("eps must not be negative");
  p.eps = float(e);
  const int64_t D = x.size(1);
  p.weight = static_cast<const float*>(c.dense(weight, "weight", {D}, at::kFloat).data_ptr());
  p.scale = c.opt(scale, "scale", {D});
  return p;
}
const void* strided(const Call& c, PyObject* o, const char* name, ScalarType t, int64_t* n, int64_t* d) {
  if (o == Py_None) return nullptr;
  const Tensor& x = c.seq(o, name, c.like.sizes(), t);
  *n = x.stride(0), *d = x.stride(1);
  return x.data_ptr();
}

// x, weight, residual, scale, eps, out
PyObject* norm_pre_fwd(PyObject* const* a) {
  const Tensor& x = lead(a[0], "x", 3);
  const Call c(x, "x");
  const ScalarType rt = a[2] == Py_None ? c.type() : tensor(a[2], "residual").scalar_type();
  seq_norm_t p = norm_args(c, a[1], a[3], a[4], rt);
  p.x = strided(c, a[0], "x", c.type(), &p.x_n, &p.x_d);
  p.residual = strided(c, a[2], "residual", rt, &p.res_n, &p.res_d);
  const Tensor out = c.out(a[5], x.sizes(), c.type()), sum = c.empty(x.sizes(), rt);
  p.out = out.data_ptr(), p.sum = sum.data_ptr();
  c.run("norm_pre_fwd", seq_norm_pre_fwd, p, seq_norm_fwd_workspace);
  return wrap({out, sum});
}

// dout, sum, weight, dsum, x, scale, eps
PyObject* norm_pre_bwd(PyObject* const* a) {
  const Tensor& dout = lead(a[0], "dout", 3);
  const Call c(dout, "dout");
  const ScalarType rt = tensor(a[1], "sum").scalar_type();
  seq_norm_t p = norm_args(c, a[2], a[5], a[6], rt);
  p.dout = strided(c, a[0], "dout", c.type(), &p.dout_n, &p.dout_d);
  p.sum = const_cast<void*>(strided(c, a[1], "sum", rt, &p.res_n, &p.res_d));
  p.dsum = strided(c, a[3], "dsum", rt, &p.dsum_n, &p.dsum_d);
  if (p.scale) {
    if (a[4] == Py_None) value_error("x is needed for the gradient of scale");
    p.x = strided(c, a[4], "x", c.type(), &p.x_n, &p.x_d);
  }
  const Tensor dx = c.empty(dout.sizes(), c.type()), dr = c.empty(dout.sizes(), rt), dw = c.empty({p.D}, at::kFloat);
  Tensor ds;
  p.dx = dx.data_ptr(), p.dresidual = dr.data_ptr(), p.dweight = static_cast<float*>(dw.data_ptr());
  if (p.scale) ds = c.empty({p.D}, at::kFloat), p.dscale = static_cast<float*>(ds.data_ptr());
  c.run("norm_pre_bwd", seq_norm_pre_bwd, p, seq_norm_bwd_workspace);
  return wrap({dx, dr, dw, ds});
}

// x, weight, gate, residual, scale, eps, out
PyObject* norm_post_fwd(PyObject* const* a) {
  const Tensor& x = lead(a[0], "x", 3);
  const Call c(x, "x");
  const ScalarType rt = a[3] == Py_None ? c.type() : tensor(a[3], "residual").scalar_type();
  seq_norm_t p = norm_args(c, a[1], a[4], a[5], rt);
  p.x = strided(c, a[0], "x", c.type(), &p.x_n, &p.x_d);
  p.gate = strided(c, a[2], "gate", c.type(), &p.gate_n, &p.gate_d);
  p.residual = strided(c, a[3], "residual", rt, &p.res_n, &p.res_d);
  const Tensor out = c.out(a[6], x.sizes(), rt);
  p.out = out.data_ptr();
  c.run("norm_post_fwd", seq_norm_post_fwd, p, seq_norm_fwd_workspace);
  return wrap(out);
}

// dout, x, weight, gate, scale, eps
PyObject* norm_post_bwd(PyObject* const* a) {
  const Tensor& x = lead(a[1], "x", 3);
  const Call c(x, "x");
  const ScalarType rt = tensor(a[0], "dout").scalar_type();
  seq_norm_t p = norm_args(c, a[2], a[4], a[5], rt);
  p.x = strided(c, a[1], "x", c.type(), &p.x_n, &p.x_d);
  p.gate = strided(c, a[3], "gate", c.type(), &p.gate_n, &p.gate_d);
  p.dout = strided(c, a[0], "dout", rt, &p.dout_n, &p.dout_d);
  const Tensor dx = c.empty(x.sizes(), c.type()), dw = c.empty({p.D}, at::kFloat);
  Tensor dg, ds;
  p.dx = dx.data_ptr(), p.dweight = static_cast<float*>(dw.data_ptr());
  if (p.gate) dg = c.empty(x.sizes(), c.type()), p.dgate = dg.data_ptr();
  if (p.scale) ds = c.empty({p.D}, at::kFloat), p.dscale = static_cast<float*>(ds.data_ptr());
  c.run("norm_post_bwd", seq_norm_post_bwd, p, seq_norm_bwd_workspace);
  return wrap({dx, dg, dw, ds});
}

// (no C++ exception leaves: they become Python's)
template <PyObject* (*F)(PyObject* const*), Py_ssize_t COUNT>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  need(n, COUNT);
  return F(args);
  END_HANDLE_TH_ERRORS
}
template <PyObject* (*F)(PyObject* const*), Py_ssize_t COUNT>
PyMethodDef method(const char* name) {
  return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&entry<F, COUNT>)), METH_FASTCALL, nullptr};
}

PyMethodDef methods[] = {
    method<conv_fwd, 8>("causal_conv_fwd"),       method<conv_bwd, 8>("causal_conv_bwd"),
    method<conv_step, 7>("causal_conv_step"),     method<scan_fwd, 14>("selective_scan_fwd"),
    method<scan_bwd, 13>("selective_scan_bwd"),   method<scan_step, 12>("selective_scan_step"),
    method<norm_pre_fwd, 6>("norm_pre_fwd"),      method<norm_pre_bwd, 7>("norm_pre_bwd"),
    method<norm_post_fwd, 7>("norm_post_fwd"),    method<norm_post_bwd, 6>("norm_post_bwd"),
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_seq", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

extern "C" __attribute__((visibility("default"))) PyObject* PyInit__seq() { return PyModule_Create(&module); }
