"""Sequence operators on channels-first tensors ``[N, D, L]``: the Python
binding of ``include/seq_ops.h`` (ctypes).

Short causal convolutions, the selective scan and channel norms, each forward,
backward and (the first two) for single tokens.  As in ``conv``, arguments are
checked and marshalled here and every step of the computation runs in the HIP
library; there is no fallback.

Sequences (``x``, ``u``, ``delta``, ``z``, ``B``, ``C``, ``gate``, ``residual``
and gradients that come in) are fp32 or bf16 with the length innermost and of
stride 1; their other strides are free.  Parameters, states and ``lengths`` are
contiguous; parameters, scan states and ``lengths`` are fp32, fp32 and int32.
``lengths`` holds each sequence's valid steps, clamped to ``0..L``; what lies
behind them is not read, and outputs and gradients are zero there.

Results, and the scratch that a call needs, come from torch's allocator, so
calls may be captured into graphs and run on any stream.  ``stream`` (a
``torch.cuda.Stream``; default: the current one of the tensors' device) is the
stream that the call's kernels run on and its results belong to; ordering the
inputs before it is the caller's part.
"""
import ctypes
from typing import NamedTuple, Optional

import torch

from .conv import CONV_DTYPE_BF16, CONV_DTYPE_F32, CONV_OK, ConvError, lib as _conv_lib

CHUNK = 128
MAX_TAPS = 8
MAX_STATE = 64

_i32, _i64, _vp, _f32 = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p, ctypes.c_float
_DTYPES = {torch.float32: CONV_DTYPE_F32, torch.bfloat16: CONV_DTYPE_BF16}
_ACTIVATIONS = {None: 0, "silu": 1}


def _fields(spec):
    types = {"i": _i32, "l": _i64, "p": _vp, "f": _f32}
    return [(name, types[kind]) for kind, names in spec for name in names.split()]


class _Conv(ctypes.Structure):
    """Mirror of ``seq_conv_t``."""
    _fields_ = _fields([
        ("i", "N D L R dtype activation"), ("l", "x_n x_d dout_n dout_d"),
        ("p", "x weight bias initial_state lengths out final_state dout dfinal_state dx dweight dbias dinitial_state"),
        ("p", "workspace"), ("l", "workspace_bytes")])


class _Scan(ctypes.Structure):
    """Mirror of ``seq_scan_t``."""
    _fields_ = _fields([
        ("i", "N D L S G dtype delta_softplus reserved"),
        ("l", "u_n u_d delta_n delta_d z_n z_d dout_n dout_d B_n B_g B_s C_n C_g C_s"),
        ("p", "u delta z A B C Dskip delta_bias initial_state lengths out final_state checkpoints dout dfinal_state"),
        ("p", "du ddelta dz dA dB dC dDskip ddelta_bias dinitial_state workspace"), ("l", "workspace_bytes")])


class _Norm(ctypes.Structure):
    """Mirror of ``seq_norm_t``."""
    _fields_ = _fields([
        ("i", "N D L dtype res_dtype"), ("f", "eps"),
        ("l", "x_n x_d gate_n gate_d res_n res_d dout_n dout_d dsum_n dsum_d"),
        ("p", "x weight scale gate residual out sum dout dsum dx dgate dresidual dweight dscale workspace"),
        ("l", "workspace_bytes")])


_lib = None


def lib():
    """The loaded HIP library with the sequence operators' signatures."""
    global _lib
    if _lib is None:
        L = _conv_lib()
        for struct, calls, sizes in (
                (_Conv, "causal_conv_fwd causal_conv_bwd causal_conv_step", "causal_conv_bwd_workspace"),
                (_Scan, "selective_scan_fwd selective_scan_bwd selective_scan_step",
                 "selective_scan_fwd_workspace selective_scan_bwd_workspace"),
                (_Norm, "norm_pre_fwd norm_pre_bwd norm_post_fwd norm_post_bwd", "norm_bwd_workspace")):
            for f in calls.split():
                getattr(L, "seq_" + f).argtypes = [ctypes.POINTER(struct), _vp]
                getattr(L, "seq_" + f).restype = _i32
            for f in sizes.split():
                getattr(L, "seq_" + f).argtypes = [ctypes.POINTER(struct)]
                getattr(L, "seq_" + f).restype = _i64
        _lib = L
    return _lib


class ConvGrads(NamedTuple):
    """Gradients of :func:`causal_conv_fwd`."""
    dx: torch.Tensor
    dweight: torch.Tensor
    dbias: Optional[torch.Tensor]
    dinitial_state: Optional[torch.Tensor]


class ScanGrads(NamedTuple):
    """Gradients of :func:`selective_scan_fwd`."""
    du: torch.Tensor
    ddelta: torch.Tensor
    dA: torch.Tensor
    dB: torch.Tensor
    dC: torch.Tensor
    dD: Optional[torch.Tensor]
    ddelta_bias: Optional[torch.Tensor]
    dz: Optional[torch.Tensor]
    dinitial_state: Optional[torch.Tensor]


class NormPreGrads(NamedTuple):
    """Gradients of :func:`norm_pre_fwd`."""
    dx: torch.Tensor
    dresidual: torch.Tensor
    dweight: torch.Tensor
    dscale: Optional[torch.Tensor]


class NormPostGrads(NamedTuple):
    """Gradients of :func:`norm_post_fwd` (the residual's is ``dout``)."""
    dx: torch.Tensor
    dgate: Optional[torch.Tensor]
    dweight: torch.Tensor
    dscale: Optional[torch.Tensor]


# ------------------------------------------------------------------ arguments

def _first(x, name, rank):
    """The tensor that sets a call's type, extents and device."""
    if not isinstance(x, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    if not x.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor (the library has no CPU path)")
    if x.dtype not in _DTYPES:
        raise TypeError(f"{name} must be float32 or bfloat16, got {x.dtype}")
    if x.dim() != rank:
        raise ValueError(f"{name} must have {rank} dimensions, got {tuple(x.shape)}")
    if x.numel() == 0:
        raise ValueError(f"{name} is empty: {tuple(x.shape)}")


def _check(x, name, shape, dtype, like):
    if not isinstance(x, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    if x.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {x.dtype}")
    if x.shape != shape:
        raise ValueError(f"{name} must be {tuple(shape)}, got {tuple(x.shape)}")
    if x.device != like.device:
        raise ValueError(f"{name} must be on {like.device}, is on {x.device}")


def _seq(x, name, shape, dtype, like):
    """A sequence tensor's address; its strides are read by the caller."""
    _check(x, name, shape, dtype, like)
    if x.stride(-1) != 1 and shape[-1] > 1:
        raise ValueError(f"{name} must have stride 1 along the length, has strides {x.stride()}")
    return x.data_ptr()


def _dense(x, name, shape, dtype, like):
    _check(x, name, shape, dtype, like)
    if not x.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return x.data_ptr()


def _opt(x, name, shape, dtype, like):
    return None if x is None else _dense(x, name, shape, dtype, like)


def _lengths(x, like):
    return None if x is None else _dense(x, "lengths", like.shape[:1], torch.int32, like)


def _activation(a):
    if a not in _ACTIVATIONS:
        raise ValueError(f"activation must be None or 'silu', got {a!r}")
    return _ACTIVATIONS[a]


def _out(x, name, shape, dtype, like):
    if x is None:
        return torch.empty(shape, dtype=dtype, device=like.device)
    _dense(x, name, shape, dtype, like)
    return x


class _On:
    """The device and stream of a call: results are allocated, and kernels
    enqueued, on them.  Tensors that come from another stream's pool are
    recorded on it, so that freeing them does not hand their memory on while
    the call still runs."""
    __slots__ = ("device", "stream", "outer", "ptr")

    def __init__(self, like, stream, tensors):
        dev = like.device.index
        self.device = self.outer = None
        self.stream = None
        if torch.cuda.current_device() != dev:
            self.device = torch.cuda.device(dev)
        if stream is not None:
            if stream.device.index != dev:
                raise ValueError(f"stream is on {stream.device}, the tensors are on {like.device}")
            if stream != torch.cuda.current_stream(dev):
                self.stream = torch.cuda.stream(stream)
                for t in tensors:
                    if t is not None:
                        t.record_stream(stream)

    def __enter__(self):
        if self.device is not None:
            self.device.__enter__()
        if self.stream is not None:
            self.stream.__enter__()
        self.ptr = _current_stream()
        return self

    def __exit__(self, *exc):
        if self.stream is not None:
            self.stream.__exit__(*exc)
        if self.device is not None:
            self.device.__exit__(*exc)
        return False


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_current_device = getattr(torch._C, "_cuda_getDevice", None)


def _current_stream():
    if _raw_stream is not None and _current_device is not None:
        return _raw_stream(_current_device())
    return torch.cuda.current_stream().cuda_stream


def _call(name, p, on, size=None, like=None):
    """Enqueues `name`; `size` names the function that gives its scratch."""
    L = _lib or lib()
    scratch = None
    if size is not None:
        n = getattr(L, size)(p)
        if n < 0:
            raise ConvError(n, name)
        if n > 0:
            scratch = torch.empty(n, dtype=torch.uint8, device=like.device)
            p.workspace, p.workspace_bytes = scratch.data_ptr(), n
    st = getattr(L, name)(p, on.ptr)
    if st != CONV_OK:
        raise ConvError(st, name)


# --------------------------------------------------------- causal convolution

def _conv(x, weight, bias, activation, initial_state, lengths, rank):
    _first(x, "x", rank)
    if not isinstance(weight, torch.Tensor):
        raise TypeError("weight must be a torch tensor")
    N, D = x.shape[:2]
    if weight.dim() != 2 or not 1 <= weight.shape[1] <= MAX_TAPS:
        raise ValueError(f"weight must be [{D}, R] with R of 1 to {MAX_TAPS}, got {tuple(weight.shape)}")
    R = weight.shape[1]
    L = x.shape[2] if rank == 3 else 1
    if rank == 3:
        _seq(x, "x", x.shape, x.dtype, x)
    return _Conv(
        N=N, D=D, L=L, R=R, dtype=_DTYPES[x.dtype], activation=_activation(activation), x_n=x.stride(0),
        x_d=x.stride(1), x=x.data_ptr(), weight=_dense(weight, "weight", (D, R), torch.float32, x),
        bias=_opt(bias, "bias", (D,), torch.float32, x),
        initial_state=_opt(initial_state, "initial_state", (N, D, R - 1), x.dtype, x) if R > 1 else None,
        lengths=_lengths(lengths, x))


def causal_conv_fwd(x, weight, bias=None, *, activation=None, initial_state=None, lengths=None,
                    return_final_state=False, out=None, stream=None):
    """``out[n, d, t] = act(bias[d] + sum_r weight[d, r] x[n, d, t - (R-1) + r])``.

    x ``[N, D, L]``, weight ``[D, R]`` (R of 1 to 8) and bias ``[D]`` fp32.
    ``activation``: None or "silu".  ``initial_state`` ``[N, D, R-1]`` (of x's
    type, oldest first) stands before t = 0, else zeros do.  Returns out
    ``[N, D, L]`` of x's type, or (out, final_state) with
    ``return_final_state``: the last R-1 entries of each sequence, the
    ``initial_state`` of the call that continues it.
    """
    p = _conv(x, weight, bias, activation, initial_state, lengths, 3)
    with _On(x, stream, (x, weight, bias, initial_state, lengths, out)) as on:
        out = _out(out, "out", x.shape, x.dtype, x)
        p.out = out.data_ptr()
        final = None
        if return_final_state:
            final = torch.empty((p.N, p.D, p.R - 1), dtype=x.dtype, device=x.device)
            p.final_state = final.data_ptr() or None
        _call("seq_causal_conv_fwd", p, on)
    return (out, final) if return_final_state else out


def causal_conv_bwd(dout, x, weight, bias=None, *, activation=None, initial_state=None, lengths=None,
                    dfinal_state=None, stream=None):
    """:class:`ConvGrads` of :func:`causal_conv_fwd` called with the same
    arguments, for ``dout`` ``[N, D, L]`` and, if the final state was used,
    ``dfinal_state``.  ``dbias`` and ``dinitial_state`` are None where the call
    had no bias or initial state."""
    p = _conv(x, weight, bias, activation, initial_state, lengths, 3)
    p.dout = _seq(dout, "dout", x.shape, x.dtype, x)
    p.dout_n, p.dout_d = dout.stride(0), dout.stride(1)
    if p.R > 1:
        p.dfinal_state = _opt(dfinal_state, "dfinal_state", (p.N, p.D, p.R - 1), x.dtype, x)
    with _On(x, stream, (dout, x, weight, bias, initial_state, lengths, dfinal_state)) as on:
        g = ConvGrads(torch.empty(x.shape, dtype=x.dtype, device=x.device), torch.empty_like(weight),
                      None if bias is None else torch.empty_like(bias),
                      None if initial_state is None else torch.empty_like(initial_state))
        p.dx, p.dweight = g.dx.data_ptr(), g.dweight.data_ptr()
        if bias is not None:
            p.dbias = g.dbias.data_ptr()
        if initial_state is not None:
            p.dinitial_state = g.dinitial_state.data_ptr() or None
        _call("seq_causal_conv_bwd", p, on, "seq_causal_conv_bwd_workspace", x)
    return g


def causal_conv_step(x, state, weight, bias=None, *, activation=None, new_state=None, out=None, stream=None):
    """One token of :func:`causal_conv_fwd`: x ``[N, D]`` (any strides), state
    ``[N, D, R-1]``.  Returns out ``[N, D]``; the state after the token goes to
    ``new_state``, by default in place of ``state``."""
    p = _conv(x, weight, bias, activation, state, None, 2)
    new_state = state if new_state is None else new_state
    p.final_state = _dense(new_state, "new_state", (p.N, p.D, p.R - 1), x.dtype, x) or None
    with _On(x, stream, (x, weight, bias, state, new_state, out)) as on:
        out = _out(out, "out", x.shape, x.dtype, x)
        p.out = out.data_ptr()
        _call("seq_causal_conv_step", p, on)
    return out


# -------------------------------------------------------------- selective scan

def _scan(u, delta, A, B, C, D, z, delta_bias, delta_softplus, initial_state, lengths, rank):
    _first(u, "u", rank)
    for t, name in ((A, "A"), (B, "B"), (C, "C")):
        if not isinstance(t, torch.Tensor):
            raise TypeError(f"{name} must be a torch tensor")
    N, Dn = u.shape[:2]
    dt = u.dtype
    if A.dim() != 2 or not 1 <= A.shape[1] <= MAX_STATE:
        raise ValueError(f"A must be [{Dn}, S] with S of 1 to {MAX_STATE}, got {tuple(A.shape)}")
    S = A.shape[1]
    if B.dim() != rank + 1:
        raise ValueError(f"B must be [N, G, S{', L' if rank == 3 else ''}], got {tuple(B.shape)}")
    G = B.shape[1]
    if G < 1 or Dn % G:
        raise ValueError(f"{Dn} channels do not divide into {G} groups")
    bshape = (N, G, S) + tuple(u.shape[2:])
    addr = _seq if rank == 3 else _any
    return _Scan(
        N=N, D=Dn, L=u.shape[2] if rank == 3 else 1, S=S, G=G, dtype=_DTYPES[dt], delta_softplus=bool(delta_softplus),
        u_n=u.stride(0), u_d=u.stride(1), u=addr(u, "u", u.shape, dt, u),
        delta=addr(delta, "delta", u.shape, dt, u), delta_n=delta.stride(0), delta_d=delta.stride(1),
        z=None if z is None else addr(z, "z", u.shape, dt, u), z_n=0 if z is None else z.stride(0),
        z_d=0 if z is None else z.stride(1), A=_dense(A, "A", (Dn, S), torch.float32, u),
        B=addr(B, "B", bshape, dt, u), B_n=B.stride(0), B_g=B.stride(1), B_s=B.stride(2),
        C=addr(C, "C", bshape, dt, u), C_n=C.stride(0), C_g=C.stride(1), C_s=C.stride(2),
        Dskip=_opt(D, "D", (Dn,), torch.float32, u), delta_bias=_opt(delta_bias, "delta_bias", (Dn,), torch.float32, u),
        initial_state=_opt(initial_state, "initial_state", (N, Dn, S), torch.float32, u), lengths=_lengths(lengths, u))


def _any(x, name, shape, dtype, like):
    _check(x, name, shape, dtype, like)
    return x.data_ptr()


def selective_scan_fwd(u, delta, A, B, C, *, D=None, z=None, delta_bias=None, delta_softplus=False,
                       initial_state=None, lengths=None, return_final_state=False, return_checkpoints=False,
                       out=None, stream=None):
    """The recurrence ``h(t) = exp(dt A) h(t-1) + dt u B(t)``, ``y = C(t) h(t) + D u``.

    u, delta, z ``[N, D, L]``; A ``[D, S]`` fp32 (S of 1 to 64); B, C
    ``[N, G, S, L]``, group g of the G serving channels ``g D/G`` and on; D and
    delta_bias ``[D]`` fp32.  ``dt = delta + delta_bias``, through softplus with
    ``delta_softplus``.  With z the output is ``y z sigmoid(z)``.
    ``initial_state`` ``[N, D, S]`` fp32, else zero.  A is meant to be negative:
    where ``A dt`` grows past fp32's range within 128 steps, states may be NaN.

    Returns out, or a tuple of out, the final state (with
    ``return_final_state``) and what :func:`selective_scan_bwd` takes as
    ``checkpoints`` (with ``return_checkpoints``; the state before every 128th
    step), in this order.
    """
    p = _scan(u, delta, A, B, C, D, z, delta_bias, delta_softplus, initial_state, lengths, 3)
    with _On(u, stream, (u, delta, A, B, C, D, z, delta_bias, initial_state, lengths, out)) as on:
        out = _out(out, "out", u.shape, u.dtype, u)
        p.out = out.data_ptr()
        res = [out]
        if return_final_state:
            res.append(torch.empty((p.N, p.D, p.S), dtype=torch.float32, device=u.device))
            p.final_state = res[-1].data_ptr()
        if return_checkpoints:
            res.append(torch.empty((p.N, -(-p.L // CHUNK), p.D, p.S), dtype=torch.float32, device=u.device))
            p.checkpoints = res[-1].data_ptr()
        _call("seq_selective_scan_fwd", p, on, "seq_selective_scan_fwd_workspace", u)
    return tuple(res) if len(res) > 1 else out


def selective_scan_bwd(dout, u, delta, A, B, C, checkpoints, *, D=None, z=None, delta_bias=None,
                       delta_softplus=False, lengths=None, dfinal_state=None, stream=None):
    """:class:`ScanGrads` of :func:`selective_scan_fwd` called with the same
    arguments, from the ``checkpoints`` that it returned.  Gradients of
    arguments that the call did not have are None; ``dinitial_state`` is always
    formed."""
    p = _scan(u, delta, A, B, C, D, z, delta_bias, delta_softplus, None, lengths, 3)
    p.dout = _seq(dout, "dout", u.shape, u.dtype, u)
    p.dout_n, p.dout_d = dout.stride(0), dout.stride(1)
    states = (p.N, p.D, p.S)
    p.dfinal_state = _opt(dfinal_state, "dfinal_state", states, torch.float32, u)
    p.checkpoints = _dense(checkpoints, "checkpoints", (p.N, -(-p.L // CHUNK), p.D, p.S), torch.float32, u)

    def new(shape, dtype=u.dtype):
        return torch.empty(shape, dtype=dtype, device=u.device)

    with _On(u, stream, (dout, u, delta, A, B, C, checkpoints, D, z, delta_bias, lengths, dfinal_state)) as on:
        f32 = torch.float32
        g = ScanGrads(new(u.shape), new(u.shape), new(A.shape, f32), new(B.shape), new(C.shape),
                      None if D is None else new((p.D,), f32), None if delta_bias is None else new((p.D,), f32),
                      None if z is None else new(u.shape), new(states, f32))
        p.du, p.ddelta, p.dA, p.dB, p.dC = (t.data_ptr() for t in g[:5])
        p.dDskip, p.ddelta_bias, p.dz, p.dinitial_state = (None if t is None else t.data_ptr() for t in g[5:])
        _call("seq_selective_scan_bwd", p, on, "seq_selective_scan_bwd_workspace", u)
    return g


def selective_scan_step(u, state, delta, A, B, C, *, D=None, z=None, delta_bias=None, delta_softplus=False,
                        new_state=None, out=None, stream=None):
    """One token of :func:`selective_scan_fwd`: u, delta, z ``[N, D]``, B, C
    ``[N, G, S]`` (any strides), state ``[N, D, S]`` fp32.  Returns out
    ``[N, D]``; the state after the token goes to ``new_state``, by default in
    place of ``state``."""
    p = _scan(u, delta, A, B, C, D, z, delta_bias, delta_softplus, None, None, 2)
    states = (p.N, p.D, p.S)
    p.initial_state = _dense(state, "state", states, torch.float32, u)
    new_state = state if new_state is None else new_state
    p.final_state = _dense(new_state, "new_state", states, torch.float32, u)
    with _On(u, stream, (u, state, delta, A, B, C, D, z, delta_bias, new_state, out)) as on:
        out = _out(out, "out", u.shape, u.dtype, u)
        p.out = out.data_ptr()
        _call("seq_selective_scan_step", p, on)
    return out


# ------------------------------------------------------------------------ norms

def _norm(x, weight, scale, eps, res_dtype):
    """x sets the type; `res_dtype` is the residual's (x's type or fp32)."""
    _first(x, "x", 3)
    if res_dtype not in (x.dtype, torch.float32):
        raise TypeError(f"the residual's type must be {x.dtype} or float32, got {res_dtype}")
    if not eps >= 0:
        raise ValueError(f"eps must not be negative, got {eps}")
    N, D, L = x.shape
    return _Norm(N=N, D=D, L=L, dtype=_DTYPES[x.dtype], res_dtype=_DTYPES[res_dtype], eps=eps,
                 x=_seq(x, "x", x.shape, x.dtype, x), x_n=x.stride(0), x_d=x.stride(1),
                 weight=_dense(weight, "weight", (D,), torch.float32, x),
                 scale=_opt(scale, "scale", (D,), torch.float32, x))


def _strided(p, key, t, name, shape, dtype, like, field=None):
    if t is None:
        return
    setattr(p, field or key, _seq(t, name, shape, dtype, like))
    setattr(p, key + "_n", t.stride(0))
    setattr(p, key + "_d", t.stride(1))


def _residual_dtype(t, x):
    return t.dtype if isinstance(t, torch.Tensor) else x.dtype if isinstance(x, torch.Tensor) else None


def norm_pre_fwd(x, weight, *, residual=None, scale=None, eps=1e-6, out=None, stream=None):
    """The norm before a block, with what joins the residual stream there:
    ``sum = residual + scale x``, ``out = weight sum rstd(sum)`` over the
    channels of each position.  x, residual ``[N, D, L]`` (residual of x's type
    or fp32), weight and scale ``[D]`` fp32.  Returns (out of x's type, sum of
    the residual's); without a residual ``sum`` is ``scale x``."""
    rt = _residual_dtype(residual, x)
    p = _norm(x, weight, scale, eps, rt)
    _strided(p, "res", residual, "residual", x.shape, rt, x, "residual")
    with _On(x, stream, (x, weight, residual, scale, out)) as on:
        out = _out(out, "out", x.shape, x.dtype, x)
        s = torch.empty(x.shape, dtype=rt, device=x.device)
        p.out, p.sum = out.data_ptr(), s.data_ptr()
        _call("seq_norm_pre_fwd", p, on)
    return out, s


def norm_pre_bwd(dout, sum, weight, *, dsum=None, x=None, scale=None, eps=1e-6, stream=None):
    """:class:`NormPreGrads` of :func:`norm_pre_fwd` from the ``sum`` that it
    returned; ``dsum`` is the gradient that reaches ``sum`` from elsewhere (the
    residual stream).  ``x`` is needed where the call had a ``scale``."""
    if scale is not None and x is None:
        raise ValueError("x is needed for the gradient of scale")
    rt = _residual_dtype(sum, dout)
    p = _norm(dout, weight, scale, eps, rt)
    shape, dt = dout.shape, dout.dtype
    p.dout, p.dout_n, p.dout_d = p.x, p.x_n, p.x_d
    p.x = None
    if scale is not None:
        _strided(p, "x", x, "x", shape, dt, dout)
    _strided(p, "res", sum, "sum", shape, rt, dout, "sum")
    _strided(p, "dsum", dsum, "dsum", shape, rt, dout)
    with _On(dout, stream, (dout, sum, weight, dsum, x, scale)) as on:
        g = NormPreGrads(torch.empty(shape, dtype=dt, device=dout.device),
                         torch.empty(shape, dtype=rt, device=dout.device), torch.empty_like(weight),
                         None if scale is None else torch.empty_like(scale))
        p.dx, p.dresidual, p.dweight = g.dx.data_ptr(), g.dresidual.data_ptr(), g.dweight.data_ptr()
        if scale is not None:
            p.dscale = g.dscale.data_ptr()
        _call("seq_norm_pre_bwd", p, on, "seq_norm_bwd_workspace", dout)
    return g


def norm_post_fwd(x, weight, *, gate=None, residual=None, scale=None, eps=1e-6, out=None, stream=None):
    """The norm after a block, with its gate and its way back to the residual
    stream: ``v = x gate sigmoid(gate)``, ``out = residual + scale weight v
    rstd(v)`` over the channels of each position.  x, gate, residual
    ``[N, D, L]`` (residual of x's type or fp32), weight and scale ``[D]``
    fp32.  Returns out, of the residual's type."""
    rt = _residual_dtype(residual, x)
    p = _norm(x, weight, scale, eps, rt)
    _strided(p, "gate", gate, "gate", x.shape, x.dtype, x)
    _strided(p, "res", residual, "residual", x.shape, rt, x, "residual")
    with _On(x, stream, (x, weight, gate, residual, scale, out)) as on:
        out = _out(out, "out", x.shape, rt, x)
        p.out = out.data_ptr()
        _call("seq_norm_post_fwd", p, on)
    return out


def norm_post_bwd(dout, x, weight, *, gate=None, scale=None, eps=1e-6, stream=None):
    """:class:`NormPostGrads` of :func:`norm_post_fwd`, for ``dout`` of its
    output's type."""
    rt = _residual_dtype(dout, x)
    p = _norm(x, weight, scale, eps, rt)
    _strided(p, "gate", gate, "gate", x.shape, x.dtype, x)
    _strided(p, "dout", dout, "dout", x.shape, rt, x)
    if dout is None:
        raise TypeError("dout must be a torch tensor")
    with _On(x, stream, (dout, x, weight, gate, scale)) as on:
        g = NormPostGrads(torch.empty(x.shape, dtype=x.dtype, device=x.device),
                          None if gate is None else torch.empty(x.shape, dtype=x.dtype, device=x.device),
                          torch.empty_like(weight), None if scale is None else torch.empty_like(scale))
        p.dx, p.dweight = g.dx.data_ptr(), g.dweight.data_ptr()
        if gate is not None:
            p.dgate = g.dgate.data_ptr()
        if scale is not None:
            p.dscale = g.dscale.data_ptr()
        _call("seq_norm_post_bwd", p, on, "seq_norm_bwd_workspace", x)
    return g
