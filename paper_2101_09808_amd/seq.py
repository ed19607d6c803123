"""Sequence operators on channels-first tensors ``[N, D, L]``: the Python
binding of ``include/seq_ops.h``.

Short causal convolutions, the selective scan and channel norms, each forward,
backward and (the first two) for single tokens.  Arguments are checked and
marshalled in the compiled module ``_seq`` (``csrc/seq_python.cpp``) and every
step of the computation runs in the HIP library; there is no fallback.  Results
are plain tensors: the calls are not recorded by autograd, their gradients are
the ``_bwd`` functions.

Sequences (``x``, ``u``, ``delta``, ``z``, ``B``, ``C``, ``gate``, ``residual``
and gradients that come in) are fp32 or bf16 with the length innermost and of
stride 1; their other strides are free, and no extent is zero.  Parameters, states and ``lengths`` are
contiguous; parameters, scan states and ``lengths`` are fp32, fp32 and int32.
``lengths`` holds each sequence's valid steps, clamped to ``0..L``; what lies
behind them is not read, and outputs and gradients are zero there.

``out`` (of the result's size and type) takes a result in the caller's memory;
it and ``new_state`` are contiguous and share no memory with one another or an
input of the call, but ``new_state`` may be ``state``.

Other results, and the scratch that a call needs, come from torch's allocator, so
calls may be captured into graphs and run on any stream.  ``stream`` (a
``torch.cuda.Stream``; default: the current one of the tensors' device) is the
stream that the call's kernels run on and its results belong to; ordering the
inputs before it is the caller's part.
"""
from typing import NamedTuple, Optional

import torch

from .conv import lib as _conv_lib

CHUNK = 128
MAX_TAPS = 8
MAX_STATE = 64

_native = None


def native():
    """The compiled module (raises if it has not been built)."""
    global _native
    if _native is None:
        _conv_lib()  # (says so if the library itself is missing)
        try:
            from . import _seq
        except ImportError as e:
            raise RuntimeError(f"_seq.so: {e}; build it with `python -m paper_2101_09808_amd.build`") from e
        _native = _seq
    return _native


def _on(stream, f, *args):
    """f(*args) on `stream`.  Results are allocated on it; tensors of another
    stream's pool are recorded on it, so that freeing them does not hand their
    memory on while the call still runs."""
    for t in args:
        if isinstance(t, torch.Tensor) and t.is_cuda:
            if t.device != stream.device:
                raise ValueError(f"stream is on {stream.device}, a tensor is on {t.device}")
            if stream != torch.cuda.current_stream(t.device):
                t.record_stream(stream)
    with torch.cuda.stream(stream):
        return f(*args)


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


# --------------------------------------------------------- causal convolution

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
    f = (_native or native()).causal_conv_fwd
    args = (x, weight, bias, activation, initial_state, lengths, return_final_state, out)
    return f(*args) if stream is None else _on(stream, f, *args)


def causal_conv_bwd(dout, x, weight, bias=None, *, activation=None, initial_state=None, lengths=None,
                    dfinal_state=None, stream=None):
    """:class:`ConvGrads` of :func:`causal_conv_fwd` called with the same
    arguments, for ``dout`` ``[N, D, L]`` and, if the final state was used,
    ``dfinal_state``.  ``dbias`` and ``dinitial_state`` are None where the call
    had no bias or initial state."""
    f = (_native or native()).causal_conv_bwd
    args = (dout, x, weight, bias, activation, initial_state, lengths, dfinal_state)
    return ConvGrads(*(f(*args) if stream is None else _on(stream, f, *args)))


def causal_conv_step(x, state, weight, bias=None, *, activation=None, new_state=None, out=None, stream=None):
    """One token of :func:`causal_conv_fwd`: x ``[N, D]`` (any strides), state
    ``[N, D, R-1]``.  Returns out ``[N, D]``; the state after the token goes to
    ``new_state``, by default in place of ``state``."""
    f = (_native or native()).causal_conv_step
    args = (x, state, weight, bias, activation, new_state, out)
    return f(*args) if stream is None else _on(stream, f, *args)


# -------------------------------------------------------------- selective scan

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
    f = (_native or native()).selective_scan_fwd
    args = (u, delta, A, B, C, D, z, delta_bias, delta_softplus, initial_state, lengths, return_final_state,
            return_checkpoints, out)
    return f(*args) if stream is None else _on(stream, f, *args)


def selective_scan_bwd(dout, u, delta, A, B, C, checkpoints, *, D=None, z=None, delta_bias=None,
                       delta_softplus=False, lengths=None, dfinal_state=None, stream=None):
    """:class:`ScanGrads` of :func:`selective_scan_fwd` called with the same
    arguments, from the ``checkpoints`` that it returned.  Gradients of
    arguments that the call did not have are None; ``dinitial_state`` is always
    formed."""
    f = (_native or native()).selective_scan_bwd
    args = (dout, u, delta, A, B, C, checkpoints, D, z, delta_bias, delta_softplus, lengths, dfinal_state)
    return ScanGrads(*(f(*args) if stream is None else _on(stream, f, *args)))


def selective_scan_step(u, state, delta, A, B, C, *, D=None, z=None, delta_bias=None, delta_softplus=False,
                        new_state=None, out=None, stream=None):
    """One token of :func:`selective_scan_fwd`: u, delta, z ``[N, D]``, B, C
    ``[N, G, S]`` (any strides), state ``[N, D, S]`` fp32.  Returns out
    ``[N, D]``; the state after the token goes to ``new_state``, by default in
    place of ``state``."""
    f = (_native or native()).selective_scan_step
    args = (u, state, delta, A, B, C, D, z, delta_bias, delta_softplus, new_state, out)
    return f(*args) if stream is None else _on(stream, f, *args)


# ------------------------------------------------------------------------ norms

def norm_pre_fwd(x, weight, *, residual=None, scale=None, eps=1e-6, out=None, stream=None):
    """The norm before a block, with what joins the residual stream there:
    ``sum = residual + scale x``, ``out = weight sum rstd(sum)`` over the
    channels of each position.  x, residual ``[N, D, L]`` (residual of x's type
    or fp32), weight and scale ``[D]`` fp32.  Returns (out of x's type, sum of
    the residual's); without a residual ``sum`` is ``scale x``."""
    f = (_native or native()).norm_pre_fwd
    args = (x, weight, residual, scale, eps, out)
    return f(*args) if stream is None else _on(stream, f, *args)


def norm_pre_bwd(dout, sum, weight, *, dsum=None, x=None, scale=None, eps=1e-6, stream=None):
    """:class:`NormPreGrads` of :func:`norm_pre_fwd` from the ``sum`` that it
    returned; ``dsum`` is the gradient that reaches ``sum`` from elsewhere (the
    residual stream).  ``x`` is needed where the call had a ``scale``."""
    f = (_native or native()).norm_pre_bwd
    args = (dout, sum, weight, dsum, x, scale, eps)
    return NormPreGrads(*(f(*args) if stream is None else _on(stream, f, *args)))


def norm_post_fwd(x, weight, *, gate=None, residual=None, scale=None, eps=1e-6, out=None, stream=None):
    """The norm after a block, with its gate and its way back to the residual
    stream: ``v = x gate sigmoid(gate)``, ``out = residual + scale weight v
    rstd(v)`` over the channels of each position.  x, gate, residual
    ``[N, D, L]`` (residual of x's type or fp32), weight and scale ``[D]``
    fp32.  Returns out, of the residual's type."""
    f = (_native or native()).norm_post_fwd
    args = (x, weight, gate, residual, scale, eps, out)
    return f(*args) if stream is None else _on(stream, f, *args)


def norm_post_bwd(dout, x, weight, *, gate=None, scale=None, eps=1e-6, stream=None):
    """:class:`NormPostGrads` of :func:`norm_post_fwd`, for ``dout`` of its
    output's type."""
    f = (_native or native()).norm_post_bwd
    args = (dout, x, weight, gate, scale, eps)
    return NormPostGrads(*(f(*args) if stream is None else _on(stream, f, *args)))
