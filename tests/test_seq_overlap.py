"""Results in the caller's memory: refused where they would overlap an input."""
import pytest
import torch

from paper_2101_09808_amd import seq
from tests.test_seq_ops import BF, F32, Gen, scan_inputs

pytestmark = pytest.mark.gpu


def refused(match, f, *a, **kw):
    with pytest.raises(ValueError, match=match):
        f(*a, **kw)


def test_out_over_an_input():
    G = Gen(41)
    N, D, L, S = 2, 6, 9, 4
    buf = G.n(2 * N * D * L)
    x, late = buf[:N * D * L].view(N, D, L), buf[D * L:(N + 1) * D * L].view(N, D, L)
    w, g = G.n(D, 4), G.n(D)
    refused("out overlaps x", seq.causal_conv_fwd, x, w, out=x)
    refused("out overlaps x", seq.causal_conv_fwd, x, w, out=late)
    refused("out overlaps initial_state", seq.causal_conv_fwd, buf[N * D * L:].view(N, D, L), w,
            initial_state=buf[:N * D * 3].view(N, D, 3), out=x)
    refused("out overlaps x", seq.norm_pre_fwd, x, g, out=x)
    refused("out overlaps residual", seq.norm_post_fwd, G.n(N, D, L), g, residual=late, out=x)
    v = scan_inputs(G, N, D, L, S, 2, F32, True, True, True, True)
    pos = [v[k] for k in ("u", "delta", "A", "B", "C")]
    refused("out overlaps u", seq.selective_scan_fwd, *pos, out=v["u"])
    refused("out overlaps z", seq.selective_scan_fwd, *pos, z=v["z"], out=v["z"])


def test_states_over_inputs():
    G = Gen(42)
    N, D, S = 2, 6, 4
    buf = G.n(N * D * 3 + 1)
    x, w, st = G.n(N, D), G.n(D, 4), buf[1:].view(N, D, 3)
    refused("new_state overlaps state", seq.causal_conv_step, x, st, w, new_state=buf[:-1].view(N, D, 3))
    refused("state overlaps x", seq.causal_conv_step, buf[:N * D].view(N, D), st, w)
    refused("out overlaps state", seq.causal_conv_step, x, st, w, out=buf[1:1 + N * D].view(N, D))
    new = torch.empty_like(st)
    refused("out overlaps new_state", seq.causal_conv_step, x, st, w, new_state=new,
            out=new.view(-1)[:N * D].view(N, D))
    v = scan_inputs(G, N, D, 1, S, 1, F32, False, True, False, True)
    u, delta, A, B, C = (v[k][..., 0] if v[k].dim() > 2 else v[k] for k in ("u", "delta", "A", "B", "C"))
    delta, h = delta.contiguous(), v["initial_state"]
    refused("state overlaps u", seq.selective_scan_step, h.view(-1)[:N * D].view(N, D), h, delta, A, B, C)
    refused("out overlaps delta", seq.selective_scan_step, u, h, delta, A, B, C, out=delta)


@pytest.mark.parametrize("t", [F32, BF])
def test_memory_between_an_inputs_slices_is_free(t):
    """A slice of a larger tensor spans memory that is not its own; results may lie there."""
    G = Gen(43)
    N, D, L = 2, 6, 40
    buf = G.n(N, 4 * D * L, dtype=t).view(-1)
    x = torch.as_strided(buf, (N, D, L), (4 * D * L, L, 1))
    out = buf[D * L:(N + 1) * D * L].view(N, D, L)
    w = G.n(D, 4)
    ref = seq.causal_conv_fwd(x.clone(), w)
    assert torch.equal(seq.causal_conv_fwd(x, w, out=out), ref) and out.data_ptr() == buf[D * L:].data_ptr()
    refused("out overlaps x", seq.causal_conv_fwd, x, w, out=buf[D * L - 1:(N + 1) * D * L - 1].view(N, D, L))


def test_a_states_other_view_is_the_state():
    G = Gen(44)
    x, w, st = G.n(3, 5), G.n(5, 4), G.n(3, 5, 3)
    keep = st.clone()
    new = torch.empty_like(st)
    ref = seq.causal_conv_step(x, keep, w, new_state=new)
    assert torch.equal(seq.causal_conv_step(x, st, w, new_state=st.view(3, 5, 3)), ref) and torch.equal(st, new)


def test_autograd_sees_what_is_written():
    """A tensor that autograd saved and a call wrote over raises in the backward
    pass, where it would give a gradient of other values."""
    G = Gen(45)
    x, w, st, out = G.n(3, 5), G.n(5, 4), G.n(3, 5, 3), torch.zeros(3, 5, device="cuda")
    p = torch.ones((), device="cuda", requires_grad=True)
    for t, f in ((st, lambda: seq.causal_conv_step(x, st, w)),
                 (st, lambda: seq.causal_conv_step(x, G.n(3, 5, 3), w, new_state=st)),
                 (out, lambda: seq.causal_conv_step(x, G.n(3, 5, 3), w, out=out))):
        y = (t * p).sum()
        f()
        with pytest.raises(RuntimeError, match="inplace"):
            y.backward()
    with torch.inference_mode():
        s2 = st.clone()
    seq.causal_conv_step(x, s2, w)
    (x * p).sum().backward()  # (inputs are as they were)
