"""How the sequence operators are used: refusals of tensors that do not fit, a
layer of them together, captured graphs, other streams, far offsets."""
import pytest
import torch

from oracle import seq as O
from paper_2101_09808_amd import conv, seq
from tests.test_seq_ops import BF, DEV, F32, Gen, check, say, scan_inputs

pytestmark = pytest.mark.gpu


# -------------------------------------------------------------------- refusals

def refused(exc, match, f, *a, **kw):
    with pytest.raises(exc, match=match):
        f(*a, **kw)


def test_conv_refusals():
    G = Gen(11)
    x, w, s = G.n(2, 6, 9), G.n(6, 4), G.n(2, 6, 3)
    f = seq.causal_conv_fwd
    refused(TypeError, "weight must be float32", f, x, w.to(BF))
    refused(TypeError, "x must be float32 or bfloat16", f, x.half(), w)
    refused(TypeError, "x must be float32 or bfloat16", f, x.double(), w)
    refused(ValueError, "3 dimensions", f, x[0], w)
    refused(ValueError, "empty", f, x[:, :, :0], w)
    refused(ValueError, "R of 1 to 8", f, x, G.n(6, 9))
    refused(ValueError, "R of 1 to 8", f, x, G.n(6, 4, 1))
    refused(ValueError, "weight must be", f, x, G.n(5, 4))
    refused(ValueError, "weight must be contiguous", f, x, G.n(4, 6).t())
    refused(ValueError, "bias must be", f, x, w, G.n(5))
    refused(ValueError, "stride 1", f, G.n(2, 9, 6).transpose(1, 2), w)
    refused(ValueError, "activation", f, x, w, activation="relu")
    refused(TypeError, "lengths must be int32", f, x, w, lengths=torch.ones(2, dtype=torch.int64, device=DEV))
    refused(ValueError, "lengths must be", f, x, w, lengths=torch.ones(3, dtype=torch.int32, device=DEV))
    refused(ValueError, "lengths must be on", f, x, w, lengths=torch.ones(2, dtype=torch.int32))
    refused(ValueError, "initial_state must be", f, x, w, initial_state=G.n(2, 6, 4))
    refused(TypeError, "initial_state must be", f, x, w, initial_state=s.to(BF))
    refused(ValueError, "out must be", f, x, w, out=G.n(2, 6, 8))
    refused(ValueError, "out must be contiguous", f, x, w, out=G.n(2, 9, 6).transpose(1, 2))
    refused(TypeError, "dout must be", seq.causal_conv_bwd, x.to(BF), x, w)
    refused(ValueError, "dfinal_state must be", seq.causal_conv_bwd, x, x, w, dfinal_state=x)
    refused(ValueError, "state must be", seq.causal_conv_step, x[..., 0], x, w)
    refused(ValueError, "new_state must be contiguous", seq.causal_conv_step, x[..., 0], s, w,
            new_state=G.n(2, 3, 6).transpose(1, 2))


def test_scan_refusals():
    G = Gen(12)
    v = scan_inputs(G, 2, 6, 9, 4, 2, F32, True, True, True, True)
    pos = [v[k] for k in ("u", "delta", "A", "B", "C")]

    def f(i=None, t=None, **kw):
        a = list(pos)
        if i is not None:
            a[i] = t
        return seq.selective_scan_fwd(*a, **kw)

    refused(ValueError, "delta must be", f, 1, v["delta"][..., :8])
    refused(TypeError, "A must be float32", f, 2, v["A"].to(BF))
    refused(ValueError, "S of 1 to 64", f, 2, G.n(6, 65))
    refused(ValueError, "B must be \\[N, G, S, L\\]", f, 3, v["u"])
    refused(ValueError, "do not divide", f, 3, G.n(2, 4, 4, 9))
    refused(ValueError, "C must be", f, 4, v["C"][:, :1])
    refused(TypeError, "C must be", f, 4, v["C"].to(BF))
    refused(ValueError, "stride 1", f, 4, G.n(2, 2, 9, 4).transpose(2, 3))
    refused(ValueError, "D must be", f, D=G.n(5))
    refused(ValueError, "z must be", f, z=v["z"][:1])
    refused(TypeError, "initial_state must be float32", f, initial_state=v["initial_state"].to(BF))
    out, chk = f(return_checkpoints=True)
    refused(ValueError, "checkpoints must be", seq.selective_scan_bwd, out, *pos, chk[:, :, :5].contiguous())
    refused(ValueError, "dfinal_state must be", seq.selective_scan_bwd, out, *pos, chk, dfinal_state=chk)
    one = [t[..., 0] if t.dim() > 2 else t for t in pos]
    refused(ValueError, "state must be", seq.selective_scan_step, one[0], chk, *one[1:])
    refused(ValueError, "B must be \\[N, G, S\\]", seq.selective_scan_step, one[0], v["initial_state"], one[1], one[2],
            pos[3], one[4])


def test_norm_refusals():
    G = Gen(13)
    x, w = G.n(2, 6, 9), G.n(6)
    refused(ValueError, "weight must be", seq.norm_pre_fwd, x, G.n(5))
    refused(TypeError, "residual's type", seq.norm_pre_fwd, x, w, residual=x.to(BF))
    refused(TypeError, "residual's type", seq.norm_post_fwd, x.to(BF), w, residual=x.double())
    refused(ValueError, "residual must be", seq.norm_pre_fwd, x, w, residual=x[:1])
    refused(ValueError, "eps", seq.norm_pre_fwd, x, w, eps=-1e-6)
    refused(ValueError, "eps", seq.norm_post_fwd, x, w, eps=float("nan"))
    refused(TypeError, "gate must be", seq.norm_post_fwd, x, w, gate=x.to(BF))
    refused(ValueError, "x is needed", seq.norm_pre_bwd, x, x, w, scale=w)
    refused(ValueError, "dsum must be", seq.norm_pre_bwd, x, x, w, dsum=x[..., 1:])
    refused(TypeError, "dout must be", seq.norm_post_bwd, None, x, w)


# ----------------------------------------------------------- a layer of them

def layer_inputs(G, N, K, D, S, R, L, t):
    p = {"win": G.n(2 * D, K, 1, 1, dtype=t, scale=K ** -0.5), "wbc": G.n(2 * S, D, 1, 1, dtype=t, scale=D ** -0.5),
         "wdt": G.n(D, D, 1, 1, dtype=t, scale=D ** -0.5), "conv_w": G.n(D, R, scale=0.5), "conv_b": G.n(D),
         "A": -(1 + torch.arange(S, device=DEV, dtype=F32)).expand(D, S).contiguous(), "D": G.n(D),
         "bias": -2 - G.u(D), "n1": 1 + 0.1 * G.n(K), "n2": 1 + 0.1 * G.n(D)}
    return p, G.n(N, K, L, dtype=t), G.n(N, K, L, dtype=F32)


def pointwise(x, w):
    """A pointwise convolution over the channels of [N, C, L], on the framework's own kernels."""
    f = conv.conv_fwd_bf16_out if x.dtype == BF else conv.conv_fwd
    return f(x.contiguous()[:, :, None], w)[:, :, 0]


def layer_fwd(p, x, res, save=False):
    """A state-space block up to its projection back: norm, projection, causal
    convolution, scan, gated norm."""
    h, s = seq.norm_pre_fwd(x, p["n1"], residual=res)
    xz = pointwise(h, p["win"])
    D = xz.shape[1] // 2
    xi, z = xz[:, :D], xz[:, D:]
    u, cs = seq.causal_conv_fwd(xi, p["conv_w"], p["conv_b"], activation="silu", return_final_state=True)
    bc, delta = pointwise(u, p["wbc"]), pointwise(u, p["wdt"])
    S = bc.shape[1] // 2
    B, C = bc[:, None, :S], bc[:, None, S:]
    args = (u, delta, p["A"], B, C)
    kw = dict(D=p["D"], delta_bias=p["bias"], delta_softplus=True)
    y, st, chk = seq.selective_scan_fwd(*args, return_final_state=True, return_checkpoints=True, **kw)
    out = seq.norm_post_fwd(y, p["n2"], gate=z)
    if not save:
        return out, s, cs, st
    return out, dict(x=xi, z=z, args=args, kw=kw, chk=chk, y=y, s=s, h=h)


def layer_step(p, x, res, cs, st):
    """One token of it; the states are updated in place."""
    h, s = seq.norm_pre_fwd(x[..., None], p["n1"], residual=res[..., None])
    xz = pointwise(h, p["win"])[..., 0]
    D = xz.shape[1] // 2
    u = seq.causal_conv_step(xz[:, :D], cs, p["conv_w"], p["conv_b"], activation="silu")
    bc, delta = pointwise(u[..., None], p["wbc"])[..., 0], pointwise(u[..., None], p["wdt"])[..., 0]
    S = bc.shape[1] // 2
    y = seq.selective_scan_step(u, st, delta, p["A"], bc[:, None, :S], bc[:, None, S:], D=p["D"],
                                delta_bias=p["bias"], delta_softplus=True)
    return seq.norm_post_fwd(y[..., None], p["n2"], gate=xz[:, D:, None])[..., 0], s[..., 0]


def test_a_layer_token_by_token_is_the_layer():
    """fp32: what a prompt's layer gives at its last positions, single tokens
    give from the states that a shorter prompt left.  Both are within their own
    rounding of one another: a few hundred steps of 2^-24, through four operators
    and three projections whose values are of order one to ten."""
    G = Gen(14)
    p, x, res = layer_inputs(G, 2, 32, 48, 16, 4, 150, F32)
    whole = layer_fwd(p, x, res)
    _, _, cs, st = layer_fwd(p, x[..., :146], res[..., :146])
    for i in range(146, 150):
        o, s = layer_step(p, x[..., i], res[..., i], cs, st)
        for got, ref in ((o, whole[0][..., i]), (s, whole[1][..., i])):
            assert (got - ref).abs().max() <= 2e-4 * ref.abs().max()
    for got, ref in ((cs, whole[2]), (st, whole[3])):
        assert (got - ref).abs().max() <= 2e-4 * ref.abs().max()


def layer_bwd(p, do, sv):
    g2 = seq.norm_post_bwd(do, sv["y"], p["n2"], gate=sv["z"])
    gs = seq.selective_scan_bwd(g2.dx, *sv["args"], sv["chk"], **sv["kw"])
    gc = seq.causal_conv_bwd(gs.du, sv["x"], p["conv_w"], p["conv_b"], activation="silu")
    g1 = seq.norm_pre_bwd(sv["h"], sv["s"], p["n1"])  # (any gradient of its type)
    return [t for g in (g2, gs, gc, g1) for t in g if t is not None]


def test_chained_gradients_against_differences():
    """The gradient of the chain convolution -> scan -> gated norm along a random
    direction, against the difference of fp32 losses in 64 bits.  Step 1e-2: the
    difference's own error is its third derivative times 1e-4 / 6, and rounding
    2^-24 of values of order ten over a step, below 1e-3 of the gradient's norm
    each."""
    G = Gen(15)
    N, D, S, L = 2, 24, 16, 140
    x, delta, z = G.n(N, D, L), G.n(N, D, L, scale=0.5), G.n(N, D, L)
    B, C = G.n(N, 1, S, L), G.n(N, 1, S, L)
    w, b, n2 = G.n(D, 4, scale=0.5), G.n(D), 1 + 0.1 * G.n(D)
    A = -(1 + torch.arange(S, device=DEV, dtype=F32)).expand(D, S).contiguous()
    bias, cot = -2 - G.u(D), G.n(N, D, L)
    kw = dict(D=b, delta_bias=bias, delta_softplus=True)

    def f(x, delta, B, C, z, save=False):
        u = seq.causal_conv_fwd(x, w, b, activation="silu")
        y, chk = seq.selective_scan_fwd(u, delta, A, B, C, return_checkpoints=True, **kw)
        return (seq.norm_post_fwd(y, n2, gate=z), u, y, chk)

    out, u, y, chk = f(x, delta, B, C, z)
    g2 = seq.norm_post_bwd(cot, y, n2, gate=z)
    gs = seq.selective_scan_bwd(g2.dx, u, delta, A, B, C, chk, **kw)
    gc = seq.causal_conv_bwd(gs.du, x, w, b, activation="silu")
    grads, ins = (gc.dx, gs.ddelta, gs.dB, gs.dC, g2.dgate), (x, delta, B, C, z)
    h = 1e-2
    for i in range(len(ins)):
        v = G.n(*ins[i].shape)
        v = v / v.norm()
        val = [(f(*[t + s * h * v if j == i else t for j, t in enumerate(ins)])[0].double() * cot.double()).sum()
               for s in (1, -1)]
        diff, lin = float(val[0] - val[1]) / (2 * h), float((grads[i].double() * v.double()).sum())
        assert abs(diff - lin) <= 2e-3 * float(grads[i].double().norm()), (i, diff, lin)


# ------------------------------------------------------------- graphs, streams

def test_captured_layer_replays_to_the_eager_results():
    """A layer forward and backward in one graph, replayed with new inputs,
    between eager calls of other sizes; a second graph of a longer layer beside
    it (scratch is each graph's own)."""
    G = Gen(16)
    p, x, res = layer_inputs(G, 2, 32, 40, 16, 4, 200, BF)
    p2, x2, res2 = layer_inputs(G, 1, 32, 16, 16, 4, 2600, BF)  # (few rows: scans in segments)

    def both(p, x, res):
        out, sv = layer_fwd(p, x, res, save=True)
        return [out, sv["s"], sv["chk"], *layer_bwd(p, out, sv)]

    s = torch.cuda.Stream()
    graphs = []
    for args in ((p, x, res), (p2, x2, res2)):
        with torch.cuda.stream(s):
            both(*args)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            outs = both(*args)
        graphs.append((g, args, outs))
    for k in range(4):
        for g, args, outs in graphs:
            args[1].copy_(G.n(*args[1].shape, dtype=BF))
            args[2].copy_(G.n(*args[2].shape))
        for g, _, _ in graphs:
            g.replay()
        torch.cuda.synchronize()
        seq.norm_post_bwd(G.n(3, 50, 70), G.n(3, 50, 70), G.n(50))  # (eager work in between)
        for g, args, outs in graphs:
            for got, ref in zip(outs, both(*args)):
                assert torch.equal(got, ref), k


def test_streams():
    """A call on a stream that is not the current one runs there, and its inputs
    may be freed at once."""
    G = Gen(17)
    x, w = G.n(4, 512, 1024), G.n(512, 4)
    ref = seq.causal_conv_fwd(x, w)
    rs = seq.norm_pre_fwd(x, w[:, 0].contiguous())[0]
    s = torch.cuda.Stream()
    for _ in range(3):
        xc = x.clone()
        s.wait_stream(torch.cuda.current_stream())
        out = seq.causal_conv_fwd(xc, w, stream=s)
        y = seq.norm_pre_fwd(xc, w[:, 0].contiguous(), stream=s)[0]
        del xc
        junk = torch.full_like(x, float("nan"))
        s.synchronize()
        assert torch.equal(out, ref) and torch.equal(y, rs)
        del junk
    with torch.cuda.stream(s):
        out = seq.causal_conv_fwd(x, w)
    s.synchronize()
    assert torch.equal(out, ref)


def test_out_buffers():
    G = Gen(18)
    x, w, n = G.n(2, 6, 9), G.n(6, 4), G.n(6)
    v = scan_inputs(G, 2, 6, 9, 4, 2, F32, True, True, True, True)
    pos = [v[k] for k in ("u", "delta", "A", "B", "C")]
    one = [t[..., 0] if t.dim() > 2 else t for t in pos]
    for f in (lambda o: seq.causal_conv_fwd(x, w, out=o), lambda o: seq.selective_scan_fwd(*pos, out=o),
              lambda o: seq.norm_post_fwd(x, n, out=o)):
        o = torch.empty_like(x)
        assert f(o).data_ptr() == o.data_ptr() and torch.equal(o, f(None))
    o = torch.empty_like(x)
    assert seq.norm_pre_fwd(x, n, out=o)[0].data_ptr() == o.data_ptr()
    o = torch.empty(2, 6, device=DEV)
    st = v["initial_state"]
    r = seq.selective_scan_step(one[0], st, *one[1:], new_state=torch.empty_like(st), out=o)
    assert r.data_ptr() == o.data_ptr()


def test_leaves_that_require_gradients_are_read_as_they_are():
    x, w = torch.randn(2, 4, 8, device=DEV, requires_grad=True), torch.randn(4, 3, device=DEV, requires_grad=True)
    out = seq.causal_conv_fwd(x, w)
    assert not out.requires_grad
    assert torch.equal(out, seq.causal_conv_fwd(x.detach(), w.detach()))


# --------------------------------------------------------------- far addresses

def test_inputs_past_32_bit_offsets():
    """Sequences 2^31 elements apart: the same results as from dense tensors."""
    G = Gen(19)
    N, D, L, S = 2, 20, 300, 8
    far = torch.empty((1 << 31) + 200000, dtype=BF, device=DEV)

    def put(t, off):
        n = t[0].numel()
        v = far.as_strided(t.shape, ((1 << 31) + 8, *t.stride()[1:]), off)
        v.copy_(t)
        return v, off + n

    v = scan_inputs(G, N, D, L, S, 1, BF, True, True, True, False)
    do = G.n(N, D, L, dtype=BF)
    off, w = 0, {}
    for k, t in (("u", v["u"]), ("delta", v["delta"]), ("B", v["B"]), ("C", v["C"]), ("z", v["z"]), ("do", do)):
        w[k], off = put(t.contiguous(), off)
    near = dict(v, do=do)
    wt, b = G.n(D, 4), G.n(D)

    def run(q):
        kw = dict(D=v["D"], z=q["z"], delta_bias=v["delta_bias"], delta_softplus=True)
        pos = (q["u"], q["delta"], v["A"], q["B"], q["C"])
        o, chk = seq.selective_scan_fwd(*pos, return_checkpoints=True, **kw)
        res = [o, *seq.selective_scan_bwd(q["do"], *pos, chk, **kw)]
        res += [seq.causal_conv_fwd(q["u"], wt, b), *seq.causal_conv_bwd(q["do"], q["u"], wt, b)]
        y, s = seq.norm_pre_fwd(q["u"], b, residual=q["z"])
        res += [y, s, seq.norm_post_fwd(q["u"], b, gate=q["z"], residual=q["delta"])]
        res += [*seq.norm_post_bwd(q["do"], q["u"], b, gate=q["z"]), *seq.norm_pre_bwd(q["do"], q["u"], b, dsum=q["z"])]
        res += [*seq.norm_pre_fwd(q["u"][..., :5], b, residual=q["z"][..., :5])]
        return res

    for a, r in zip(run(w), run(near)):
        assert (a is None and r is None) or torch.equal(a, r)


def test_outputs_past_32_bit_offsets():
    """2^31 elements and more in one call: its last rows are those of a call of their own."""
    D, L = 70000, 30688
    x = torch.empty((1, D, L), dtype=BF, device=DEV)
    G = Gen(20)
    tail = G.n(1, 3, L, dtype=BF)
    x[:, -3:] = tail
    x[:, :-3] = 1
    w, b = G.n(D, 4), G.n(D)
    say("[gpu] causal_conv", tuple(x.shape))
    out = seq.causal_conv_fwd(x, w, b, activation="silu")
    assert torch.equal(out[:, -3:], seq.causal_conv_fwd(tail, w[-3:].contiguous(), b[-3:].contiguous(), activation="silu"))
    dx = seq.causal_conv_bwd(out, x, w, b, activation="silu").dx
    ref = seq.causal_conv_bwd(out[:, -3:], tail, w[-3:].contiguous(), b[-3:].contiguous(), activation="silu").dx
    assert torch.equal(dx[:, -3:], ref)


# ------------------------------------------------------------- values that break

def test_infinities_and_nans_stay_where_they_are():
    """A NaN or infinity at a step changes that step and later ones of its own
    channel only (in dB and dC: that step's sums over the channels)."""
    G = Gen(21)
    v = scan_inputs(G, 1, 9, 300, 16, 1, F32, True, True, True, False)
    pos = [v[k] for k in ("u", "delta", "A", "B", "C")]
    kw = dict(D=v["D"], z=v["z"], delta_bias=v["delta_bias"], delta_softplus=True)
    ref = seq.selective_scan_fwd(*pos, **kw)
    for bad in (float("nan"), float("inf")):
        u = v["u"].clone()
        u[0, 4, 200] = bad
        out = seq.selective_scan_fwd(u, *pos[1:], **kw)
        keep = torch.ones_like(out, dtype=torch.bool)
        keep[0, 4, 200:] = False
        assert torch.equal(out[keep], ref[keep]) and not torch.isfinite(out[0, 4, 200])
    x = G.n(1, 6, 40)
    w = G.n(6, 4)
    ref = seq.causal_conv_fwd(x, w)
    x[0, 2, 20] = float("nan")
    out = seq.causal_conv_fwd(x, w)
    keep = torch.ones_like(out, dtype=torch.bool)
    keep[0, 2, 20:24] = False
    assert torch.equal(out[keep], ref[keep]) and torch.isnan(out[0, 2, 20:24]).all()


def test_large_steps_and_dead_states():
    """Steps so large that every decay underflows, and softplus arguments of both
    signs far from zero."""
    G = Gen(22)
    N, D, L, S = 1, 8, 260, 16
    v = scan_inputs(G, N, D, L, S, 1, F32, False, True, False, True)
    v["delta"] = 40 * G.n(N, D, L)
    pos = [v[k] for k in ("u", "delta", "A", "B", "C")]
    out, fin = seq.selective_scan_fwd(*pos, delta_softplus=True, initial_state=v["initial_state"],
                                      return_final_state=True)
    ref, rfin, _, _, bound, fbound = O.selective_scan(*pos, None, None, None, True, v["initial_state"])
    check("out", out, ref, 1.0, bound)
    check("final", fin, rfin, 1.0, fbound)
