"""Parity of the sequence operators with their 64-bit forms (oracle/seq.py).

Tolerances, set from the arithmetic before the first run.  A value that is
stored in type t is off by at most half a step of t (eps/2 relative) more than
the fp32 value it is rounded from.  That one is off by at most a count of
2^-24 steps of the magnitude it was summed from (the 64-bit form evaluated with
absolute values): one for every product and sum on the way to it, plus a few
for each exponential or reciprocal (an ulp each; a rounded exponent x counts
|x|).  For the scan the 64-bit form carries the bound along the recurrence.
"""
import pytest
import torch

from oracle import seq as O
from paper_2101_09808_amd import seq

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


def say(*a):
    print(*a, flush=True)


class Gen:
    def __init__(self, seed):
        self.g = torch.Generator().manual_seed(seed)

    def n(self, *shape, dtype=F32, scale=1.0):
        return (torch.randn(*shape, generator=self.g) * scale).to(dtype).to(DEV)

    def u(self, *shape):
        return torch.rand(*shape, generator=self.g).to(DEV)


def sliced(x):
    """The same values as a slice of a larger tensor, one element off alignment."""
    N, D = x.shape[:2]
    big = torch.full((N, D + 3) + tuple(x.shape[2:-1]) + (x.shape[-1] + 5,), float("nan"), dtype=x.dtype, device=x.device)
    v = big[:, 1:D + 1, ..., 1:1 + x.shape[-1]]
    v.copy_(x)
    return v


def check(name, got, ref, count, mag):
    """|got - ref| <= half a step of got's type + count * 2^-24 * mag."""
    assert got.shape == ref.shape, (name, got.shape, ref.shape)
    half = torch.finfo(got.dtype).eps / 2 if got.dtype != F32 else 0.0
    g = got.detach().double().cpu()
    tol = half * ref.abs() + (1 + half) * count * U * mag + 2.0 ** -126
    err = (g - ref).abs()
    bad = ~(err <= tol)
    assert not bad.any(), (f"{name}: {int(bad.sum())} of {bad.numel()} off, first at {bad.nonzero()[0].tolist()}, "
                           f"worst {float((err / tol).nan_to_num(9e9).max()):.3g} times the tolerance")


def spoil(x, lengths):
    """NaN behind each sequence's end, where nothing may be read."""
    if lengths is None:
        return x
    x = x.clone()
    for n, k in enumerate(lengths.tolist()):
        x[n, ..., max(0, min(k, x.shape[-1])):] = float("nan")
    return x


def lens_of(kind, N, L):
    if kind is None:
        return None
    v = {"ragged": [L, 0, 1, L - 1, L // 2 + 1, L + 7, -3], "ends": [127, 128, 129, 511, 512, 513, 8]}[kind]
    return torch.tensor([v[i % len(v)] for i in range(N)], dtype=torch.int32, device=DEV)


# --------------------------------------------------------- causal convolution

CONV = [  # N, D, L, R, dtype, activation, bias, states, lengths, sliced
    (1, 1, 1, 1, F32, None, False, False, None, False),
    (2, 3, 1, 4, BF, "silu", True, True, None, False),
    (7, 5, 9, 4, F32, "silu", True, True, "ragged", True),
    (7, 6, 37, 3, BF, None, True, True, "ragged", True),
    (2, 70, 512, 4, BF, "silu", True, False, None, False),
    (7, 3, 520, 2, F32, "silu", False, True, "ends", False),
    (3, 4, 1301, 8, BF, "silu", True, True, None, True),
    (7, 2, 600, 5, F32, None, True, True, "ends", True),
    (1, 2, 4099, 4, BF, "silu", True, True, None, False),
    (3, 1100, 64, 4, F32, "silu", True, False, None, False),
    (2, 5, 40, 6, F32, "silu", True, True, None, False),
    (2, 5, 41, 7, BF, "silu", True, True, None, False),
]


@pytest.mark.parametrize("case", CONV, ids=lambda c: "-".join(map(str, c)).replace("torch.", ""))
def test_causal_conv(case):
    N, D, L, R, t, act, has_b, states, lk, sl = case
    say("[gpu] causal_conv", case)
    G = Gen(1)
    x, w = G.n(N, D, L, dtype=t), G.n(D, R, scale=R ** -0.5)
    b = G.n(D) if has_b else None
    lengths = lens_of(lk, N, L)
    i0, df = (G.n(N, D, R - 1, dtype=t), G.n(N, D, R - 1, dtype=t)) if states else (None, None)
    do = G.n(N, D, L, dtype=t)
    x, do = spoil(x, lengths), spoil(do, lengths)
    if sl:
        x, do = sliced(x), sliced(do)
    kw = dict(activation=act, initial_state=i0, lengths=lengths)
    out, fin = seq.causal_conv_fwd(x, w, b, return_final_state=True, **kw)
    ref, rfin, mag = O.causal_conv(x, w, b, act, i0, lengths)
    # R products and sums, the sigmoid's exponent and four more roundings; the
    # slope of x sigmoid(x) stays below 1.1
    check("out", out, ref, 1.1 * (R + 1) + 16, mag)
    assert torch.equal(fin.double().cpu(), rfin)
    g = seq.causal_conv_bwd(do, x, w, b, dfinal_state=df, **kw)
    args = (do, x, w, b, act, i0, lengths, df)
    rg, mg = O.causal_conv_grads(*args), O.causal_conv_grads(*args, absolute=True)
    c = 3 * R + 32
    check("dx", g.dx, rg[0], c, mg[0])
    # (a sum over N L terms, of which a lane adds up to N L / 64 one by one)
    check("dweight", g.dweight, rg[1], c + 16 + N * L / 16, mg[1])
    if has_b:
        check("dbias", g.dbias, rg[2], c + 16 + N * L / 16, mg[2])
    if states:
        check("dinitial_state", g.dinitial_state, rg[3], c, mg[3])
    assert (g.dbias is None) == (not has_b) and (g.dinitial_state is None) == (not states)


@pytest.mark.parametrize("t", [F32, BF])
@pytest.mark.parametrize("R", [1, 2, 4, 8])
@pytest.mark.parametrize("N,D", [(1, 1), (3, 301)])
def test_causal_conv_step(t, R, N, D):
    say("[gpu] causal_conv_step", t, R, N, D)
    G = Gen(2)
    x, w, b = G.n(N, D, 3, dtype=t)[..., 1], G.n(D, R), G.n(D)
    state = G.n(N, D, R - 1, dtype=t)
    ref, rfin, mag = O.causal_conv(x[..., None], w, b, "silu", state)
    new = torch.empty_like(state)
    out = seq.causal_conv_step(x, state, w, b, activation="silu", new_state=new)
    check("out", out, ref[..., 0], 1.1 * (R + 1) + 16, mag[..., 0])
    assert torch.equal(new.double().cpu(), rfin)
    again = seq.causal_conv_step(x, state, w, b, activation="silu")  # in place
    assert torch.equal(again, out) and torch.equal(state, new)


# -------------------------------------------------------------- selective scan

SCAN = [  # N, D, L, S, G, dtype, gate, soft, D and bias, states, lengths, sliced
    (1, 1, 1, 1, 1, F32, False, False, False, False, None, False),
    (2, 5, 3, 16, 1, BF, True, True, True, True, None, False),
    (7, 6, 150, 4, 2, F32, True, True, True, True, "ragged", True),
    (7, 33, 140, 16, 1, BF, True, True, True, True, "ends", True),
    (2, 40, 128, 16, 1, F32, False, True, True, False, None, False),
    (1, 70, 300, 17, 1, BF, True, True, True, True, None, True),
    (2, 24, 129, 64, 3, F32, True, True, True, True, None, False),
    (1, 36, 70, 64, 1, BF, True, True, True, True, None, False),
    (1, 36, 70, 40, 1, F32, True, True, False, True, None, False),
    (3, 18, 1000, 3, 1, F32, False, True, True, True, "ragged", False),
    (1, 8, 2100, 8, 2, BF, True, True, True, True, None, False),
    (7, 4, 700, 16, 1, F32, True, True, True, True, "ends", False),
    (7, 4, 2600, 16, 1, BF, True, True, True, True, "ragged", True),
    (3, 1400, 650, 5, 1, F32, True, True, True, True, "ragged", False),
    (2, 70, 2100, 33, 1, BF, True, True, True, True, "ends", False),
]


def scan_inputs(G, N, D, L, S, Gr, t, gate, soft, extra, states):
    v = {"u": G.n(N, D, L, dtype=t), "delta": G.n(N, D, L, dtype=t, scale=0.5)}
    if not soft:
        v["delta"] = v["delta"].abs() * 0.1
    v["A"] = -torch.arange(1, S + 1, device=DEV, dtype=F32) * (0.5 + G.u(D, 1))
    v["B"], v["C"] = G.n(N, Gr, S, L, dtype=t), G.n(N, Gr, S, L, dtype=t)
    v["z"] = G.n(N, D, L, dtype=t) if gate else None
    v["D"], v["delta_bias"] = (G.n(D), -4 * G.u(D) - 1) if extra else (None, None)
    v["initial_state"] = G.n(N, D, S) if states else None
    return v


def scan_tolerance(L, S):
    """Counts for the gradients: a state or its gradient has at most L steps
    behind it, each with 8 roundings (3 for the decay, whose exponent is a few at
    most, 5 products and sums); S states are summed, and 40 for an element's
    functions."""
    return 40 + 8 * L + S


@pytest.mark.parametrize("case", SCAN, ids=lambda c: "-".join(map(str, c)).replace("torch.", ""))
def test_selective_scan(case):
    N, D, L, S, Gr, t, gate, soft, extra, states, lk, sl = case
    say("[gpu] selective_scan", case)
    G = Gen(3)
    v = scan_inputs(G, N, D, L, S, Gr, t, gate, soft, extra, states)
    lengths = lens_of(lk, N, L)
    do, df = G.n(N, D, L, dtype=t), G.n(N, D, S)
    for k in ("u", "delta", "B", "C", "z"):
        if v[k] is not None:
            v[k] = spoil(v[k], lengths)
            v[k] = sliced(v[k]) if sl else v[k]
    do = spoil(do, lengths)
    pos = [v[k] for k in ("u", "delta", "A", "B", "C")]
    kw = dict(D=v["D"], z=v["z"], delta_bias=v["delta_bias"], delta_softplus=soft, lengths=lengths)
    out, fin, chk = seq.selective_scan_fwd(*pos, initial_state=v["initial_state"], return_final_state=True,
                                           return_checkpoints=True, **kw)
    ref, rfin, _, _, bound, fbound = O.selective_scan(*pos, v["D"], v["z"], v["delta_bias"], soft, v["initial_state"],
                                                      lengths)
    check("out", out, ref, 1.0, bound)
    check("final_state", fin, rfin, 1.0, fbound)
    g = seq.selective_scan_bwd(do, *pos, chk, dfinal_state=df, **kw)
    args = (do, *pos, v["D"], v["z"], v["delta_bias"], soft, v["initial_state"], lengths, df)
    rg, mg = O.selective_scan_grads(*args), O.selective_scan_grads(*args, absolute=True)
    c = scan_tolerance(L, S)
    names = ("du", "ddelta", "dA", "dB", "dC", "dD", "ddelta_bias", "dz", "dinitial_state")
    have = (1, 1, 1, 1, 1, extra, extra, gate, 1)
    for name, got, r, m, h in zip(names, g, rg, mg, have):
        assert (got is None) == (not h), name
        if h:
            many = D / Gr if name in ("dB", "dC") else N * L / 16 if name in ("dA", "dD", "ddelta_bias") else 0
            check(name, got, r, c + many, m)
    # the same bits again
    out2 = seq.selective_scan_fwd(*pos, initial_state=v["initial_state"], **kw)
    g2 = seq.selective_scan_bwd(do, *pos, chk, dfinal_state=df, **kw)
    assert torch.equal(out, out2) and all(a is b or torch.equal(a, b) for a, b in zip(g, g2))


@pytest.mark.parametrize("t", [F32, BF])
@pytest.mark.parametrize("N,D,S,Gr", [(1, 1, 1, 1), (3, 70, 16, 2), (2, 33, 7, 1), (2, 9, 64, 3), (1, 5, 21, 1),
                                      (301, 1900, 16, 1), (301, 3801, 3, 1)])
def test_selective_scan_step(t, N, D, S, Gr):
    say("[gpu] selective_scan_step", t, N, D, S, Gr)
    G = Gen(4)
    v = scan_inputs(G, N, D, 3, S, Gr, t, True, True, True, True)
    state = v["initial_state"]
    cur = {k: v[k][..., 1] if N < 300 else v[k][..., 1].contiguous() for k in ("u", "delta", "B", "C", "z")}
    ref, rfin, _, _, bound, fbound = O.selective_scan(
        *(cur[k][..., None] if k != "A" else v["A"] for k in ("u", "delta", "A", "B", "C")), v["D"],
        cur["z"][..., None], v["delta_bias"], True, state)
    new = torch.empty_like(state)
    args = (cur["u"], state, cur["delta"], v["A"], cur["B"], cur["C"])
    kw = dict(D=v["D"], z=cur["z"], delta_bias=v["delta_bias"], delta_softplus=True)
    out = seq.selective_scan_step(*args, new_state=new, **kw)
    check("out", out, ref[..., 0], 1.0, bound[..., 0])
    check("state", new, rfin, 1.0, fbound)
    again = seq.selective_scan_step(*args, **kw)  # in place
    assert torch.equal(again, out) and torch.equal(state, new)


def test_scan_in_parts_is_the_whole():
    """A prompt in two calls and then single tokens gives what one call gives."""
    G = Gen(5)
    N, D, L, S, R = 2, 24, 300, 16, 4
    v = scan_inputs(G, N, D, L, S, 1, F32, True, True, True, False)
    w, b = G.n(D, R), G.n(D)
    kw = dict(D=v["D"], delta_bias=v["delta_bias"], delta_softplus=True)

    def layer(cut, conv_state, state):
        x, cs = seq.causal_conv_fwd(v["u"][..., cut], w, b, activation="silu", initial_state=conv_state,
                                    return_final_state=True)
        o, st = seq.selective_scan_fwd(x, v["delta"][..., cut], v["A"], v["B"][..., cut], v["C"][..., cut],
                                       z=v["z"][..., cut], initial_state=state, return_final_state=True, **kw)
        return o, cs, st

    whole, cs, st = layer(slice(0, L), None, None)
    x_ref, _, mag = O.causal_conv(v["u"], w, b, "silu")
    ref, rst, _, _, bound, fbound = O.selective_scan(x_ref, v["delta"], v["A"], v["B"], v["C"], v["D"], v["z"],
                                                     v["delta_bias"], True)
    parts, c2, s2 = layer(slice(0, 131), None, None)
    parts = [parts]
    o, c2, s2 = layer(slice(131, 296), c2, s2)
    parts.append(o)
    for i in range(296, L):
        x = seq.causal_conv_step(v["u"][..., i], c2, w, b, activation="silu")
        parts.append(seq.selective_scan_step(x, s2, v["delta"][..., i], v["A"], v["B"][..., i], v["C"][..., i],
                                             z=v["z"][..., i], **kw)[..., None])
    got = torch.cat(parts, -1)
    # the convolution's output is off by (1.1 (R + 1) + 16) steps, which pass
    # through the scan like dt's in x, of which its bound counts eight and more
    grow = (2 + (1.1 * (R + 1) + 16) * float((mag / x_ref.abs().clamp(min=1e-3)).max()) / 8)
    for o, s in ((whole, st), (got, s2)):
        check("out", o, ref, grow, bound)
        check("state", s, rst, grow, fbound)
    assert torch.equal(c2, cs)


# ------------------------------------------------------------------------ norms

NORM = [  # N, D, L, dtype, residual dtype, residual, scale, gate, sliced
    (1, 1, 1, F32, F32, False, False, False, False),
    (3, 300, 1, BF, F32, True, True, True, False),
    (2, 2050, 1, BF, BF, True, True, True, True),
    (2, 77, 7, F32, F32, True, True, True, True),
    (2, 300, 15, BF, BF, True, False, True, False),
    (2, 100, 16, BF, F32, True, True, True, True),
    (3, 64, 33, F32, F32, False, True, False, False),
    (1, 1500, 90, BF, BF, True, True, True, True),
    (2, 4100, 40, F32, F32, True, True, True, False),
    (30, 20, 600, BF, F32, True, True, False, False),
    (2, 9000, 17, BF, BF, False, False, False, False),
    (1, 2600, 5, BF, F32, True, True, True, True),
    (2, 1100, 15, F32, F32, True, True, True, False),
    (3, 4097, 1, BF, BF, True, True, True, False),
    (2, 1100, 129, F32, F32, True, True, True, True),
    (200, 300, 3, BF, BF, True, True, True, False),
    (600, 30, 2, F32, F32, True, True, True, False),
]


@pytest.mark.parametrize("case", NORM, ids=lambda c: "-".join(map(str, c)).replace("torch.", ""))
def test_norms(case):
    N, D, L, t, rt, has_r, has_s, has_g, sl = case
    say("[gpu] norms", case)
    G = Gen(6)
    x, w = G.n(N, D, L, dtype=t), 1 + 0.1 * G.n(D)
    res = G.n(N, D, L, dtype=rt) if has_r else None
    sc = G.n(D) if has_s else None
    gate = G.n(N, D, L, dtype=t) if has_g else None
    x[:, :, L // 2] = 0  # a position without a value
    if has_r:
        res[:, :, L // 2] = 0
    if sl:
        x, res, gate = sliced(x), sliced(res) if has_r else None, sliced(gate) if has_g else None
    c = 40 + D / 64  # sums of squares are of one sign; the rest is a dozen steps
    y, r = seq.norm_pre_fwd(x, w, residual=res, scale=sc)
    ry, rr = O.norm_pre(x, w, res, sc)
    mag = O.norm_pre(x.abs(), w, res.abs() if has_r else None, sc.abs() if has_s else None)
    check("sum", r, rr, 4, mag[1])
    rstd = 1 / (rr.square().mean(1, keepdim=True) + 1e-6).sqrt()
    check("out", y, ry, c, mag[1] * rstd * O.d(w)[:, None].abs() + ry.abs())
    do, ds = G.n(N, D, L, dtype=t), G.n(N, D, L, dtype=r.dtype)
    if sl:
        do, ds = sliced(do), sliced(ds)
    g = seq.norm_pre_bwd(do, r, w, dsum=ds, x=x if has_s else None, scale=sc)
    args = (do, r, w, ds, x if has_s else None, sc)
    rg, mg = O.norm_pre_grads(*args), O.norm_pre_grads(*args, absolute=True)
    for name, got, ref, m, n in zip(g._fields, g, rg, mg, (c, c, c + N * L / 4, c + N * L / 4)):
        assert (got is None) == (ref is None)
        if got is not None:
            check(name, got, ref, n, m)
    o = seq.norm_post_fwd(x, w, gate=gate, residual=res, scale=sc)
    ro = O.norm_post(x, w, gate, res, sc)
    assert o.dtype == (rt if has_r else t)
    check("post", o, ro, c, O.norm_post(x, w, gate, None, sc).abs() + (O.d(res).abs() if has_r else 0))
    do = G.n(N, D, L, dtype=o.dtype)
    g = seq.norm_post_bwd(do, x, w, gate=gate, scale=sc)
    args = (do, x, w, gate, sc)
    rg, mg = O.norm_post_grads(*args), O.norm_post_grads(*args, absolute=True)
    for name, got, ref, m, n in zip(g._fields, g, rg, mg, (c, c, c + N * L / 4, c + N * L / 4)):
        if got is not None:
            check(name, got, ref, n, m)
    assert (g.dgate is None) == (not has_g) and (g.dscale is None) == (not has_s)
