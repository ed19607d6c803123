"""The kernels' instances that ordinary training steps and long prompts take: each
case states the route that the shape rules have to give it."""
import pytest
import torch

from oracle import seq as O
from paper_2101_09808_amd import seq
from tests import seq_shapes
from tests.test_seq_bounds import NAMES
from tests.test_seq_ops import BF, DEV, F32, Gen, check, say, scan_inputs, spoil

# N, D, L, S, G, type, gate, lengths; the forward and the backward route
SCAN = [
    # 16 steps a lane in segments cut into pieces; eight waves over segments of several chunks
    ((2, 320, 4200, 11, 16, BF, True, (4200, 1999)), dict(rows=4, steps=16, segs=6, seg_chunks=6, fine=2),
     dict(waves=8, segs=7, seg_chunks=5, fine=2, fine_chunks=3, batch=16)),
    ((1, 64, 8300, 5, 64, F32, True, None), dict(steps=16, segs=7, fine=4),
     dict(waves=4, segs=8, seg_chunks=9, fine=4)),
    # eight waves, whole sequences of several chunks, for each batch of states
    ((65, 64, 300, 16, 1, F32, True, (300, 129, 0, 77)), dict(rows=4, steps=8, segs=1),
     dict(waves=8, segs=1, chunks=3, batch=16)),
    ((65, 64, 300, 9, 1, BF, True, None), dict(rows=4, segs=1), dict(waves=8, segs=1, chunks=3, batch=16)),
    ((65, 64, 300, 21, 1, F32, True, None), dict(rows=4, segs=1), dict(waves=8, segs=1, chunks=3, batch=8)),
    ((65, 64, 150, 40, 2, BF, False, None), dict(rows=4, waves=8, segs=1), dict(waves=8, segs=1, chunks=2, batch=4)),
    # a channel a wave over three passes; segments of two chunks
    ((2, 520, 1030, 8, 2, F32, False, None), dict(rows=1, segs=1, chunks=9), dict(waves=8, segs=5, seg_chunks=2)),
    # segments of one chunk: sums of parameters' gradients over many of them
    ((7, 4, 2600, 16, 1, BF, True, (2600, 0, 1, 2599)), dict(segs=21), dict(waves=4, segs=21, seg_chunks=1)),
    ((1, 8, 2100, 8, 2, F32, True, None), dict(segs=17), dict(waves=4, segs=17, seg_chunks=1)),
    # 16 steps a lane, whole sequences of several passes
    ((66, 64, 2300, 3, 1, BF, True, None), dict(rows=4, steps=16, segs=1, chunks=18), dict(waves=8, segs=1, chunks=18)),
]

# N, D, L, type, residual's type, residual, scale, gate; the route; whether channels
# are left over that do not stay in registers (forward, backward)
NORM = [
    ((257, 1100, 20, BF, BF, True, True, True), dict(nt=1024, cl=4, tiles=257, parts=0), (False, True)),
    ((129, 1030, 64, BF, BF, False, True, True), dict(nt=1024, cl=4, tiles=258, parts=0), (False, True)),
    ((129, 1000, 72, BF, BF, True, False, True), dict(nt=1024, cl=8, tiles=258, parts=0), (False, True)),
    ((129, 600, 100, BF, F32, True, True, True), dict(nt=1024, cl=8, tiles=258, parts=0), (True, True)),
    ((129, 600, 100, F32, F32, True, True, False), dict(nt=1024, cl=8, tiles=258, parts=0), (True, True)),
    ((257, 2100, 16, F32, F32, True, True, True), dict(nt=1024, cl=2, tiles=257, parts=0), (True, True)),
    ((257, 2060, 16, BF, BF, True, True, True), dict(nt=1024, cl=2, tiles=257, parts=0), (False, True)),
    ((2, 200, 100, BF, BF, True, True, True), dict(nt=1024, cl=2, tiles=14, parts=0), (False, False)),
]


def name(case):
    return "-".join(map(str, case[0])).replace("torch.", "").replace(" ", "")


def has(shape, route):
    assert {k: getattr(shape, k) for k in route} == route, vars(shape)


@pytest.mark.parametrize("case", SCAN, ids=name)
def test_scan_routes(case):
    (N, D, L, S, G, *_), fwd, bwd = case
    has(seq_shapes.scan(N, D, L, S, G), fwd)
    has(seq_shapes.scan(N, D, L, S, G, bwd=True), bwd)


@pytest.mark.parametrize("case", NORM, ids=name)
def test_norm_routes(case):
    (N, D, L, _, rt, *_), route, left = case
    s = seq_shapes.norm(N, D, L, rt == BF)
    has(s, route)
    rows = s.nt // s.cl  # (channels at once; the forward pass holds twice the backward's)
    assert (D > 2 * s.held * rows, D > s.held * rows) == left


@pytest.mark.gpu
@pytest.mark.parametrize("case", SCAN, ids=name)
def test_scan_instances(case):
    N, D, L, S, Gr, t, gate, lens = case[0]
    say("[gpu] scan instance", case[0])
    G = Gen(51)
    v = scan_inputs(G, N, D, L, S, Gr, t, gate, True, True, True)
    lengths = None
    if lens is not None:
        lengths = torch.tensor([lens[n % len(lens)] for n in range(N)], dtype=torch.int32, device=DEV)
    do, df = spoil(G.n(N, D, L, dtype=t), lengths), G.n(N, D, S)
    for k in ("u", "delta", "B", "C", "z"):
        if v[k] is not None:
            v[k] = spoil(v[k], lengths)
    pos = [v[k] for k in ("u", "delta", "A", "B", "C")]
    kw = dict(D=v["D"], z=v["z"], delta_bias=v["delta_bias"], delta_softplus=True, lengths=lengths)
    args = (*pos, v["D"], v["z"], v["delta_bias"], True, v["initial_state"], lengths)
    out, fin, chk = seq.selective_scan_fwd(*pos, initial_state=v["initial_state"], return_final_state=True,
                                           return_checkpoints=True, **kw)
    ref, rfin, _, _, bound, fbound = O.selective_scan(*args)
    check("out", out, ref, 1.0, bound)
    check("final_state", fin, rfin, 1.0, fbound)
    g = seq.selective_scan_bwd(do, *pos, chk, dfinal_state=df, **kw)
    s = seq_shapes.scan(N, D, L, S, Gr, bwd=True)
    grads, bounds = O.selective_scan_grad_bounds(do, *args, df, cut=(s.segs, s.seg_chunks))
    for nm, got, r, b in zip(NAMES, g, grads, bounds):
        assert (got is None) == (nm == "dz" and not gate)
        if got is not None:
            check(nm, got, r, 1.0, b)


@pytest.mark.gpu
@pytest.mark.parametrize("case", NORM, ids=name)
def test_norm_instances(case):
    N, D, L, t, rt, has_r, has_s, has_g = case[0]
    say("[gpu] norm instance", case[0])
    G = Gen(52)
    x, w = G.n(N, D, L, dtype=t), 1 + 0.1 * G.n(D)
    res = G.n(N, D, L, dtype=rt) if has_r else None
    sc = G.n(D) if has_s else None
    gate = G.n(N, D, L, dtype=t) if has_g else None
    # Sums of squares are of one sign, the rest is a dozen steps; a parameter's
    # gradient is added over eight columns, up to eight lanes, the workgroup's tiles,
    # a sixteenth of the workgroups and the sixteen waves that take them.
    s = seq_shapes.norm(N, D, L, rt == BF)
    c = 40 + D / 64
    p = c + 12 * -(-s.tiles // s.wgs) + s.wgs / 16 + 20
    y, r = seq.norm_pre_fwd(x, w, residual=res, scale=sc)
    ry, rr = O.norm_pre(x, w, res, sc)
    mag = O.norm_pre(x.abs(), w, None if res is None else res.abs(), None if sc is None else sc.abs())[1]
    check("sum", r, rr, 4, mag)
    check("out", y, ry, c, mag / (rr.square().mean(1, keepdim=True) + 1e-6).sqrt() * O.d(w)[:, None].abs() + ry.abs())
    do, ds = G.n(N, D, L, dtype=t), G.n(N, D, L, dtype=r.dtype)
    args = (do, r, w, ds, x if has_s else None, sc)
    g = seq.norm_pre_bwd(do, r, w, dsum=ds, x=args[4], scale=sc)
    rg, mg = O.norm_pre_grads(*args), O.norm_pre_grads(*args, absolute=True)
    for nm, got, ref, m, k in zip(g._fields, g, rg, mg, (c, c, p, p)):
        if got is not None:
            check(nm, got, ref, k, m)
    o = seq.norm_post_fwd(x, w, gate=gate, residual=res, scale=sc)
    check("post", o, O.norm_post(x, w, gate, res, sc), c,
          O.norm_post(x, w, gate, None, sc).abs() + (O.d(res).abs() if has_r else 0))
    do = G.n(N, D, L, dtype=o.dtype)
    g = seq.norm_post_bwd(do, x, w, gate=gate, scale=sc)
    args = (do, x, w, gate, sc)
    rg, mg = O.norm_post_grads(*args), O.norm_post_grads(*args, absolute=True)
    for nm, got, ref, m, k in zip(g._fields, g, rg, mg, (c, c, p, p)):
        if got is not None:
            check(nm, got, ref, k, m)
