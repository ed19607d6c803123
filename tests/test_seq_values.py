"""Values at the ends of fp32's range in the selective scan: what is finite in
the definition stays finite and right."""
import pytest
import torch

from oracle import seq as O
from paper_2101_09808_amd import seq
from tests.test_seq_ops import DEV, F32, Gen, check, say, scan_inputs, scan_tolerance

pytestmark = pytest.mark.gpu

NAMES = ("du", "ddelta", "dA", "dB", "dC", "dD", "ddelta_bias", "dz", "dinitial_state")


def check_finite(name, got, ref, count, mag):
    """`check` where the definition is finite; elsewhere neither is."""
    fin, zero = torch.isfinite(ref), torch.zeros((), dtype=ref.dtype)
    other = torch.isfinite(got.cpu()) != fin
    assert not other.any(), (name, other.nonzero()[:4].tolist())
    got = torch.where(fin.to(got.device), got, 0)
    check(name, got, torch.where(fin, ref, zero), count, torch.where(fin, mag, zero))


@pytest.mark.parametrize("N,D,L,S", [(2, 6, 140, 1), (2, 6, 300, 5), (2, 6, 300, 16), (1, 70, 290, 17), (1, 5, 200, 33),
                                     (1, 4, 2600, 3)])
def test_infinite_step(N, D, L, S):
    """A step of infinite length wipes its channel's states out: gradients of
    earlier steps, and of the step itself but for what multiplies it, are finite."""
    say("[gpu] infinite step", N, D, L, S)
    G = Gen(31)
    v = scan_inputs(G, N, D, L, S, 1, F32, True, True, True, True)
    t = L // 2 + 3
    v["delta"][0, 2, t] = float("inf")
    do, df = G.n(N, D, L), G.n(N, D, S)
    pos = [v[k] for k in ("u", "delta", "A", "B", "C")]
    kw = dict(D=v["D"], z=v["z"], delta_bias=v["delta_bias"], delta_softplus=True)
    out, fin, chk = seq.selective_scan_fwd(*pos, initial_state=v["initial_state"], return_final_state=True,
                                           return_checkpoints=True, **kw)
    args = (*pos, v["D"], v["z"], v["delta_bias"], True, v["initial_state"])
    ref, rfin, _, _, bound, fbound = O.selective_scan(*args)
    check_finite("out", out, ref, 1.0, bound)
    check_finite("final_state", fin, rfin, 1.0, fbound)
    g = seq.selective_scan_bwd(do, *pos, chk, dfinal_state=df, **kw)
    rg = O.selective_scan_grads(do, *args, None, df)
    mg = O.selective_scan_grads(do, *args, None, df, absolute=True)
    assert torch.isfinite(rg[0][0, 2, :t]).all() and torch.isfinite(rg[1][0, 2, :t + 1]).all()
    for name, got, r, m in zip(NAMES, g, rg, mg):
        many = D if name in ("dB", "dC") else N * L / 16 if name in ("dA", "dD", "ddelta_bias") else 0
        check_finite(name, got, r, scan_tolerance(L, S) + many, m)


GROWING = [(2, 2100, 300, 3), (1, 2100, 700, 3), (1, 6, 500, 4), (1, 6, 1500, 4), (1, 1024, 4096, 2),
           (1, 512, 2304, 33)]


def growing_inputs(G, N, D, L, S):
    """Channels of A = 1 and -1 in turn, steps of 0.5 to 0.55: e^70 over 128 steps,
    past fp32 over 256."""
    v = scan_inputs(G, N, D, L, S, 1, F32, False, False, False, False)
    v["A"] = torch.ones_like(v["A"])
    v["A"][::2] = -1
    v["delta"] = 0.5 + 0.05 * G.u(N, D, L)
    return v


@pytest.mark.parametrize("N,D,L,S", GROWING)
def test_zeros_under_growing_decays(N, D, L, S):
    """Where a state and its gradient are zero they stay so, however far apart the
    inputs are that decays are composed over: u begins 100 steps before the end,
    dout ends 100 steps after the beginning."""
    say("[gpu] zeros under growing decays", N, D, L, S)
    G = Gen(32)
    v = growing_inputs(G, N, D, L, S)
    v["u"][..., :L - 100] = 0
    do = G.n(N, D, L)
    do[..., 100:] = 0
    pos = [v[k] for k in ("u", "delta", "A", "B", "C")]
    out, fin, chk = seq.selective_scan_fwd(*pos, return_final_state=True, return_checkpoints=True)
    ref, rfin, _, _, bound, fbound = O.selective_scan(*pos)
    check("out", out, ref, 1.0, bound)
    check("final_state", fin, rfin, 1.0, fbound)
    g = seq.selective_scan_bwd(do, *pos, chk)
    rg, mg = O.selective_scan_grads(do, *pos), O.selective_scan_grads(do, *pos, absolute=True)
    for name, got, r, m in zip(NAMES, g, rg, mg):
        if got is not None:
            many = D if name in ("dB", "dC") else N * L / 16 if name == "dA" else 0
            check(name, got, r, scan_tolerance(L, S) + many, m)


@pytest.mark.parametrize("N,D,L,S", GROWING)
def test_small_values_grow(N, D, L, S):
    """A value of 2e-36 grows over 250 steps to 1e18 and more, by a factor that
    fp32 does not hold; the other steps have no length."""
    say("[gpu] small values grow", N, D, L, S)
    G = Gen(33)
    v = growing_inputs(G, N, D, L, S)
    first = L // 512 * 256
    v["delta"][..., :first] = 0
    v["delta"][..., first + 250:] = 0
    v["u"].zero_()
    v["u"][..., first] = 2e-36
    pos = [v[k] for k in ("u", "delta", "A", "B", "C")]
    out, fin = seq.selective_scan_fwd(*pos, return_final_state=True)
    ref, rfin, _, _, bound, fbound = O.selective_scan(*pos)
    assert (rfin.abs() > 1e18).any()
    check("out", out, ref, 1.0, bound)
    check("final_state", fin, rfin, 1.0, fbound)


@pytest.mark.parametrize("N,D,L,S", [(3, 9, 150, 4), (3, 9, 700, 3), (3, 5, 2600, 16)])
def test_states_without_memory(N, D, L, S):
    """A = -inf: nothing of a state outlives a step, and steps behind a sequence's
    end leave it alone.  The same bits as from a decay that underflows in each step."""
    say("[gpu] states without memory", N, D, L, S)
    G = Gen(34)
    v = scan_inputs(G, N, D, L, S, 1, F32, True, True, True, True)
    do, df = G.n(N, D, L), G.n(N, D, S)
    lengths = torch.tensor([L, L // 2, 0], dtype=torch.int32, device=DEV)
    kw = dict(D=v["D"], z=v["z"], delta_bias=v["delta_bias"], delta_softplus=True, lengths=lengths)

    def run(a):
        v["A"][::2, 0] = a
        pos = [v[k] for k in ("u", "delta", "A", "B", "C")]
        o, f, c = seq.selective_scan_fwd(*pos, initial_state=v["initial_state"], return_final_state=True,
                                         return_checkpoints=True, **kw)
        one = [t[..., 0] if t.dim() > 2 else t for t in pos]
        st = v["initial_state"].clone()
        step = seq.selective_scan_step(one[0], st, *one[1:], delta_softplus=True)
        return [o, f, *seq.selective_scan_bwd(do, *pos, c, dfinal_state=df, **kw), step, st]

    far, inf = run(-1e7), run(float("-inf"))
    assert torch.equal(far[1][2], v["initial_state"][2])
    for a, b in zip(far, inf):
        assert torch.isfinite(b).all() and torch.equal(a, b)
