"""The 64-bit forms that the sequence operators are tested against: their
written-out gradients against torch's automatic ones and against differences
(CPU only)."""
import pytest
import torch

from oracle import seq as O

F64 = torch.float64


def rand(*shape, seed=0):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed + sum(shape)), dtype=F64)


def leaves(*ts):
    return [t.clone().requires_grad_() for t in ts]


def close(got, ref):
    for g, r in zip(got, ref):
        assert torch.allclose(g, r, rtol=1e-9, atol=1e-11)


# The forms detach what they are given; for automatic gradients they are
# evaluated without that.
@pytest.fixture()
def attached(monkeypatch):
    monkeypatch.setattr(O, "d", lambda v: None if v is None else v.to(F64))


def differences(f, ts, cots, grads):
    """<grads, direction> against a central difference along a random direction:
    step 1e-5, so its own error is about 1e-10 of third derivatives near one."""
    dirs = [rand(*t.shape, seed=50 + i) for i, t in enumerate(ts)]
    val = [sum((o * c).sum() for o, c in zip(f(*[t + s * 1e-5 * v for t, v in zip(ts, dirs)]), cots)) for s in (1, -1)]
    lhs = (val[0] - val[1]) / 2e-5
    rhs = sum((g * v).sum() for g, v in zip(grads, dirs))
    assert abs(lhs - rhs) <= 1e-6 * (1 + abs(rhs))


@pytest.mark.parametrize("act", [None, "silu"])
@pytest.mark.parametrize("R", [1, 4])
def test_conv_grads(act, R, attached):
    x, w, b, i = rand(2, 3, 7), rand(3, R), rand(3), rand(2, 3, R - 1)
    lens = torch.tensor([7, 2])
    f = lambda x, w, b, i: O.causal_conv(x, w, b, act, i, lens)[:2]  # noqa: E731
    do, df = rand(2, 3, 7, seed=1), rand(2, 3, R - 1, seed=2)
    ts = leaves(x, w, b, i)
    o, fin = f(*ts)
    auto = torch.autograd.grad((o * do).sum() + (fin * df).sum(), ts)
    got = O.causal_conv_grads(do, x, w, b, act, i, lens, df)
    close(got, auto)
    differences(f, (x, w, b, i), (do, df), got)


@pytest.mark.parametrize("gate", [False, True])
@pytest.mark.parametrize("soft", [False, True])
def test_scan_grads(gate, soft, attached):
    N, D, S, G, L = 2, 4, 3, 2, 9
    u, dl, A, B, C = rand(N, D, L), rand(N, D, L, seed=1), -rand(D, S).abs(), rand(N, G, S, L), rand(N, G, S, L, seed=3)
    Dk, db, h0, z = rand(D), rand(D, seed=4), rand(N, D, S), rand(N, D, L, seed=5)
    lens = torch.tensor([9, 4])

    def f(u, dl, A, B, C, Dk, db, h0, *z):
        return O.selective_scan(u, dl, A, B, C, Dk, z[0] if z else None, db, soft, h0, lens)[:2]

    do, df = rand(N, D, L, seed=6), rand(N, D, S, seed=7)
    args = (u, dl, A, B, C, Dk, db, h0) + ((z,) if gate else ())
    ts = leaves(*args)
    o, fin = f(*ts)
    auto = torch.autograd.grad((o * do).sum() + (fin * df).sum(), ts)
    g = O.selective_scan_grads(do, u, dl, A, B, C, Dk, z if gate else None, db, soft, h0, lens, df)
    got = [*g[:7], g[8]] + ([g[7]] if gate else [])
    close(got, auto)
    differences(f, args, (do, df), got)


@pytest.mark.parametrize("full", [False, True])
def test_norm_grads(full, attached):
    x, w, r, sc, z = rand(2, 5, 3), rand(5), rand(2, 5, 3, seed=1), rand(5, seed=2), rand(2, 5, 3, seed=3)
    do, ds = rand(2, 5, 3, seed=4), rand(2, 5, 3, seed=5)
    if full:
        f = lambda x, r, w, sc: O.norm_pre(x, w, r, sc)  # noqa: E731
        args = (x, r, w, sc)
    else:
        f = lambda x, w: O.norm_pre(x, w)  # noqa: E731
        args = (x, w)
    ts = leaves(*args)
    o, s = f(*ts)
    auto = torch.autograd.grad((o * do).sum() + (s * ds).sum(), ts)
    g = O.norm_pre_grads(do, s.detach(), w, ds, x, sc if full else None)
    got = g if full else (g[0], g[2])
    close(got, auto)
    differences(f, args, (do, ds), got)
    if full:
        f = lambda x, z, w, sc: (O.norm_post(x, w, z, r, sc),)  # noqa: E731
        args = (x, z, w, sc)
    else:
        f = lambda x, w: (O.norm_post(x, w),)  # noqa: E731
        args = (x, w)
    ts = leaves(*args)
    auto = torch.autograd.grad((f(*ts)[0] * do).sum(), ts)
    g = O.norm_post_grads(do, x, w, z if full else None, sc if full else None)
    got = g if full else (g[0], g[2])
    close(got, auto)
    differences(f, args, (do,), got)
