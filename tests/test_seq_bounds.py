"""The error bounds of the scan's gradients (oracle/seq.py), on the CPU: the
formulas in 32 bits keep them, and a sum that lost a part does not."""
import pytest
import torch

from oracle import seq as O

NAMES = ("du", "ddelta", "dA", "dB", "dC", "dD", "ddelta_bias", "dz", "dinitial_state")


def inputs(N, D, L, S, G, gate, soft, extra, seed=7):
    g = torch.Generator().manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    v = dict(u=n(N, D, L), delta=n(N, D, L) * 0.5)
    if not soft:
        v["delta"] = v["delta"].abs() * 0.1
    v.update(A=-torch.arange(1, S + 1.) * (0.5 + torch.rand(D, 1, generator=g)),
             B=n(N, G, S, L), C=n(N, G, S, L), D=n(D) if extra else None, z=n(N, D, L) if gate else None,
             delta_bias=-4 * torch.rand(D, generator=g) - 1 if extra else None)
    return (n(N, D, L), *v.values(), soft, n(N, D, S))


SHAPES = [(1, 2, 5, 1, 1, False, False, False), (2, 6, 70, 4, 2, True, True, True), (1, 4, 500, 3, 1, False, True, True),
          (3, 4, 200, 16, 1, True, False, False)]


@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_gradients_in_32_bits_keep_the_bounds(shape, monkeypatch):
    do, *args = inputs(*shape)
    lengths = torch.tensor([args[0].shape[2] - 3 * n for n in range(args[0].shape[0])])
    df = torch.randn(args[-1].shape, generator=torch.Generator().manual_seed(8))
    grads, bounds = O.selective_scan_grad_bounds(do, *args, lengths, df)
    for a, b in zip(grads, O.selective_scan_grads(do, *args, lengths, df)):
        assert torch.allclose(a, b, rtol=1e-12, atol=1e-13)
    monkeypatch.setattr(O, "F64", torch.float32)
    for name, ref, bound, got in zip(NAMES, grads, bounds, O.selective_scan_grads(do, *args, lengths, df)):
        assert got.dtype == torch.float32
        over = (got.double() - ref).abs() - 2.0 ** -24 * bound - 2.0 ** -126
        assert (over <= 0).all(), (name, float(over.max()))


@pytest.mark.parametrize("N,D,L,S,cut", [(7, 4, 2600, 16, (21, 1)), (1, 8, 2100, 8, (17, 1)), (2, 8, 1030, 8, (5, 2)),
                                         (1, 8, 2100, 8, (1, 17))])
def test_a_lost_part_is_seen(N, D, L, S, cut):
    """Sums over 128 steps are what the backward pass adds up: one of them is far
    more than the bounds allow in nearly every entry."""
    do, *args = inputs(N, D, L, S, 1, True, True, True)
    grads, bounds = O.selective_scan_grad_bounds(do, *args, cut=cut)
    part = torch.zeros_like(do)
    part[0, :, L // 2:L // 2 + 128] = do[0, :, L // 2:L // 2 + 128]
    lost = O.selective_scan_grads(part, *args)
    for i in (2, 5, 6):  # dA, dD, ddelta_bias: sums over sequences and steps
        tol = 2.0 ** -24 * bounds[i]
        assert tol.square().mean().sqrt() < 0.04 * grads[i].square().mean().sqrt(), NAMES[i]
        assert (lost[i].abs() > tol).double().mean() > 0.9, NAMES[i]
