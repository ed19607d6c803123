"""The sequence operators in 64 bits, from their definitions -- TEST
INFRASTRUCTURE ONLY.

Torch on the CPU in float64, one step at a time.  Each ``*_grads`` writes the
gradients' formulas out.  With ``absolute=True`` every product and sum is taken
of absolute values, which gives the magnitude that a result was summed from:
what its rounding errors are relative to.
"""
import torch

F64 = torch.float64


def d(x):
    return None if x is None else x.detach().cpu().to(F64)


def _lens(lengths, N, L):
    return [L] * N if lengths is None else [max(0, min(L, int(v))) for v in lengths.tolist()]


def _mask(lens, L):
    return (torch.arange(L)[None, None] < torch.tensor(lens)[:, None, None]).to(F64)


def _clean(x, mask):
    return None if x is None else torch.where(mask > 0, x, torch.zeros((), dtype=F64))


def silu(z):
    return z * torch.sigmoid(z)


def dsilu(z):
    s = torch.sigmoid(z)
    return s * (1 + z * (1 - s))


def softplus(x):
    return x.clamp(min=0) + torch.log1p(torch.exp(-x.abs()))


# --------------------------------------------------------- causal convolution

def _entries(x, initial_state, lens, R):
    N, D, L = x.shape
    init = torch.zeros((N, D, R - 1), dtype=F64) if initial_state is None else d(initial_state)
    return torch.cat((init, _clean(d(x), _mask(lens, L))), -1)


def causal_conv(x, weight, bias=None, activation=None, initial_state=None, lengths=None):
    """out, final_state, and the magnitude of the sum before the activation."""
    N, D, L = x.shape
    w, R = d(weight), weight.shape[1]
    lens = _lens(lengths, N, L)
    e = _entries(x, initial_state, lens, R)
    b = torch.zeros(D, dtype=F64) if bias is None else d(bias)
    p = b[:, None] + sum(w[:, r, None] * e[..., r:r + L] for r in range(R))
    m = b.abs()[:, None] + sum(w[:, r, None].abs() * e[..., r:r + L].abs() for r in range(R))
    out = _clean(silu(p) if activation == "silu" else p, _mask(lens, L).expand_as(p))
    final = torch.stack([e[n, :, k:k + R - 1] for n, k in enumerate(lens)])
    return out, final, m


def causal_conv_grads(dout, x, weight, bias=None, activation=None, initial_state=None, lengths=None,
                      dfinal_state=None, absolute=False):
    """dx, dweight, dbias, dinitial_state."""
    N, D, L = x.shape
    w, R = d(weight), weight.shape[1]
    lens = _lens(lengths, N, L)
    mask = _mask(lens, L)
    e = _entries(x, initial_state, lens, R)
    b = torch.zeros(D, dtype=F64) if bias is None else d(bias)
    p = b[:, None] + sum(w[:, r, None] * e[..., r:r + L] for r in range(R))
    m = b.abs()[:, None] + sum(w[:, r, None].abs() * e[..., r:r + L].abs() for r in range(R))
    q = _clean(d(dout), mask.expand_as(p))
    dfin = None if dfinal_state is None else d(dfinal_state)
    if absolute:
        q, w, e = q.abs() * (1.1 + m if activation == "silu" else 1), w.abs(), e.abs()
        dfin = None if dfin is None else dfin.abs()
    elif activation == "silu":
        q = q * dsilu(p)
    q = _clean(q, mask.expand_as(q))
    de = torch.zeros_like(e)
    dw = torch.empty_like(w)
    for r in range(R):
        de[..., r:r + L] += w[:, r, None] * q
        dw[:, r] = (q * e[..., r:r + L]).sum((0, 2))
    if dfin is not None:
        for n, k in enumerate(lens):
            de[n, :, k:k + R - 1] += dfin[n]
    dx = _clean(de[..., R - 1:], mask.expand_as(p))
    return dx, dw, q.sum((0, 2)), de[..., :R - 1]


# -------------------------------------------------------------- selective scan

def _scan_inputs(u, delta, A, B, C, z, delta_bias, delta_softplus, lengths):
    N, D, L = u.shape
    G = B.shape[1]
    mask = _mask(_lens(lengths, N, L), L)
    raw = _clean(d(delta), mask.expand(N, D, L))
    if delta_bias is not None:
        raw = raw + d(delta_bias)[:, None]
    dt = (softplus(raw) if delta_softplus else raw) * mask
    u = _clean(d(u), mask.expand(N, D, L))
    z = None if z is None else _clean(d(z), mask.expand(N, D, L))
    B, C = (_clean(d(v), mask[:, None].expand(v.shape)) for v in (B, C))
    Be, Ce = (v.repeat_interleave(D // G, 1) for v in (B, C))  # [N, D, S, L]
    return u, raw, dt, d(A), Be, Ce, z, mask


def selective_scan(u, delta, A, B, C, D=None, z=None, delta_bias=None, delta_softplus=False, initial_state=None,
                   lengths=None):
    """out, final state, states before each step [L][N, D, S], y, and bounds
    (in units of 2^-24) of what fp32 arithmetic may be off by in out and the
    final state."""
    u, raw, dt, A, B, C, z, mask = _scan_inputs(u, delta, A, B, C, z, delta_bias, delta_softplus, lengths)
    N, Dn, L = u.shape
    h = torch.zeros((N, Dn, A.shape[1]), dtype=F64) if initial_state is None else d(initial_state)
    m, err = h.abs(), torch.zeros_like(h)
    before, ys, ms, es = [], [], [], []
    for t in range(L):
        before.append(h)
        a = torch.exp(dt[..., t, None] * A)
        x = (dt[..., t] * u[..., t])[..., None] * B[..., t]
        h = a * h + x
        m = a * m + x.abs()
        # In steps of 2^-24.  dt: without softplus one rounding; through it, for
        # v = raw far below zero, dt is about e = exp(v), whose relative error is
        # |v| for v's own rounding, 1.3 |v| for its product with log2(e) and that
        # constant, and 10 for exp2, the reciprocal, three products, the
        # polynomial and the last sum; for v above zero e's part of dt shrinks.
        # a: the exponent's relative error (dt's, A's product with the constant,
        # the product, a sum over dt) times the exponent, 2 for exp2.  x: dt's
        # and three products.  The state: products and sums of the composition.
        edt = 2.5 * raw[..., t].abs() + 10 if delta_softplus else torch.ones_like(dt[..., t])
        err = a * err + m * (8 + (8 + edt[..., None]) * (A * dt[..., t, None]).abs()) + x.abs() * edt[..., None]
        ys.append((h * C[..., t]).sum(-1))
        ms.append((m * C[..., t].abs()).sum(-1))
        es.append((err * C[..., t].abs()).sum(-1))
    y, ym, ye = (torch.stack(v, -1) for v in (ys, ms, es))
    if D is not None:
        y, ym = y + d(D)[:, None] * u, ym + (d(D)[:, None] * u).abs()
    bound = ye + (A.shape[1] + 8) * ym  # the sum over the states, the skip, the gate
    out = y
    if z is not None:
        out, bound = y * silu(z), bound * silu(z).abs() + 16 * y.abs() * silu(z).abs()
    return out * mask, h, before, y, bound, err


def selective_scan_grads(dout, u, delta, A, B, C, D=None, z=None, delta_bias=None, delta_softplus=False,
                         initial_state=None, lengths=None, dfinal_state=None, absolute=False):
    """du, ddelta, dA, dB, dC, dD, ddelta_bias, dz, dinitial_state."""
    G = B.shape[1]
    if absolute:
        u0, B0, C0 = u.abs(), B.abs(), C.abs()
        i0 = None if initial_state is None else initial_state.abs()
        D0 = None if D is None else D.abs()
    else:
        u0, B0, C0, i0, D0 = u, B, C, initial_state, D
    _, _, before, y, _, _ = selective_scan(u0, delta, A, B0, C0, D0, None, delta_bias, delta_softplus, i0, lengths)
    u, raw, dt, A, Be, Ce, z, mask = _scan_inputs(u0, delta, A, B0, C0, z, delta_bias, delta_softplus, lengths)
    N, Dn, L = u.shape
    g = _clean(d(dout), mask.expand(N, Dn, L))
    gate = torch.ones_like(u) if z is None else silu(z)
    dgate = torch.zeros_like(u) if z is None else dsilu(z)
    if absolute:
        g, gate, dgate = g.abs(), gate.abs(), dgate.abs() + 0.1 * (z is not None)
    dy = g * gate
    As = A.abs() if absolute else A
    r = torch.zeros((N, Dn, A.shape[1]), dtype=F64) if dfinal_state is None else d(dfinal_state)
    r = r.abs() if absolute else r
    dA = torch.zeros_like(A)
    ddt, dx = torch.zeros_like(u), torch.zeros_like(u)
    dB, dC = torch.zeros_like(Be), torch.zeros_like(Ce)
    for t in reversed(range(L)):
        a = torch.exp(dt[..., t, None] * A)
        x = dt[..., t] * u[..., t]
        h = a * before[t] + (x.abs() if absolute else x)[..., None] * Be[..., t]
        e = r + dy[..., t, None] * Ce[..., t]
        dC[..., t] = dy[..., t, None] * h
        dB[..., t] = e * (x.abs() if absolute else x)[..., None]
        dx[..., t] = (e * Be[..., t]).sum(-1)
        r = a * e
        k = r * before[t]
        ddt[..., t] = (k * As).sum(-1)
        dA += (k * (dt[..., t, None].abs() if absolute else dt[..., t, None])).sum(0)
    skip = torch.zeros(Dn, dtype=F64) if D0 is None else d(D0)
    ddelta = ddt + dx * u
    if delta_softplus:
        ddelta = ddelta * torch.sigmoid(raw)
    ddelta = ddelta * mask
    du = dx * (dt.abs() if absolute else dt) + skip[:, None] * dy
    dB, dC = (v.view(N, G, Dn // G, A.shape[1], L).sum(2) * mask[:, None] for v in (dB, dC))
    return du * mask, ddelta, dA, dB, dC, (dy * u).sum((0, 2)), ddelta.sum((0, 2)), g * y * dgate, r


def selective_scan_grad_bounds(dout, u, delta, A, B, C, D=None, z=None, delta_bias=None, delta_softplus=False,
                               initial_state=None, lengths=None, dfinal_state=None, cut=None):
    """The gradients again, and bounds (in units of 2^-24) of what fp32 arithmetic
    may be off by in each, carried along both recurrences: (grads, bounds), in the
    order of :func:`selective_scan_grads`.

    What is counted: a gradient of a state is off by what reaches it of the next
    step's, decayed, and its own roundings, as a state is in
    :func:`selective_scan`; a product by each factor's error times the other one's
    magnitude, and its rounding; a sum by its terms' errors and one rounding of the
    whole (in absolute values) for each level of the tree it is formed by.  `cut`:
    the segments of a sequence and their chunks of 128 steps (else one).
    """
    G = B.shape[1]
    _, _, before, y, ybound, _ = selective_scan(u, delta, A, B, C, D, None, delta_bias, delta_softplus, initial_state,
                                                lengths)
    u, raw, dt, A, Be, Ce, z, mask = _scan_inputs(u, delta, A, B, C, z, delta_bias, delta_softplus, lengths)
    N, Dn, L = u.shape
    S = A.shape[1]
    g = _clean(d(dout), mask.expand(N, Dn, L))
    zero = torch.zeros_like(u)
    gate, dgate, mdgate, az = torch.ones_like(u), zero, zero, zero
    if z is not None:
        s = torch.sigmoid(z)
        gate, dgate, mdgate, az = silu(z), dsilu(z), s * (1 + z.abs() * (1 - s)), z.abs()
    dy = g * gate
    # relative, in 2^-24: dt and dy (a sigmoid: its rounded exponent and four more,
    # two products), the slope of softplus
    edt = (2.5 * raw.abs() + 10 if delta_softplus else torch.ones_like(raw)) * mask
    edy = (2 * az + 8 if z is not None else zero)
    eslope = 3 * raw.abs() + 6
    x = dt * u
    # the states' errors
    h = torch.zeros((N, Dn, S), dtype=F64) if initial_state is None else d(initial_state)
    m, herr = h.abs(), [torch.zeros_like(h)]
    for t in range(L):
        a, xb = torch.exp(dt[..., t, None] * A), x[..., t, None].abs() * Be[..., t].abs()
        decay = 8 + (8 + edt[..., t, None]) * (A * dt[..., t, None]).abs()
        m = a * m + xb
        herr.append(a * herr[-1] + m * decay + xb * edt[..., t, None])
    # levels of sums: a wave's four channels, a workgroup's waves, the workgroups; 8
    # steps of a lane, 4 levels over lanes, the chunks of a segment (dD and
    # ddelta_bias: all steps of a lane before the lanes) and then the segments and
    # sequences one by one
    per, (segs, chunks) = Dn // G, cut or (1, -(-L // 128))
    over_channels, over_steps = 2 + 8 + -(-per // 16), 12 + chunks + N * segs
    over_elements = 8 * chunks + 4 + N * segs
    r = torch.zeros((N, Dn, S), dtype=F64) if dfinal_state is None else d(dfinal_state)
    mr, er = r.abs(), torch.zeros_like(r)
    dA, edA = torch.zeros_like(A), torch.zeros_like(A)
    ddt, eddt, dx, edx = (torch.zeros_like(u) for _ in range(4))
    dB, dC = torch.zeros_like(Be), torch.zeros_like(Ce)
    edB, edC = torch.zeros_like(Be), torch.zeros_like(Ce)
    for t in reversed(range(L)):
        p, hp, ehp = dt[..., t, None], before[t], herr[t]
        a, decay = torch.exp(p * A), 8 + (8 + edt[..., t, None]) * (A * p).abs()
        c, b, q, xt = Ce[..., t], Be[..., t], dy[..., t, None], x[..., t, None]
        ht, eht = a * hp + xt * b, herr[t + 1]
        e, me = r + q * c, mr + (q * c).abs()
        ee = er + (q * c).abs() * (edy[..., t, None] + 1) + me
        dC[..., t], edC[..., t] = q * ht, q.abs() * eht + (q * ht).abs() * (edy[..., t, None] + 2 + over_channels)
        dB[..., t] = e * xt
        edB[..., t] = ee * xt.abs() + (e * xt).abs() * (edt[..., t, None] + 3 + over_channels)
        dx[..., t], edx[..., t] = (e * b).sum(-1), ((ee + e.abs() * (S + 1)) * b.abs()).sum(-1)
        r, mr, er = a * e, a * me, a * ee + a * me * decay
        k = r * hp
        ek = 1.01 * (er * hp.abs() + r.abs() * ehp) + k.abs()
        ddt[..., t], eddt[..., t] = (k * A).sum(-1), ((ek + k.abs() * (S + 4)) * A.abs()).sum(-1)
        dA += (k * p).sum(0)
        edA += ((ek + k.abs() * (edt[..., t, None] + 2 + over_steps)) * p.abs()).sum(0)
    skip = torch.zeros(Dn, dtype=F64) if D is None else d(D)
    slope = torch.sigmoid(raw) if delta_softplus else torch.ones_like(raw)
    ddelta = (ddt + dx * u) * slope * mask
    eddelta = (edx * u.abs() + eddt + 3 * ((dx * u).abs() + ddt.abs())) * slope * mask
    if delta_softplus:
        eddelta = eddelta + ddelta.abs() * (eslope + 1)
    sk = (skip[:, None] * dy).abs()
    du, edu = dx * dt + skip[:, None] * dy, edx * dt.abs() + (dx * dt).abs() * (edt + 2) + sk * (edy + 2)
    fold = lambda v: v.view(N, G, per, S, L).sum(2) * mask[:, None]  # noqa: E731
    # (ybound is the ungated y's)
    edz = (g * dgate).abs() * ybound + (g * y).abs() * mdgate * (4 * az + 16)
    grads = (du * mask, ddelta, dA, fold(dB), fold(dC), (dy * u).sum((0, 2)), ddelta.sum((0, 2)), g * y * dgate, r)
    bounds = (edu * mask, eddelta, edA, fold(edB), fold(edC), ((dy * u).abs() * (edy + 2 + over_elements)).sum((0, 2)),
              (eddelta + ddelta.abs() * over_elements).sum((0, 2)), edz, er)
    return grads, bounds


# ------------------------------------------------------------------------ norms

def norm_pre(x, weight, residual=None, scale=None, eps=1e-6):
    """out, sum."""
    r = d(x) * (1 if scale is None else d(scale)[:, None])
    if residual is not None:
        r = r + d(residual)
    return d(weight)[:, None] * r / (r.square().mean(1, keepdim=True) + eps).sqrt(), r


def _dnorm(n, h, rstd, absolute):
    if absolute:
        return rstd * (h.abs() + n.abs() * (h * n).abs().mean(1, keepdim=True))
    return rstd * (h - n * (h * n).mean(1, keepdim=True))


def norm_pre_grads(dout, sum, weight, dsum=None, x=None, scale=None, eps=1e-6, absolute=False):
    """dx, dresidual, dweight, dscale."""
    r, g, w = d(sum), d(dout), d(weight)[:, None]
    rstd = 1 / (r.square().mean(1, keepdim=True) + eps).sqrt()
    n, mag = r * rstd, torch.abs if absolute else (lambda v: v)
    dr = _dnorm(n, w * g, rstd, absolute)
    if dsum is not None:
        dr = dr + mag(d(dsum))
    sc = 1 if scale is None else mag(d(scale)[:, None])
    return sc * dr, dr, mag(g * n).sum((0, 2)), None if scale is None else (dr * mag(d(x))).sum((0, 2))


def norm_post(x, weight, gate=None, residual=None, scale=None, eps=1e-6):
    v = d(x) * (1 if gate is None else silu(d(gate)))
    n = v / (v.square().mean(1, keepdim=True) + eps).sqrt()
    out = n * d(weight)[:, None] * (1 if scale is None else d(scale)[:, None])
    return out if residual is None else out + d(residual)


def norm_post_grads(dout, x, weight, gate=None, scale=None, eps=1e-6, absolute=False):
    """dx, dgate, dweight, dscale."""
    x, g, w = d(x), d(dout), d(weight)[:, None]
    sc = torch.ones_like(w) if scale is None else d(scale)[:, None]
    z = None if gate is None else d(gate)
    v = x if z is None else x * silu(z)
    rstd = 1 / (v.square().mean(1, keepdim=True) + eps).sqrt()
    n, mag = v * rstd, torch.abs if absolute else (lambda v: v)
    dv = _dnorm(n, sc * w * g, rstd, absolute)
    dx = dv if z is None else dv * mag(silu(z))
    dz = None if z is None else dv * mag(x) * (mag(dsilu(z)) + (0.1 if absolute else 0))
    gn = mag(g * n)
    return dx, dz, (mag(sc) * gn).sum((0, 2)), (mag(w) * gn).sum((0, 2))
