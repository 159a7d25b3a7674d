"""The encoder's layers in float64, from their definitions, each output with a
bound on what a float32 evaluation with one final rounding may be off by.

Bounds.  u is the unit roundoff of the array's type (2^-24, 2^-11, 2^-8) and
U = 2^-24.  A float32 sum of products with n roundings on its way is off by at
most n U (1 + tiny) times the sum of the products' magnitudes, and the final
rounding adds u |value| (plus the type's smallest subnormal).  ``fast`` covers
the exponential, error function, division and reciprocal square root: 2^-20 of
the value.
"""
import math

import torch

U = 2.0 ** -24
FAST = 2.0 ** -20
ROUND = {torch.float32: U, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
LEAST = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -24, torch.bfloat16: 2.0 ** -133}


def rounded(value, bound, dtype):
    """The bound after the final rounding."""
    return bound * (1 + ROUND[dtype]) + ROUND[dtype] * value.abs() + LEAST[dtype]


def within(got, value, bound):
    off = (got.double() - value).abs()
    ok = off <= bound
    assert bool(ok.all()), "off by %g where %g is allowed (%d of %d)" % (
        float(off[~ok].max()), float(bound.expand_as(off)[~ok][off[~ok].argmax()]), int((~ok).sum()), ok.numel())


def embed(table, ids, scale):
    ids = ids.long()
    out = table.double()[ids.clamp(min=0)] * scale
    out[ids < 0] = 0
    return out, rounded(out, 2 * U * out.abs(), table.dtype)


def embed_grad(d_out, ids, scale, V):
    ids = ids.long()
    keep = ids >= 0
    rows = d_out.double()[keep]
    total = torch.zeros(V, d_out.shape[1], dtype=torch.float64, device=d_out.device).index_add_(0, ids[keep], rows)
    size = torch.zeros_like(total).index_add_(0, ids[keep], rows.abs())
    n = torch.zeros(V, 1, dtype=torch.float64, device=d_out.device).index_add_(
        0, ids[keep], torch.ones(rows.shape[0], 1, dtype=torch.float64, device=d_out.device))
    return scale * total, rounded(scale * total, (n + 3) * U * abs(scale) * size, d_out.dtype)


def sequences(offsets, T, device):
    if offsets is None:
        return torch.zeros(T, dtype=torch.long, device=device)
    lengths = offsets[1:] - offsets[:-1]
    return torch.repeat_interleave(torch.arange(len(lengths), device=device), lengths)


def _inverse_rms(v, eps):
    return 1 / torch.sqrt((v * v).mean(1, keepdim=True) + eps)


def norm_join(x, y, gate, w_post, w_pre, offsets, rho, eps):
    """[(value, bound)] of x_out and n_out (None where absent)."""
    dt, (T, D) = x.dtype, x.shape
    c = (D + 16) * U + FAST
    xd = x.double()
    if y is None:
        xo, mag, bound = xd, xd.abs(), torch.zeros_like(xd)
    else:
        yd = y.double()
        post = w_post.double() * yd * _inverse_rms(yd, eps)
        if gate is not None:
            post = post * gate.double()[sequences(offsets, T, x.device)]
        xo = rho * xd + post
        mag = abs(rho) * xd.abs() + post.abs()
        bound = c * mag
    first = None if y is None else (xo, rounded(xo, bound, dt))
    if w_pre is None:
        return first, None
    ix = _inverse_rms(xo, eps)
    n = w_pre.double() * xo * ix
    # the mean square's relative error: the terms' own and the sum's
    rel = bound.norm(dim=1, keepdim=True) / (xo.norm(dim=1, keepdim=True) + 1e-300) + c
    return first, (n, rounded(n, w_pre.double().abs() * ix * bound + n.abs() * (rel + c), dt))


def norm_join_grad(xo, y, gate, w_post, w_pre, dxo, dn, offsets, rho, eps):
    """[(value, bound)] of dx, dy, d_gate, d_w_post, d_w_pre (None where absent)."""
    dt, (T, D) = xo.dtype, xo.shape
    dev = xo.device
    c = 4 * (D + 32) * U + 4 * FAST
    x = xo.double()
    zero = torch.zeros_like(x)
    g = zero if dxo is None else dxo.double()
    size = g.abs()
    d_pre = None
    if dn is not None:
        ix = _inverse_rms(x, eps)
        z = dn.double() * w_pre.double()
        g = g + ix * (z - x * ix ** 2 * (z * x).mean(1, keepdim=True))
        size = size + ix * (z.abs() + x.abs() * ix ** 2 * (z * x).abs().mean(1, keepdim=True))
        t = dn.double() * x * ix
        d_pre = (t.sum(0), rounded(t.sum(0), (c + T * U) * t.abs().sum(0), dt))
    if y is None:
        return [(g, rounded(g, c * size, dt)), None, None, None, d_pre]
    dx = (rho * g, rounded(rho * g, abs(rho) * c * size, dt))
    yd = y.double()
    iy = _inverse_rms(yd, eps)
    u = yd * iy
    B = 1 if offsets is None else len(offsets) - 1
    seq = sequences(offsets, T, dev)
    gates = torch.ones(B, D, dtype=torch.float64, device=dev) if gate is None else gate.double()
    w = w_post.double()
    du, du_size = gates[seq] * w * g, (gates[seq] * w).abs() * size
    dy = iy * (du - u * (du * u).mean(1, keepdim=True))
    dy_size = iy * (du_size + u.abs() * (du_size * u.abs()).mean(1, keepdim=True))
    empty = torch.zeros(B, D, dtype=torch.float64, device=dev)
    S, S_size = empty.index_add(0, seq, g * u), empty.index_add(0, seq, size * u.abs())
    n = torch.bincount(seq, minlength=B).double()[:, None]
    d_gate = None if gate is None else (w * S, rounded(w * S, w.abs() * (c + n * U) * S_size, dt))
    post = (gates * S).sum(0)
    d_post = (post, rounded(post, (c + (T + B) * U) * (gates.abs() * S_size).sum(0), dt))
    return [dx, (dy, rounded(dy, c * dy_size, dt)), d_gate, d_post, d_pre]


def _phi(x):
    return torch.erfc(-x / math.sqrt(2)) / 2


def activation(name, g):
    """act(g), its slope and a bound on the slope's change per unit of g."""
    if name == "relu":
        return g.clamp(min=0), (g > 0).double(), 0.0
    if name == "silu":
        p = torch.sigmoid(g)
        return g * p, p * (1 + g * (1 - p)), 0.5
    d = torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    return g * _phi(g), _phi(g) + g * d, 0.8


def _hidden(x, w_in, act, F):
    D = x.shape[1]
    gu, size = x @ w_in.t(), x.abs() @ w_in.abs().t()
    e = (D + 4) * U * size
    a, slope, bend = activation(act, gu[:, :F])
    return gu[:, :F], gu[:, F:], a, slope, bend, e[:, :F], e[:, F:]


def ffn(x, w_in, w_out, act):
    dt, F = x.dtype, w_out.shape[1]
    x, w_in, w_out = x.double(), w_in.double(), w_out.double()
    g, u, a, _, _, eg, eu = _hidden(x, w_in, act, F)
    h = a * u
    # |act'| <= 1.13 for all three
    eh = rounded(h, 1.13 * eg * (u.abs() + eu) + a.abs() * eu + FAST * (h.abs() + g.abs() * u.abs() * 2 ** -3), dt)
    y = h @ w_out.t()
    return y, rounded(y, eh @ w_out.abs().t() + (F + 4) * U * ((h.abs() + eh) @ w_out.abs().t()), dt)


def ffn_grad(x, w_in, w_out, dy, act):
    """[(value, bound)] of dx, d_w_in, d_w_out."""
    dt, F = x.dtype, w_out.shape[1]
    (T, D) = x.shape
    x, w_in, w_out, dy = x.double(), w_in.double(), w_out.double(), dy.double()
    g, u, a, slope, bend, eg, eu = _hidden(x, w_in, act, F)
    dh = dy @ w_out
    ed = (D + 4) * U * (dy.abs() @ w_out.abs())
    h, dg, du = a * u, dh * u * slope, dh * a
    ea = 1.13 * eg + FAST * (a.abs() + g.abs() * 2 ** -3)
    es = bend * eg + 4 * FAST * (1 + g.abs())
    if act == "relu":       # the slope of a value that rounding may carry across 0
        es = es + (g.abs() <= eg).double()
    eh = rounded(h, ea * (u.abs() + eu) + a.abs() * eu, dt)
    edg = rounded(dg, ed * ((u.abs() + eu) * (slope.abs() + es)) + dh.abs() * (eu * (slope.abs() + es) + u.abs() * es), dt)
    edu = rounded(du, ed * (a.abs() + ea) + dh.abs() * ea, dt)
    dgu, e = torch.cat([dg, du], 1), torch.cat([edg, edu], 1)

    def product(p, ep, q):
        v = p @ q
        n = p.shape[1] + 4
        return v, rounded(v, ep @ q.abs() + n * U * ((p.abs() + ep) @ q.abs()), dt)

    d_out, ed_out = dy.t() @ h, dy.abs().t() @ eh + (T + 4) * U * (dy.abs().t() @ (h.abs() + eh))
    return [product(dgu, e, w_in), product(dgu.t(), e.t(), x), (d_out, rounded(d_out, ed_out, dt))]
