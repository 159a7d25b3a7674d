"""The linear layer, attention and dropout in float64, from their definitions, each
output with a bound on what a float32 evaluation with the operators' roundings may
be off by (layers_util.py states the model)."""
import math

import torch

from layers_util import FAST, U, activation, rounded


def _act(name, z):
    return (z, torch.ones_like(z), 0.0) if name == "none" else activation(name, z)


def _z(x, w, bias):
    b = 0 if bias is None else bias.double()
    z, size = x.double() @ w.double().t() + b, x.double().abs() @ w.double().abs().t() + abs(b)
    return z, (x.shape[1] + 4) * U * size


def linear(x, w, bias, act, residual):
    z, e = _z(x, w, bias)
    v, _, _ = _act(act, z)
    e = 1.13 * e + (0 if act == "none" else FAST * (v.abs() + z.abs() * 2 ** -3))
    r = 0 if residual is None else residual.double()
    return v + r, rounded(v + r, e + U * (v.abs() + e + abs(r)), x.dtype)


def linear_grad(x, w, dy, bias, act):
    """[(value, bound)] of dx, d_w and (with a bias) d_bias."""
    dt, (T, D_in), D_out = x.dtype, x.shape, w.shape[0]
    x, w, dy = x.double(), w.double(), dy.double()
    z, e = _z(x, w, bias)
    _, slope, bend = _act(act, z)
    dz, edz = dy * slope, torch.zeros_like(z)
    if act != "none":
        es = bend * e + 4 * FAST * (1 + z.abs())
        if act == "relu":       # the slope of a value that rounding may carry across 0
            es = es + (z.abs() <= e).double()
        edz = rounded(dz, dy.abs() * es + U * dz.abs(), dt)
    size = dz.abs() + edz

    def product(p, q, ep, mag, n):
        return p @ q, rounded(p @ q, ep @ q.abs() + (n + 4) * U * (mag @ q.abs()), dt)

    out = [product(dz, w, edz, size, D_out), product(dz.t(), x, edz.t(), size.t(), T)]
    if bias is not None:
        out.append((dz.sum(0), rounded(dz.sum(0), edz.sum(0) + (T + 4) * U * size.sum(0), dt)))
    return out


# ---- dropout: Philox4x32-10 in Python's whole numbers

def philox(block, step, seed):
    m = 0xFFFFFFFF
    c, k = [block & m, block >> 32 & m, step & m, step >> 32 & m], [seed & m, seed >> 32 & m]
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [b >> 32 ^ c[1] ^ k[0], b & m, a >> 32 ^ c[3] ^ k[1], a & m]
        k = [k[0] + 0x9E3779B9 & m, k[1] + 0xBB67AE85 & m]
    return c


def words(first, count, step, seed):
    """Words first .. first + count - 1, as an int64 tensor of the host."""
    out = []
    for block in range(first // 4, (first + count + 3) // 4):
        out += philox(block, step % 2**64, seed % 2**64)
    return torch.tensor(out[first % 4:first % 4 + count], dtype=torch.int64)


def dropout(x, p, seed, step, residual):
    """value, bound: the scale is rounded once, the value is one product and sum."""
    keep = (words(0, x.numel(), step, seed) >= min(round(p * 2**32), 2**32 - 1)).view(x.shape).to(x.device)
    kept = torch.where(keep, x.double() / (1 - p), torch.zeros((), dtype=torch.float64, device=x.device))
    r = 0 if residual is None else residual.double()
    return kept + r, rounded(kept + r, 3 * U * (kept.abs() + abs(r)), x.dtype)


# ---- attention over packed sequences

# The base-2 exponential (ex2.approx.ftz) flushes results below float32's normal range,
# 2^-126, to zero: a probability may be off by that much whatever its relative error.
FLUSH = 2.0 ** -126

def _sequences(Tq, Tk, q_offsets, kv_offsets, ids):
    """(queries' slice, keys' indices) of every sequence"""
    qo = [0, Tq] if q_offsets is None else q_offsets.tolist()
    ko = [0, Tk] if kv_offsets is None else kv_offsets.tolist()
    for a, b, c, d in zip(qo, qo[1:], ko, ko[1:]):
        keys = torch.arange(c, d)
        if ids is not None:
            keys = keys[(ids[c:d] >= 0).cpu()]
        yield slice(a, b), keys


def _probabilities(q, k, scale, dt):
    """softmax(scale q k^T) per head, log-sum-exp and the relative error of a
    probability: the scores' absolute errors, the exponential and the sum.  q
    [Tq][H][d], k [n][H][d] -> [H][Tq][n]."""
    d, n = q.shape[2], k.shape[0]
    s = torch.einsum("qhd,khd->hqk", q, k) * scale
    es = (d + 8) * U * torch.einsum("qhd,khd->hqk", q.abs(), k.abs()) * abs(scale)
    es = es + 4 * U * s.abs()                       # the change of base
    worst = es.amax(-1, keepdim=True)
    lse = torch.logsumexp(s, -1, keepdim=True)
    # the sum is rescaled at most once per tile of keys
    rel = 2 * worst + 4 * FAST + (n + 2 * (n // 16 + 2)) * U + 4 * U * lse.abs()
    return torch.exp(s - lse), lse, rel, worst + (n + 8) * U + 2 * FAST + 4 * U * (lse.abs() + s.abs().amax(-1, keepdim=True))


def attend(q, k, v, q_offsets=None, kv_offsets=None, ids=None, scale=None):
    """(value, bound) of the output and of the log-sum-exp (where it is finite).
    p is rounded to the arrays' type before its product with v."""
    dt, (Tq, H, d) = q.dtype, q.shape
    scale = 1 / math.sqrt(d) if scale is None else scale
    group = H // k.shape[1]
    r = 2.0 ** -11 if dt == torch.float16 else 2.0 ** -8
    out = torch.zeros(Tq, H, d, dtype=torch.float64, device=q.device)
    eo = torch.zeros_like(out)
    lse = torch.full((Tq, H), -math.inf, dtype=torch.float64, device=q.device)
    el = torch.zeros_like(lse)
    for here, keys in _sequences(Tq, k.shape[0], q_offsets, kv_offsets, ids):
        if not len(keys):
            continue
        kk, vv = (t[keys.to(t.device)].double().repeat_interleave(group, 1) for t in (k, v))
        p, l, rel, e_lse = _probabilities(q[here].double(), kk, scale, dt)
        o = torch.einsum("hqk,khd->qhd", p, vv)
        size = torch.einsum("hqk,khd->qhd", p, vv.abs())
        # a p below the type's normal range rounds absolutely: 2^-25 of the largest in float16
        tiny = (2.0 ** -25 if dt == torch.float16 else FLUSH) * torch.einsum("hqk,khd->qhd", torch.ones_like(p), vv.abs())
        e = (rel[..., 0].t()[:, :, None] + r + 4 * U * (len(keys) + 8)) * size + tiny
        out[here], eo[here] = o, rounded(o, e, dt)
        lse[here], el[here] = l[..., 0].t(), e_lse[..., 0].t()
    return (out, eo), (lse, el)


def attend_grad(q, k, v, d_out, q_offsets=None, kv_offsets=None, ids=None, scale=None):
    """[(value, bound)] of dq, dk, dv.  p and ds are rounded to the arrays' type before
    the products that sum them; delta is taken from the forward call's rounded output."""
    dt, (Tq, H, d) = q.dtype, q.shape
    Hk = k.shape[1]
    scale = 1 / math.sqrt(d) if scale is None else scale
    group = H // Hk
    r = 2.0 ** -11 if dt == torch.float16 else 2.0 ** -8
    least = 2.0 ** -25 if dt == torch.float16 else FLUSH
    value = [torch.zeros(t.shape, dtype=torch.float64, device=t.device) for t in (q, k, v)]
    bound = [torch.zeros_like(t) for t in value]
    heads = lambda t: t.double().repeat_interleave(group, 1)  # noqa: E731
    shared = lambda t: t.unflatten(1, (Hk, group)).sum(2)  # noqa: E731
    for here, keys in _sequences(Tq, k.shape[0], q_offsets, kv_offsets, ids):
        if not len(keys) or here.start == here.stop:
            continue
        keys = keys.to(q.device)
        qq, do, kk, vv = q[here].double(), d_out[here].double(), heads(k[keys]), heads(v[keys])
        n, m = len(keys), here.stop - here.start
        p, _, rel, _ = _probabilities(qq, kk, scale, dt)
        ep = p * (rel + r) + least
        dp = torch.einsum("qhd,khd->hqk", do, vv)
        dp_size = torch.einsum("qhd,khd->hqk", do.abs(), vv.abs())
        o, o_size = torch.einsum("hqk,khd->qhd", p, vv), torch.einsum("hqk,khd->qhd", p, vv.abs())
        delta = torch.einsum("qhd,qhd->hq", o, do)[..., None]
        # the forward output's own error (p's and its rounding), and the float32 sums
        eo = (rel[..., 0].t()[:, :, None] + 2 * r + 4 * U * (n + 8)) * o_size + least * vv.abs().sum(0) + least
        e_delta = torch.einsum("qhd,qhd->hq", eo, do.abs())[..., None] + (d + 8) * U * torch.einsum(
            "qhd,qhd->hq", o.abs(), do.abs())[..., None]
        x = dp - delta
        ex = e_delta + (d + 8) * U * dp_size + 4 * U * (dp.abs() + delta.abs())
        ds = p * x
        eds = (p * (rel + 4 * U) + FLUSH) * x.abs() + (p + ep) * ex + r * (ds.abs() + (p + ep) * ex) + least

        def put(i, at, val, err):
            value[i][at], bound[i][at] = val, rounded(val, err, dt)

        put(0, here, scale * torch.einsum("hqk,khd->qhd", ds, kk),
            scale * torch.einsum("hqk,khd->qhd", eds + (n + 8) * U * (ds.abs() + eds), kk.abs()))
        put(1, keys, shared(scale * torch.einsum("hqk,qhd->khd", ds, qq)),
            shared(scale * torch.einsum("hqk,qhd->khd", eds + (m * group + 8) * U * (ds.abs() + eds), qq.abs())))
        put(2, keys, shared(torch.einsum("hqk,qhd->khd", p, do)),
            shared(torch.einsum("hqk,qhd->khd", ep + (m * group + 8) * U * (p + ep), do.abs())))
    return list(zip(value, bound))
