"""Operators of an encoder whose tokens attend to one another, measured over the
sizes that users of them have.

The encoder's blocks work on tokens one by one.  These mix them: the tokens of a
query (one per subspace, or one in all) attend to the tokens of its predicate,
or of any other encoder, through projections, with dropout while it trains.
Five kinds of case, three operators with their gradients:

``linear``       y = residual + act(x W^T + bias).
``linear_grad``  gradients of x, W and the bias.
``attend``       per sequence and head, each query's mean of the values weighted
                 by softmax(scale q k); keys whose id is negative are padding; a
                 query without keys gives zeros.  Heads may share keys and values.
``attend_grad``  gradients of q, k and v from those of the output.
``dropout``      residual + x / (1 - p) where the element's random number says
                 so, else residual; of a gradient it is the same call.

With ``own`` false the operators run in their plain form, in float32 whatever
the type of the inputs, rounded once at the end.
"""
import math

import torch

own = False

DEV = "cuda"
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}

_layers = None        # the handle that a program makes once


def layers():
    global _layers
    if _layers is None:
        from paper_2607_22922_gb300 import ifvs
        _layers = ifvs.Layers(device=0)
    return _layers


def listed():
    return [
        # serving: the output projection of one predicate's pooled token
        dict(kind="linear", name="linear-token", t=1, d_in=960, d_out=960, act="none", bias=True, residual=False,
             type="bf16"),
        # the tokens of 1024 queries, up to the hidden width
        dict(kind="linear", name="linear-batch", t=17_408, d_in=960, d_out=2560, act="gelu", bias=True,
             residual=True, type="bf16"),
        # a training batch of a narrow encoder
        dict(kind="linear_grad", name="linear_grad-narrow", t=2_051, d_in=128, d_out=344, act="silu", bias=True,
             type="f16"),
        # a training batch of a wide encoder: the largest case
        dict(kind="linear_grad", name="linear_grad-wide", t=16_411, d_in=1024, d_out=4096, act="gelu", bias=True,
             type="bf16"),
        # serving: one query's token and the 17 tokens of its predicate
        dict(kind="attend", name="attend-predicate", b=1, q_min=1, q_max=1, k_min=17, k_max=17,
             heads=4, kv_heads=4, dh=32, ids=False, lse=False, fused=False, type="bf16"),
        # training: 1024 queries of 120 subspace tokens, predicates of 0 to 65 tokens, padding among them
        dict(kind="attend", name="attend-batch", b=1024, q_min=120, q_max=120, k_min=0, k_max=65,
             heads=8, kv_heads=2, dh=64, ids=True, lse=True, fused=True, type="bf16"),
        # serving: one token for each of 8 workloads that took about 16 000 tokens to describe
        dict(kind="attend", name="attend-states", b=8, q_min=1, q_max=1, k_min=16_001, k_max=16_801,
             heads=8, kv_heads=8, dh=64, ids=False, lse=False, fused=False, type="f16"),
        # every token of a batch attends to the tokens of 1024 predicates
        dict(kind="attend", name="attend-workload", b=1, q_min=4_099, q_max=4_099, k_min=17_403, k_max=17_403,
             heads=8, kv_heads=8, dh=128, ids=False, lse=False, fused=False, type="bf16"),
        # training as above, with 64 subspace tokens
        dict(kind="attend_grad", name="attend_grad-batch", b=1000, q_min=60, q_max=68, k_min=1, k_max=65,
             heads=8, kv_heads=2, dh=64, ids=True, lse=True, fused=True, type="f16"),
        # four workloads, long on both sides
        dict(kind="attend_grad", name="attend_grad-workload", b=4, q_min=1_301, q_max=1_701, k_min=3_500, k_max=5_003,
             heads=8, kv_heads=8, dh=64, ids=False, lse=True, fused=False, type="bf16"),
        # the joined tokens of a small training batch
        dict(kind="dropout", name="dropout-batch", t=17_393, d=100, p=0.1, residual=True, type="f32"),
        # the gradient over the tokens of 10^4 queries
        dict(kind="dropout", name="dropout-workload", t=163_847, d=960, p=0.25, residual=False, type="bf16"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["linear", "linear_grad", "attend", "attend", "attend_grad", "attend_grad", "dropout"])
    if kind == "dropout":
        d = _log_int(rng, 32, 1536)
        return dict(kind=kind, t=_log_int(rng, 1, min(200_000, int(1.5e8 / d))), d=d, p=rng.choice([0.05, 0.1, 0.25, 0.5]),
                    residual=rng.random() < 0.5, type=rng.choice(["f32", "bf16", "f16"]))
    kind_of_type = rng.choice(["bf16", "f16"])
    if kind.startswith("linear"):
        d_in, d_out = 8 * _log_int(rng, 8, 512), 8 * _log_int(rng, 8, 512)      # 64 .. 4096
        most = int(4e11 / (6.0 * d_in * d_out))                                 # within the largest listed case
        case = dict(kind=kind, t=_log_int(rng, 1, min(20_000, most)), d_in=d_in, d_out=d_out,
                    act=rng.choice(["none", "silu", "gelu", "relu"]), bias=rng.random() < 0.7, type=kind_of_type)
        if kind == "linear":
            case["residual"] = rng.random() < 0.5
        return case
    kv_heads = rng.choice([1, 2, 4, 8])
    heads = kv_heads * rng.choice([1, 1, 2, 4])
    dh = rng.choice([32, 64, 128]) if rng.random() < 0.6 else 8 * rng.randint(2, 16)
    form = rng.choice(["short", "single", "long"])
    if form == "short":
        b = _log_int(rng, 1, 4096)
        q1, k1 = _log_int(rng, 1, 128), _log_int(rng, 4, 96)
        q, k = [rng.choice([q1, (q1 + 1) // 2]), q1], [rng.choice([0, 1, k1]), k1]
    elif form == "single":
        b = _log_int(rng, 1, 64)
        k1 = _log_int(rng, 64, 20_000)
        q, k = [1, 1], [k1 - rng.randint(0, k1 // 4), k1]
    else:
        b = rng.choice([1, 2, 3, 5, 8])
        q1, k1 = _log_int(rng, 64, 4_500), _log_int(rng, 64, 16_000)
        q, k = [q1 - rng.randint(0, q1 // 4), q1], [k1 - rng.randint(0, k1 // 4), k1]
    if b == 1:
        q, k = [q[1]] * 2, [k[1]] * 2
    # the scores fit, and the work is within the largest listed case
    while b * q[1] * k[1] * heads > min(6e8, 3e11 / (10 * dh)) or b * max(q[1] * heads, k[1] * kv_heads) * dh > 8e7:
        if b > 8:
            b = b // 2
        else:
            q, k = [max(1, v // 2) for v in q], [max(1, v // 2) for v in k]
    grad = kind == "attend_grad"
    return dict(kind=kind, b=b, q_min=q[0], q_max=q[1], k_min=k[0], k_max=k[1], heads=heads, kv_heads=kv_heads, dh=dh,
                ids=rng.random() < 0.4, lse=grad or rng.random() < 0.5, fused=rng.random() < 0.4, type=kind_of_type)


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


def _spread(n, lo, hi):
    """n lengths spread evenly over lo .. hi."""
    return torch.linspace(lo, hi, n).round().long()


def _offsets(lengths):
    return torch.cat([torch.zeros(1, dtype=torch.int64), lengths.cumsum(0)]).to(DEV)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    dt = DTYPES[case["type"]]
    kind = case["kind"]
    s = dict(case=case)
    if kind == "dropout":
        t, d = case["t"], case["d"]
        s["x"] = _normal(g, t, d).to(dt)
        s["residual"] = _normal(g, t, d).to(dt) if case["residual"] else None
        s["seed"], s["step"] = (int(v) for v in torch.randint(0, 2**62, (2,), generator=g, device=DEV))
        s["out"] = torch.empty(t, d, dtype=dt, device=DEV)
    elif kind.startswith("linear"):
        t, i, o = case["t"], case["d_in"], case["d_out"]
        s["x"] = _normal(g, t, i).to(dt)
        s["w"] = (_normal(g, o, i) / math.sqrt(i)).to(dt)
        s["bias"] = (0.1 * _normal(g, o)).to(dt) if case["bias"] else None
        if kind == "linear":
            s["residual"] = _normal(g, t, o).to(dt) if case["residual"] else None
            s["out"] = torch.empty(t, o, dtype=dt, device=DEV)
        else:
            s["dy"] = _normal(g, t, o).to(dt)
            s["out"] = [torch.empty(n, i, dtype=dt, device=DEV) for n in (t, o)] + [
                torch.empty(o, dtype=dt, device=DEV) if case["bias"] else None]
    else:
        b, h, hk, dh = case["b"], case["heads"], case["kv_heads"], case["dh"]
        order = torch.Generator()
        order.manual_seed(seed)
        lq, lk = (_spread(b, case[n + "_min"], case[n + "_max"])[torch.randperm(b, generator=order)] for n in ("q", "k"))
        tq, tk = int(lq.sum()), int(lk.sum())
        s["q_offsets"], s["kv_offsets"] = _offsets(lq), _offsets(lk)
        s["ids"] = None
        if case["ids"]:      # 3 % of the keys are padding
            ids = torch.randint(0, 4096, (tk,), generator=g, device=DEV)
            ids[torch.rand(tk, generator=g, device=DEV) < 0.03] = -1
            s["ids"] = ids.int()
        s["scale"] = 1 / math.sqrt(dh)
        s["q"] = _normal(g, tq, h, dh).to(dt)

        def pair(make):      # keys and values: of one projection's output, or apart
            if case["fused"]:
                both = make(tk, 2, hk, dh)
                return both[:, 0], both[:, 1]
            return make(tk, hk, dh), make(tk, hk, dh)

        s["k"], s["v"] = pair(lambda *n: _normal(g, *n).to(dt))
        empty = lambda *n: torch.empty(*n, dtype=dt, device=DEV)  # noqa: E731
        if kind == "attend":
            s["out"] = empty(tq, h, dh)
            s["lse"] = torch.empty(tq, h, device=DEV) if case["lse"] else None
        else:
            s["d_out"] = _normal(g, tq, h, dh).to(dt)
            out, s["lse"] = _attend(s)
            s["forward"] = out.to(dt)
            s["out"] = [empty(tq, h, dh), *pair(empty)]
    return s


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    case, at, o = s["case"], layers(), s["out"]
    kind, stream = case["kind"], torch.cuda.current_stream()
    if kind == "dropout":
        return at.dropout(s["x"], case["p"], s["seed"], s["step"], residual=s["residual"], out=o, stream=stream)
    if kind == "linear":
        return at.linear(s["x"], s["w"], s["bias"], act=case["act"], residual=s["residual"], y=o, stream=stream)
    if kind == "linear_grad":
        got = at.linear_grad(s["x"], s["w"], s["dy"], s["bias"], act=case["act"], dx=o[0], d_w=o[1], d_bias=o[2], stream=stream)
        return got if case["bias"] else got[:2]
    if kind == "attend":
        got = at.attend(s["q"], s["k"], s["v"], q_offsets=s["q_offsets"], kv_offsets=s["kv_offsets"], kv_ids=s["ids"],
                        scale=s["scale"], out=o, lse=s["lse"], stream=stream)
        return got if case["lse"] else got[0]
    return at.attend_grad(s["q"], s["k"], s["v"], s["forward"], s["lse"], s["d_out"], q_offsets=s["q_offsets"],
                          kv_offsets=s["kv_offsets"], kv_ids=s["ids"], scale=s["scale"], dq=o[0], dk=o[1], dv=o[2], stream=stream)


# ------------------------------------------------------------- plain forms

def _phi(x):
    return 0.5 * (1 + torch.erf(x * math.sqrt(0.5)))


def _act(name, x):
    if name == "none":
        return x
    if name == "relu":
        return torch.where(x > 0, x, torch.zeros_like(x))
    return x * (torch.sigmoid(x) if name == "silu" else _phi(x))


def _act_slope(name, x):
    if name == "relu":
        return (x > 0).to(x.dtype)
    if name == "silu":
        p = torch.sigmoid(x)
        return p * (1 + x * (1 - p))
    return _phi(x) + x * torch.exp(-0.5 * x * x) * (1 / math.sqrt(2 * math.pi))


def _places(offsets, most):
    """Of every sequence's places 0 .. most - 1 the tokens, and whether there is one."""
    at = offsets[:-1, None] + torch.arange(most, device=DEV)[None]
    there = at < offsets[1:, None]
    return torch.where(there, at, torch.zeros_like(at)), there


def _pad(x, at, there):
    return x[at].float() * there[:, :, None, None] if x.shape[0] else x.new_zeros(*at.shape, *x.shape[1:]).float()


def _scores(s):
    """q, k [B][places][kv heads][(group)][dh], the scores and which of them count."""
    case = s["case"]
    qa, qt = _places(s["q_offsets"], case["q_max"])
    ka, kt = _places(s["kv_offsets"], case["k_max"])
    q = _pad(s["q"], qa, qt).unflatten(2, (case["kv_heads"], case["heads"] // case["kv_heads"]))
    k = _pad(s["k"], ka, kt)
    if s["ids"] is not None and s["ids"].shape[0]:
        kt = kt & (s["ids"][ka] >= 0)
    score = torch.einsum("bqhgd,bkhd->bhgqk", q, k) * s["scale"]
    return q, k, score.masked_fill(~kt[:, None, None, None], -math.inf), (qt, ka, kt)


def _softmax(score):
    m = score.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    e = torch.exp(score - m)
    total = e.sum(-1, keepdim=True)
    return e / torch.where(total > 0, total, torch.ones_like(total)), (m + torch.log(total))[..., 0]


def _attend(s):
    """out [Tq][heads][dh] and the logarithm of the softmax's sum [Tq][heads], float32"""
    case = s["case"]
    _, _, score, (qt, ka, _) = _scores(s)
    p, lse = _softmax(score)
    _, there = _places(s["kv_offsets"], case["k_max"])
    out = torch.einsum("bhgqk,bkhd->bqhgd", p, _pad(s["v"], ka, there))
    return out.flatten(2, 3)[qt], lse.permute(0, 3, 1, 2).flatten(2, 3)[qt]


def _attend_grad(s):
    case = s["case"]
    group = (case["kv_heads"], case["heads"] // case["kv_heads"])
    q, k, score, (qt, ka, _) = _scores(s)
    p, _ = _softmax(score)
    qa, _ = _places(s["q_offsets"], case["q_max"])
    _, there = _places(s["kv_offsets"], case["k_max"])
    v, d_out = _pad(s["v"], ka, there), _pad(s["d_out"], qa, qt).unflatten(2, group)
    dv = torch.einsum("bhgqk,bqhgd->bkhd", p, d_out)
    dp = torch.einsum("bqhgd,bkhd->bhgqk", d_out, v)
    ds = p * (dp - (p * dp).sum(-1, keepdim=True)) * s["scale"]
    dq = torch.einsum("bhgqk,bkhd->bqhgd", ds, k)
    dk = torch.einsum("bhgqk,bqhgd->bkhd", ds, q)
    return dq.flatten(2, 3)[qt], dk[there], dv[there]


def _words(seed, step, blocks):
    """Philox 4x32 with 10 rounds (Salmon, Moraes, Dror and Shaw, SC 2011): the counter
    is the block's number and the step, the key is the seed.  int64 products wrap,
    which keeps their 64 bits."""
    low = 0xFFFFFFFF
    n = torch.arange(blocks, device=DEV)
    c = [n & low, n >> 32, torch.full_like(n, step & low), torch.full_like(n, step >> 32)]
    key = [seed & low, seed >> 32]
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(b >> 32 & low) ^ c[1] ^ key[0], b & low, (a >> 32 & low) ^ c[3] ^ key[1], a & low]
        key = [(key[0] + 0x9E3779B9) & low, (key[1] + 0xBB67AE85) & low]
    return torch.stack(c, 1).flatten()


def _run_plain(s):
    case = s["case"]
    kind, dt = case["kind"], DTYPES[case["type"]]
    if kind == "dropout":
        x = s["x"].float()
        keep = _words(s["seed"], s["step"], (x.numel() + 3) // 4)[: x.numel()].view_as(x) >= round(case["p"] * 2**32)
        out = torch.where(keep, x * (1 / (1 - case["p"])), torch.zeros_like(x))
        return (out if s["residual"] is None else s["residual"].float() + out).to(dt)
    if kind.startswith("attend"):
        if kind == "attend_grad":
            return [g.to(dt) for g in _attend_grad(s)]
        out, lse = _attend(s)
        return (out.to(dt), lse) if case["lse"] else out.to(dt)
    x, w = s["x"].float(), s["w"].float()
    z = None
    if kind == "linear" or case["act"] != "none":
        z = x @ w.t()
        if s["bias"] is not None:
            z = z + s["bias"].float()
    if kind == "linear":
        y = _act(case["act"], z)
        return (y if s["residual"] is None else y + s["residual"].float()).to(dt)
    dz = s["dy"].float()
    if case["act"] != "none":
        dz = dz * _act_slope(case["act"], z)
    got = [(dz @ w).to(dt), (dz.t() @ x).to(dt)]
    return got + [dz.sum(0).to(dt)] if case["bias"] else got


# ---------------------------------------------- 64 bits, from the definitions

def _random_words(seed, step, first, count):
    """Words first .. first + count - 1 of Philox4x32-10, products by 16-bit halves."""
    def product(a, m):
        """high and low 32 bits of a m"""
        p0, p1 = a * (m & 0xFFFF), a * (m >> 16)        # a m = p0 + 2^16 p1, each below 2^48
        mid = (p0 >> 16) + p1
        return mid >> 16, ((mid & 0xFFFF) << 16) | (p0 & 0xFFFF)

    i = torch.arange(first, first + count, dtype=torch.int64, device=DEV)
    block, word = i // 4, i % 4
    x0, x1 = block % 2**32, block // 2**32
    x2, x3 = torch.full_like(i, step % 2**32), torch.full_like(i, step // 2**32)
    for r in range(10):
        k0, k1 = (seed + r * 0x9E3779B9) % 2**32, (seed // 2**32 + r * 0xBB67AE85) % 2**32
        (h0, l0), (h1, l1) = product(x0, 0xD2511F53), product(x2, 0xCD9E8D57)
        x0, x1, x2, x3 = h1 ^ x1 ^ k0, l1, h0 ^ x3 ^ k1, l0
    return torch.where(word < 2, torch.where(word == 0, x0, x1), torch.where(word == 2, x2, x3))


def exact(case, seed):
    """Each operator's definition in float64; the gradients by differentiating it."""
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "dropout":
        x = s["x"].double().flatten()
        out = torch.zeros_like(x) if s["residual"] is None else s["residual"].double().flatten()
        for first in range(0, x.numel(), 1 << 24):
            part = x[first:first + (1 << 24)]
            kept = _random_words(s["seed"], s["step"], first, part.numel()).double() / 2**32 >= round(case["p"] * 2**32) / 2**32
            out[first:first + (1 << 24)] += torch.where(kept, part / (1 - case["p"]), part.new_zeros(()))
        return out.view(case["t"], case["d"])
    with torch.enable_grad():
        if kind.startswith("linear"):
            p = {k: s[k].double().requires_grad_() for k in ("x", "w", "bias") if s[k] is not None}
            z = torch.nn.functional.linear(p["x"], p["w"], p.get("bias"))
            if case["act"] == "silu":
                z = z / (1 + torch.exp(-z))
            elif case["act"] == "gelu":
                z = z * torch.erfc(-z / math.sqrt(2)) / 2
            elif case["act"] == "relu":
                z = z.clamp(min=0)
            if kind == "linear":
                return (z if s["residual"] is None else z + s["residual"].double()).detach()
            return list(torch.autograd.grad(z, list(p.values()), s["dy"].double()))
        group = case["heads"] // case["kv_heads"]
        out = torch.zeros_like(s["q"], dtype=torch.float64)
        lse = torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device=DEV)
        grads = [torch.zeros_like(s[n], dtype=torch.float64) for n in ("q", "k", "v")]
        qo, ko = s["q_offsets"].tolist(), s["kv_offsets"].tolist()
        for b in range(case["b"]):
            here = slice(qo[b], qo[b + 1])
            keys = torch.arange(ko[b], ko[b + 1], device=DEV)
            if s["ids"] is not None:
                keys = keys[s["ids"][keys] >= 0]
            if not len(keys) or qo[b] == qo[b + 1]:
                continue
            q, k, v = (t.double().requires_grad_() for t in (s["q"][here], s["k"][keys], s["v"][keys]))
            score = torch.matmul(q.transpose(0, 1), k.repeat_interleave(group, 1).permute(1, 2, 0)) * s["scale"]
            lse[here] = torch.logsumexp(score.detach(), -1).t()
            o = torch.matmul(torch.softmax(score, -1), v.repeat_interleave(group, 1).transpose(0, 1)).transpose(0, 1)
            out[here] = o.detach()
            if kind == "attend_grad":
                dq, dk, dv = torch.autograd.grad(o, [q, k, v], s["d_out"][here].double())
                grads[0][here] = dq
                grads[1][keys], grads[2][keys] = dk, dv
        if kind == "attend_grad":
            return grads
        return (out, lse) if case["lse"] else out


def work(case):
    e = 4 if case["type"] == "f32" else 2
    kind = case["kind"]
    if kind == "dropout":
        n = case["t"] * case["d"]
        return {"bytes": (3 if case["residual"] else 2) * n * e, "flops": 2 * n}
    if kind.startswith("linear"):
        t, i, o, bias = case["t"], case["d_in"], case["d_out"], case["d_out"] if case["bias"] else 0
        if kind == "linear":
            return {"bytes": (t * i + o * i + bias + (2 if case["residual"] else 1) * t * o) * e, "flops": 2.0 * t * i * o}
        # the gradient starts from x: with an activation the product again
        products = 4.0 if case["act"] == "none" else 6.0
        return {"bytes": (2 * t * i + 2 * o * i + t * o + 2 * bias) * e, "flops": products * t * i * o}
    h, hk, dh = case["heads"], case["kv_heads"], case["dh"]
    tq, tk = (int(_spread(case["b"], case[n + "_min"], case[n + "_max"]).sum()) for n in ("q", "k"))
    pairs = tq * tk / case["b"]
    other = 8 * (2 * case["b"] + 2) + (4 * tk if case["ids"] else 0) + (4 * tq * h if case["lse"] else 0)
    if kind == "attend":
        return {"bytes": 2 * (tq * h + tk * hk) * dh * e + other, "flops": 4.0 * pairs * h * dh}
    return {"bytes": 4 * (tq * h + tk * hk) * dh * e + other, "flops": 10.0 * pairs * h * dh}
