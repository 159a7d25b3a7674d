"""The encoder's operators, measured over the sizes that users of them have.

An encoder turns a predicate's tokens (column, operator and bounds of each
clause) into the filter weights' vector w_z.  Six kinds of case, three
operators with their gradients:

``embed``      rows of an embedding table, scaled; id -1 is padding.
``embed_grad`` the table's gradient: the rows of every id summed.
``join``       the norm after a block, its gate (one vector per sequence of
               tokens), the scaled residual and the norm before the next block.
``join_grad``  gradients of the residual, the block's output, the gates and
               both norms' weights.
``ffn``        the gated feed-forward block: y = (act(x Wg^T) * (x Wu^T)) Wo^T.
``ffn_grad``   gradients of x, [Wg; Wu] and Wo from x, the weights and dy.

With ``own`` false the operators run in their plain form, in float32 whatever
the type of the inputs, rounded once at the end.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
EPS = 1e-5
RHO = 0.7071          # residual scale

_layers = None        # the handle that a program makes once


def layers():
    global _layers
    if _layers is None:
        from paper_2607_22922_gb300 import ifvs
        _layers = ifvs.Layers(device=0)
    return _layers


def listed():
    return [
        # one predicate at serving time: 4 clauses of 4 tokens and a start token
        dict(kind="embed", name="embed-predicate", t=17, d=128, v=4096, type="f32"),
        # the tokens of 10^4 queries, wide rows
        dict(kind="embed", name="embed-workload", t=163_847, d=960, v=100_003, type="bf16"),
        # the training batch of 1024 queries
        dict(kind="embed_grad", name="embed_grad-batch", t=17_408, d=128, v=3_760, type="f32"),
        # a large batch on a table of attribute values
        dict(kind="embed_grad", name="embed_grad-workload", t=400_009, d=384, v=50_021, type="bf16"),
        # one predicate
        dict(kind="join", name="join-predicate", t=17, d=128, b=1, type="f32"),
        # the tokens of 10^4 queries, a gate per query
        dict(kind="join", name="join-workload", t=163_847, d=960, b=10_000, type="bf16"),
        # the training batch of 1024 queries, an uneven width
        dict(kind="join_grad", name="join_grad-batch", t=17_393, d=100, b=1_024, type="f16"),
        # one gate for all tokens of a long batch
        dict(kind="join_grad", name="join_grad-long", t=131_101, d=1024, b=1, type="bf16"),
        # one token: the weights are read once for it
        dict(kind="ffn", name="ffn-token", t=1, d=960, f=2560, act="silu", type="bf16"),
        # the tokens of 1024 queries
        dict(kind="ffn", name="ffn-batch", t=17_408, d=960, f=2560, act="gelu", type="bf16"),
        # a training batch of a narrow encoder
        dict(kind="ffn_grad", name="ffn_grad-narrow", t=2_051, d=128, f=344, act="silu", type="f16"),
        # a training batch of a wide encoder: the largest case
        dict(kind="ffn_grad", name="ffn_grad-wide", t=16_411, d=1024, f=4096, act="silu", type="bf16"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["embed", "embed_grad", "join", "join_grad", "ffn", "ffn_grad"])
    if kind.startswith("ffn"):
        d = 8 * _log_int(rng, 8, 192)           # 64 .. 1536
        f = 8 * _log_int(rng, 16, 640)          # 128 .. 5120
        most = int(3.2e11 / (6.0 * d * f))      # within the largest listed case
        return dict(kind=kind, t=_log_int(rng, 1, min(20_000, most)), d=d, f=f, act=rng.choice(["silu", "gelu", "relu"]),
                    type=rng.choice(["bf16", "f16"]))
    d = _log_int(rng, 32, 1536)
    if rng.random() < 0.5:
        d = max(32, d // 8 * 8)
    t = _log_int(rng, 1, min(300_000, int(1.3e8 / d)))
    case = dict(kind=kind, t=t, d=d, type=rng.choice(["f32", "bf16", "f16"]))
    if kind.startswith("embed"):
        case["v"] = _log_int(rng, 40, min(200_000, int(1.3e8 / d)))
    else:
        case["b"] = min(t, rng.choice([1, _log_int(rng, 1, 10_000)]))
    return case


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    dt = DTYPES[case["type"]]
    t, d, kind = case["t"], case["d"], case["kind"]
    s = dict(case=case)
    if kind.startswith("embed"):
        v = case["v"]
        # a few ids (columns, operators) make up half of the tokens, the
        # bounds' buckets follow a power law over the rest, 3 % is padding
        few = torch.randint(0, min(v, 12), (t,), generator=g, device=DEV)
        u = torch.rand(t, generator=g, device=DEV)
        tail = (v * u ** 3).long().clamp_(max=v - 1)
        ids = torch.where(torch.rand(t, generator=g, device=DEV) < 0.5, few, tail)
        ids[torch.rand(t, generator=g, device=DEV) < 0.03] = -1
        s["ids"] = ids.int()
        s["scale"] = math.sqrt(d)
        if kind == "embed":
            s["table"] = (_normal(g, v, d) / math.sqrt(d)).to(dt)
            s["out"] = torch.empty(t, d, dtype=dt, device=DEV)
        else:
            s["dout"] = _normal(g, t, d).to(dt)
            s["out"] = torch.empty(v, d, dtype=dt, device=DEV)
    elif kind.startswith("join"):
        b = case["b"]
        cuts = torch.randint(0, t + 1, (b + 1,), generator=g, device=DEV).sort().values   # empty ones among them
        cuts[0], cuts[b] = 0, t
        s["offsets"] = cuts
        s["lengths"] = cuts[1:] - cuts[:-1]
        s["y"] = (0.5 * _normal(g, t, d)).to(dt)
        s["gate"] = (1 + 0.3 * _normal(g, b, d)).to(dt)
        s["w_post"] = (1 + 0.1 * _normal(g, d)).to(dt)
        s["w_pre"] = (1 + 0.1 * _normal(g, d)).to(dt)
        s["x"] = (1.5 * _normal(g, t, d)).to(dt)       # the residual; in the gradient the joined one
        if kind == "join_grad":
            s["dx_ext"] = _normal(g, t, d).to(dt)
            s["dn"] = _normal(g, t, d).to(dt)
            s["out"] = [torch.empty(n, d, dtype=dt, device=DEV) for n in (t, t, b)] + [
                torch.empty(d, dtype=dt, device=DEV) for _ in range(2)]
        else:
            s["out"] = [torch.empty(t, d, dtype=dt, device=DEV) for _ in range(2)]
    else:
        f = case["f"]
        s["x"] = _normal(g, t, d).to(dt)
        s["w_in"] = (_normal(g, 2 * f, d) / math.sqrt(d)).to(dt)
        s["w_out"] = (_normal(g, d, f) / math.sqrt(f)).to(dt)
        if kind == "ffn_grad":
            s["dy"] = _normal(g, t, d).to(dt)
            s["out"] = [torch.empty(n, m, dtype=dt, device=DEV) for n, m in ((t, d), (2 * f, d), (d, f))]
        else:
            s["out"] = torch.empty(t, d, dtype=dt, device=DEV)
    return s


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    kind, o = s["case"]["kind"], s["out"]
    at = layers()
    stream = torch.cuda.current_stream()
    if kind == "embed":
        return at.embed(s["table"], s["ids"], s["scale"], out=o, stream=stream)
    if kind == "embed_grad":
        return at.embed_grad(s["dout"], s["ids"], s["scale"], d_table=o, stream=stream)
    if kind == "join":
        return at.norm_join(s["x"], s["y"], s["gate"], s["w_post"], s["w_pre"], offsets=s["offsets"], res_scale=RHO,
                            eps=EPS, x_out=o[0], n_out=o[1], stream=stream)
    if kind == "join_grad":
        return at.norm_join_grad(s["x"], s["y"], s["gate"], s["w_post"], s["w_pre"], s["dx_ext"], s["dn"],
                                 offsets=s["offsets"], res_scale=RHO, eps=EPS, dx=o[0], dy=o[1], d_gate=o[2],
                                 d_w_post=o[3], d_w_pre=o[4], stream=stream)
    act = s["case"]["act"]
    if kind == "ffn":
        return at.ffn(s["x"], s["w_in"], s["w_out"], act=act, y=o, stream=stream)
    return at.ffn_grad(s["x"], s["w_in"], s["w_out"], s["dy"], act=act, dx=o[0], d_w_in=o[1], d_w_out=o[2],
                       stream=stream)


# ------------------------------------------------------------- plain forms

def _sequence_of(s):
    b, t = s["case"]["b"], s["case"]["t"]
    return torch.repeat_interleave(torch.arange(b, device=DEV), s["lengths"], output_size=t)


def _phi(x):
    return 0.5 * (1 + torch.erf(x * math.sqrt(0.5)))


def _act(name, x):
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


def _run_plain(s):
    case = s["case"]
    kind, dt = case["kind"], DTYPES[case["type"]]
    if kind == "embed":
        ids = s["ids"].long()
        rows = s["table"][ids.clamp(min=0)].float() * s["scale"]
        return torch.where((ids >= 0)[:, None], rows, torch.zeros_like(rows)).to(dt)
    if kind == "embed_grad":
        ids = s["ids"].long()
        total = torch.zeros(case["v"] + 1, case["d"], device=DEV)      # the last row takes the padding
        total.index_add_(0, torch.where(ids >= 0, ids, torch.full_like(ids, case["v"])), s["dout"].float())
        return (total[:-1] * s["scale"]).to(dt)
    if kind.startswith("join"):
        x, y, gate, wp, wn = (s[k].float() for k in ("x", "y", "gate", "w_post", "w_pre"))
        gates = gate if case["b"] == 1 else gate[_sequence_of(s)]
        iy = torch.rsqrt((y * y).mean(1, keepdim=True) + EPS)
        u = y * iy
        if kind == "join":
            xo = RHO * x + gates * (wp * u)
            no = wn * xo * torch.rsqrt((xo * xo).mean(1, keepdim=True) + EPS)
            return xo.to(dt), no.to(dt)
        dn, dxo = s["dn"].float(), s["dx_ext"].float()
        ix = torch.rsqrt((x * x).mean(1, keepdim=True) + EPS)
        z = dn * wn
        dxo = dxo + ix * (z - x * (ix * ix * (z * x).mean(1, keepdim=True)))
        dn_x = (dn * x * ix).sum(0)
        t = dxo * u
        if case["b"] == 1:
            sums = t.sum(0, keepdim=True)
        else:
            sums = torch.zeros_like(gate).index_add_(0, _sequence_of(s), t)
        du = gates * wp * dxo
        dy = iy * (du - u * (du * u).mean(1, keepdim=True))
        return ((RHO * dxo).to(dt), dy.to(dt), (wp * sums).to(dt), (gate * sums).sum(0).to(dt), dn_x.to(dt))
    f = case["f"]
    x, w_in, w_out = s["x"].float(), s["w_in"].float(), s["w_out"].float()
    gu = x @ w_in.t()
    g, u = gu[:, :f], gu[:, f:]
    a = _act(case["act"], g)
    if kind == "ffn":
        return ((a * u) @ w_out.t()).to(dt)
    dy = s["dy"].float()
    dh = dy @ w_out
    dgu = torch.cat([dh * u * _act_slope(case["act"], g), dh * a], 1)
    return (dgu @ w_in).to(dt), (dgu.t() @ x).to(dt), (dy.t() @ (a * u)).to(dt)


# ---------------------------------------------- 64 bits, from the definitions

def exact(case, seed):
    """Each operator's definition in float64; the gradients by differentiating it."""
    s = prepare(case, seed)
    kind = case["kind"]
    if kind.startswith("embed"):
        ids = s["ids"].cpu().numpy()
        if kind == "embed":
            table = s["table"].double().cpu().numpy()
            out = np.zeros((case["t"], case["d"]))
            out[ids >= 0] = s["scale"] * table[ids[ids >= 0]]
            return torch.from_numpy(out)
        rows = s["dout"].double().cpu().numpy()
        order = np.argsort(ids, kind="stable")
        order = order[ids[order] >= 0]
        out = np.zeros((case["v"], case["d"]))
        if order.size:
            found, first = np.unique(ids[order], return_index=True)
            out[found] = s["scale"] * np.add.reduceat(rows[order], first, axis=0)
        return torch.from_numpy(out)
    names = [k for k in ("x", "y", "gate", "w_post", "w_pre", "w_in", "w_out") if k in s]
    with torch.enable_grad():
        p = {k: s[k].double().requires_grad_() for k in names}
        if kind.startswith("join"):
            seq = torch.bucketize(torch.arange(case["t"], device=DEV), s["offsets"][1:], right=True)
            norm = lambda v: v / torch.sqrt(torch.sum(v ** 2, 1, keepdim=True) / case["d"] + EPS)  # noqa: E731
            post = norm(p["y"]) * p["w_post"] * p["gate"].index_select(0, seq)
            if kind == "join":
                xo = RHO * p["x"] + post
                return xo.detach(), (norm(xo) * p["w_pre"]).detach()
            # x is the joined residual: x = RHO * before + post
            before = ((s["x"].double() - post.detach()) / RHO).requires_grad_()
            xo = RHO * before + post
            n = norm(xo) * p["w_pre"]
            wrt = [before, p["y"], p["gate"], p["w_post"], p["w_pre"]]
            return list(torch.autograd.grad([xo, n], wrt, [s["dx_ext"].double(), s["dn"].double()]))
        f = case["f"]
        g = p["x"].matmul(p["w_in"][:f].t())
        u = p["x"].matmul(p["w_in"][f:].t())
        if case["act"] == "silu":
            a = g / (1 + torch.exp(-g))
        elif case["act"] == "gelu":
            a = g * torch.erfc(-g / math.sqrt(2)) / 2
        else:
            a = g.clamp(min=0)
        y = (a * u).matmul(p["w_out"].t())
        if kind == "ffn":
            return y.detach()
        return list(torch.autograd.grad(y, [p["x"], p["w_in"], p["w_out"]], s["dy"].double()))


def work(case):
    t, d = case["t"], case["d"]
    e = 4 if case["type"] == "f32" else 2
    kind = case["kind"]
    if kind == "embed":
        # of the table the rows that the tokens name: the expected number for prepare()'s distribution
        edge = np.cbrt(np.arange(case["v"] + 1) / case["v"])
        named = float(np.sum(-np.expm1(-0.485 * t * np.diff(edge))))
        return {"bytes": 4 * t + (t + min(t, named)) * d * e, "flops": t * d}
    if kind == "embed_grad":
        return {"bytes": 4 * t + (t + case["v"]) * d * e, "flops": t * d}
    if kind == "join":
        return {"bytes": (4 * t + case["b"] + 2) * d * e + 8 * case["b"], "flops": 12 * t * d}
    if kind == "join_grad":
        return {"bytes": (6 * t + 2 * case["b"] + 4) * d * e + 8 * case["b"], "flops": 30 * t * d}
    f = case["f"]
    if kind == "ffn":
        return {"bytes": (2 * t * d + 3 * d * f) * e, "flops": 6.0 * t * d * f}
    # the gradient starts from x: both projections again, then five products
    return {"bytes": (3 * t * d + 6 * d * f) * e, "flops": 16.0 * t * d * f}
