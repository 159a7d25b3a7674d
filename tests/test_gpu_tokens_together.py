"""Projections, cross attention and dropout as a block of them is used: forward and
backward on one stream, the block captured and replayed, two streams at once, outputs and
inputs of other streams than the call's."""
import pytest

import tokens_util as ref
from layers_util import within

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
LONG = 100_000_000          # clocks: about 50 ms
BF = torch.bfloat16


@pytest.fixture(scope="module")
def layers():
    from paper_2607_22922_gb300 import build
    build.build()
    from paper_2607_22922_gb300 import ifvs
    L = ifvs.Layers()
    yield L
    L.close()


class Block:
    """y = x + dropout(attend(x Wq, e Wkv) Wo): every query's tokens x look at the
    encoder's states e of their sequence."""

    def __init__(self, lq, lk, D, E, H, Hk, d, seed=1):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        r = lambda *n: torch.randn(*n, generator=g, device="cuda")  # noqa: E731
        self.H, self.Hk, self.d = H, Hk, d
        self.x, self.e, self.dy = r(sum(lq), D).to(BF), r(sum(lk), E).to(BF), r(sum(lq), D).to(BF)
        self.w = {n: (r(o, i) / i ** 0.5).to(BF) for n, o, i in (("q", H * d, D), ("kv", 2 * Hk * d, E), ("o", D, H * d))}
        self.b = {n: (0.1 * r(w.shape[0])).to(BF) for n, w in self.w.items()}
        self.kw = dict(q_offsets=torch.tensor([0] + lq, device="cuda").cumsum(0),
                       kv_offsets=torch.tensor([0] + lk, device="cuda").cumsum(0),
                       kv_ids=torch.where(torch.rand(sum(lk), generator=g, device="cuda") < 0.1, -1, 3).int())

    def forward(self, L, step, stream=None):
        s = dict(stream=stream)
        q = L.linear(self.x, self.w["q"], self.b["q"], **s).view(-1, self.H, self.d)
        kv = L.linear(self.e, self.w["kv"], self.b["kv"], act="silu", **s).view(-1, 2, self.Hk, self.d)
        a, lse = L.attend(q, kv[:, 0], kv[:, 1], lse=True, **self.kw, **s)
        o = L.linear(a.view(len(self.x), -1), self.w["o"], self.b["o"], **s)
        y = L.dropout(o, 0.25, 7, step, residual=self.x, **s)
        return dict(q=q, kv=kv, a=a, lse=lse, o=o, y=y)

    def backward(self, L, f, step, stream=None):
        s = dict(stream=stream)
        g = dict(o=L.dropout(self.dy, 0.25, 7, step, **s))
        g["a"], g["w_o"], g["b_o"] = L.linear_grad(f["a"].view(len(self.x), -1), self.w["o"], g["o"], self.b["o"], **s)
        g["kv"] = torch.empty_like(f["kv"])
        g["q"], _, _ = L.attend_grad(f["q"], f["kv"][:, 0], f["kv"][:, 1], f["a"], f["lse"], g["a"].view_as(f["q"]),
                                     dk=g["kv"][:, 0], dv=g["kv"][:, 1], **self.kw, **s)
        g["e"], g["w_kv"], g["b_kv"] = L.linear_grad(self.e, self.w["kv"], g["kv"].view(len(self.e), -1), self.b["kv"], act="silu", **s)
        g["x"], g["w_q"], g["b_q"] = L.linear_grad(self.x, self.w["q"], g["q"].view(len(self.x), -1), self.b["q"], **s)
        return g

    def check(self, f, g, step):
        """Every call's outputs against its definition at the inputs that it had."""
        n, want = len(self.x), dict(q_offsets=self.kw["q_offsets"], kv_offsets=self.kw["kv_offsets"], ids=self.kw["kv_ids"])
        k, v = f["kv"][:, 0], f["kv"][:, 1]
        within(f["q"].view(n, -1), *ref.linear(self.x, self.w["q"], self.b["q"], "none", None))
        within(f["kv"].view(len(self.e), -1), *ref.linear(self.e, self.w["kv"], self.b["kv"], "silu", None))
        within(f["a"], *ref.attend(f["q"], k, v, **want)[0])
        within(f["o"], *ref.linear(f["a"].view(n, -1), self.w["o"], self.b["o"], "none", None))
        within(f["y"], *ref.dropout(f["o"], 0.25, 7, step, self.x))
        within(g["o"], *ref.dropout(self.dy, 0.25, 7, step, None))
        for names, grads in ((("a", "w_o", "b_o"), ref.linear_grad(f["a"].view(n, -1), self.w["o"], g["o"], self.b["o"], "none")),
                             (("e", "w_kv", "b_kv"), ref.linear_grad(self.e, self.w["kv"], g["kv"].view(len(self.e), -1), self.b["kv"], "silu")),
                             (("x", "w_q", "b_q"), ref.linear_grad(self.x, self.w["q"], g["q"].view(n, -1), self.b["q"], "none"))):
            for name, w in zip(names, grads):
                within(g[name], *w)
        for got, w in zip((g["q"], g["kv"][:, 0], g["kv"][:, 1]), ref.attend_grad(f["q"], k, v, g["a"].view_as(f["q"]), **want)):
            within(got, *w)


SIZES = {"few": ([1], [17], 64, 64, 2, 2, 32),
         "ragged": ([5, 0, 70, 33], [9, 4, 0, 130], 136, 72, 4, 2, 40),
         "many": ([20, 60] * 90, [17, 5, 0] * 60, 64, 128, 8, 2, 64),
         "long": ([300, 420], [513, 600], 128, 64, 2, 1, 128),
         "parts": ([2, 3], [1_500, 2_100], 64, 64, 4, 4, 64)}


def _same(a, b):
    for n in a:
        assert torch.equal(a[n], b[n]), n


@pytest.mark.parametrize("name", sorted(SIZES))
def test_forward_and_backward(layers, name):
    b = Block(*SIZES[name])
    f = b.forward(layers, 3)
    b.check(f, b.backward(layers, f, 3), 3)


@pytest.mark.parametrize("name", sorted(SIZES))
def test_captured_and_replayed_on_new_inputs(layers, name):
    """The replays' outputs are those of eager calls on the same inputs, though eager calls
    of the same tensors, and of larger ones, came between."""
    b, other = Block(*SIZES[name]), Block(*SIZES[name], seed=2)
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    b.backward(layers, b.forward(layers, step), step)         # the workspace has its size
    s, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        f = b.forward(layers, step, s)
        g = b.backward(layers, f, step, s)
    for seed in (2, 3):
        other = Block(*SIZES[name], seed=seed)
        for t, new in zip((b.x, b.e, b.dy, b.kw["kv_ids"]), (other.x, other.e, other.dy, other.kw["kv_ids"])):
            t.copy_(new)
        step.fill_(seed)
        graph.replay()
        torch.cuda.synchronize()
        want = b.forward(layers, seed)
        _same(f, want)
        _same(g, b.backward(layers, want, seed))
        big = Block([700, 60], [2_049, 1_024], 64, 64, 4, 4, 64)
        big.backward(layers, big.forward(layers, 1), 1)
    layers.status()


def test_two_graphs_of_one_handle(layers):
    """Two captures share the handle's workspace; replayed one after the other they are
    right in any order."""
    blocks, graphs, s = [Block(*SIZES[n]) for n in ("parts", "long")], [], torch.cuda.Stream()
    want = [b.forward(layers, 3) for b in blocks]
    grads = [b.backward(layers, f, 3) for b, f in zip(blocks, want)]
    for b in blocks:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            f = b.forward(layers, 3, s)
            g = b.backward(layers, f, 3, s)
        graphs.append((graph, f, g))
    for order in ((0, 1), (1, 0), (1, 1, 0)):
        for i in order:
            for t in list(graphs[i][1].values()) + list(graphs[i][2].values()):
                t.zero_()
            graphs[i][0].replay()
            torch.cuda.synchronize()
            _same(graphs[i][1], want[i])
            _same(graphs[i][2], grads[i])


def test_two_streams_at_once(layers):
    """Calls that use the workspace wait for each other, whatever their streams."""
    blocks = [Block(*SIZES[n]) for n in ("parts", "long", "many")]
    want = [b.forward(layers, 3) for b in blocks]
    grads = [b.backward(layers, f, 3) for b, f in zip(blocks, want)]
    streams = [torch.cuda.Stream() for _ in blocks]
    torch.cuda.synchronize()
    for _ in range(3):
        got = []
        for b, s in zip(blocks, streams):
            with torch.cuda.stream(s):
                f = b.forward(layers, 3, s)
                got.append((f, b.backward(layers, f, 3, s)))
        torch.cuda.synchronize()
        for (f, g), a, b in zip(got, want, grads):
            _same(f, a)
            _same(g, b)


def _operators(layers):
    """name: call, of x [40][64]"""
    r = lambda *n: torch.full(n, 0.5, dtype=BF, device="cuda")  # noqa: E731
    w, b, dy, k = r(24, 64), r(24), r(40, 24), r(30, 2, 32)
    lse = torch.ones(40, 2, device="cuda")
    return {"linear": lambda x, **s: [layers.linear(x, w, b, act="gelu", **s)],
            "linear_grad": lambda x, **s: layers.linear_grad(x, w, dy, b, act="gelu", **s),
            "attend": lambda x, **s: layers.attend(x.view(40, 2, 32), k, k, lse=True, **s),
            "attend_grad": lambda x, **s: layers.attend_grad(x.view(40, 2, 32), k, k, r(40, 2, 32), lse, r(40, 2, 32), **s),
            "dropout": lambda x, **s: [layers.dropout(x, 0.5, 1, residual=x, **s)]}


NAMES = ["linear", "linear_grad", "attend", "attend_grad", "dropout"]


@pytest.mark.parametrize("name", NAMES)
def test_a_call_without_a_stream_follows_the_current_one(layers, name):
    call = _operators(layers)[name]
    x = torch.zeros(40, 64, dtype=BF, device="cuda")
    want = call(torch.full_like(x, 1.5))
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(LONG)
        x.fill_(1.5)
        got = call(x)
    for p, q in zip(want, got):
        assert torch.equal(p, q)


@pytest.mark.parametrize("raw", [False, True])
@pytest.mark.parametrize("name", [n for n in NAMES if n != "attend_grad"])
def test_outputs_are_the_memory_of_the_calls_stream(layers, name, raw):
    """An output that is dropped before its kernel has run: its memory may not go to a
    tensor of the current stream, where the kernel would overwrite it."""
    call = _operators(layers)[name]
    x = torch.full((40, 64), 1.5, dtype=BF, device="cuda")
    call(x)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(LONG)
    out = call(x, stream=s.cuda_stream if raw else s)
    shapes = [(t.shape, t.dtype) for t in out]
    del out
    mine = [torch.full(tuple(n), 7.0, dtype=dt, device="cuda") for n, dt in shapes for _ in range(4)]
    torch.cuda.synchronize()
    for t in mine:
        assert bool((t == 7).all())
