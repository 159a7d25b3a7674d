"""Attention inside wider rows, between guards and in captured graphs, at sizes that reach
each of its kernels: the same bits as with arrays of their own, and what lies between and
beside them is left."""
import pytest

from test_gpu_attend import TYPES, _args
from test_gpu_attend_reach import NAMES, _both, _equal, _lengths

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
every = pytest.mark.parametrize("name", NAMES)
dims = pytest.mark.parametrize("d", [40, 64, 128])


@pytest.fixture(scope="module")
def layers():
    from paper_2607_22922_gb300 import build
    build.build()
    from paper_2607_22922_gb300 import ifvs
    L = ifvs.Layers()
    yield L
    L.close()


@every
@dims
@pytest.mark.parametrize("type_", sorted(TYPES))
def test_rows_with_gaps_and_guards(layers, name, type_, d):
    H, Hk, dt = 8, 4, TYPES[type_]
    q, k, v, d_out, kw = _args(*_lengths(name), H, Hk, d, dt, seed=d, padding=0.05)
    want = _both(layers, q, k, v, d_out, kw)
    n, m = q.shape[0], k.shape[0]
    # places of heads in rows of 16 elements more than they need
    wide = lambda rows, heads, count: torch.full((rows + 4, count * heads * d + 16), 7.0, dtype=dt, device="cuda")  # noqa: E731
    rows, keys = wide(n, H, 5), wide(m, Hk, 4)
    at = lambda a, heads, i: a[2:-2, i * heads * d + 8:(i + 1) * heads * d + 8].unflatten(1, (heads, d))  # noqa: E731
    parts = [at(rows, H, i) for i in range(5)] + [at(keys, Hk, i) for i in range(4)]
    for to, of in zip((parts[0], parts[1], parts[5], parts[6]), (q, d_out, k, v)):
        to.copy_(of)
    lse = torch.full((n + 4, H), 7.0, device="cuda")
    out, dq, dk, dv = parts[2], parts[4], parts[7], parts[8]
    layers.attend(parts[0], parts[5], parts[6], out=out, lse=lse[2:-2], **kw)
    layers.attend_grad(parts[0], parts[5], parts[6], out, lse[2:-2], parts[1], dq=dq, dk=dk, dv=dv, **kw)
    _equal(want, (out, lse[2:-2], dq, dk, dv))
    _equal((q, d_out, k, v), (parts[0], parts[1], parts[5], parts[6]))
    for a in (rows, keys):
        assert bool((a[:2] == 7).all()) and bool((a[-2:] == 7).all())
        assert bool((a[:, :8] == 7).all()) and bool((a[:, -8:] == 7).all())
    assert bool((parts[3] == 7).all()) and bool((lse[:2] == 7).all()) and bool((lse[-2:] == 7).all())


@every
@pytest.mark.parametrize("d", [64, 128])
def test_captured(layers, name, d):
    """Replays take the inputs, the padding and the offsets that the arrays hold then."""
    lq, lk = _lengths(name)
    q, k, v, d_out, kw = _args(lq, lk, 8, 4, d, torch.bfloat16, seed=1, padding=0.1)
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
    grads = [torch.empty_like(t) for t in (q, k, v)]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())

    def call():
        layers.attend(q, k, v, out=out, lse=lse, stream=stream, **kw)
        layers.attend_grad(q, k, v, out, lse, d_out, dq=grads[0], dk=grads[1], dv=grads[2], stream=stream, **kw)

    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        call()
    # other values, and the sequences the other way round
    other = _args(lq[::-1], lk[::-1], 8, 4, d, torch.bfloat16, seed=2, padding=0.2)
    want = _both(layers, *other)
    for a, b in zip((q, k, v, d_out), other):
        a.copy_(b)
    for key, value in other[4].items():
        kw[key].copy_(value)
    for t in (out, lse, *grads):
        t.fill_(7)
    for _ in range(2):
        graph.replay()
        torch.cuda.synchronize()
        _equal(want, (out, lse, *grads))
    layers.status()
