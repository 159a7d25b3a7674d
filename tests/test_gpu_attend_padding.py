"""Queries without keys whose values are not finite: a sequence of padding alone gives
zeros, whatever its queries and their gradients hold, in every form of the kernels."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def layers():
    from paper_2607_22922_gb300 import build
    build.build()
    from paper_2607_22922_gb300 import ifvs
    L = ifvs.Layers()
    yield L
    L.close()


# a few sequences: keys that stay in shared memory, keys that pass, keys in parts; long
# ones; many short ones, of one chunk of keys and of several
LENGTHS = {"few keys": ([30, 20, 40], [40, 50, 33]),
           "more keys": ([30, 20, 40], [200, 150, 170]),
           "parts": ([2, 3, 1], [3_000, 2_000, 2_500]),
           "long": ([300, 200, 400], [400, 700, 500]),
           "many": ([50] * 200, [30] * 200),
           "many, more keys": ([40] * 200, [90] * 200)}


@pytest.mark.parametrize("type_", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("name", sorted(LENGTHS))
def test_queries_without_keys(layers, type_, d, bad, name):
    lq, lk = LENGTHS[name]
    g = torch.Generator(device="cuda")
    g.manual_seed(d)
    off = [torch.tensor([0] + n, device="cuda").cumsum(0) for n in (lq, lk)]
    q, d_out = (torch.randn(sum(lq), 4, d, generator=g, device="cuda").to(type_) for _ in range(2))
    k, v = (torch.randn(sum(lk), 2, d, generator=g, device="cuda").to(type_) for _ in range(2))
    ids = torch.ones(sum(lk), dtype=torch.int32, device="cuda")
    keys, rows = (slice(int(o[1]), int(o[2])) for o in reversed(off))
    ids[keys] = -1
    kw = dict(q_offsets=off[0], kv_offsets=off[1], kv_ids=ids)
    out, lse = layers.attend(q, k, v, lse=True, **kw)
    want = layers.attend_grad(q, k, v, out, lse, d_out, **kw)
    for only in ((q,), (d_out,), (q, d_out)):
        kept = [t[rows].clone() for t in only]
        for t in only:
            t[rows] = bad
        got, got_lse = layers.attend(q, k, v, lse=True, **kw)
        assert torch.equal(got, out) and torch.equal(got_lse, lse)
        assert not got[rows].any() and bool((got_lse[rows] == -float("inf")).all())
        for a, b in zip(layers.attend_grad(q, k, v, got, got_lse, d_out, **kw), want):
            assert torch.equal(a, b)
        for t, was in zip(only, kept):
            t[rows] = was
    assert not want[0][rows].any() and not want[1][keys].any() and not want[2][keys].any()
