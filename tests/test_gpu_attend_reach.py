"""What must not be seen, at sizes that reach each of attention's kernels on the device at
hand (the batches of many sequences have five sequences an SM, twice what their rules ask):
values that are no numbers in padding among keys that count, in a sequence without keys, and
in another sequence change no bit of the rest; equal calls give equal bits."""
import pytest

from test_gpu_attend import TYPES, _args

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def layers():
    from paper_2607_22922_gb300 import build
    build.build()
    from paper_2607_22922_gb300 import ifvs
    L = ifvs.Layers()
    yield L
    L.close()


def _many():
    return 5 * torch.cuda.get_device_properties(0).multi_processor_count


def _lengths(name):
    n = _many()
    return {"few rows": ([2, 1, 3], [3_000, 2_000, 2_500]),
            "long": ([300, 200, 400], [400, 700, 500]),
            "long, parts": ([130, 150], [2_000, 3_001]),
            "tiles of warps": ([30, 20, 40], [200, 150, 170]),
            "many": ([40] * n, [30] * n),
            "many, two tiles": ([90] * n, [20, 41, 64, 9, 33] * (n // 5)),
            "many, some longer": ([40] * n, [20, 100, 17, 70, 65] * (n // 5)),
            "many, wide": ([40] * n, [90, 130, 60, 128, 129] * (n // 5))}[name]


NAMES = ["few rows", "long", "long, parts", "tiles of warps", "many", "many, two tiles", "many, some longer", "many, wide"]
every = pytest.mark.parametrize("name", NAMES)
types = pytest.mark.parametrize("type_", sorted(TYPES))
dims = pytest.mark.parametrize("d", [64, 128])


def _both(layers, q, k, v, d_out, kw):
    out, lse = layers.attend(q, k, v, lse=True, **kw)
    return [out, lse, *layers.attend_grad(q, k, v, out, lse, d_out, **kw)]


def _equal(a, b):
    for x, y in zip(a, b):
        assert torch.equal(x, y)


@every
@types
@dims
def test_padding(layers, name, type_, d):
    q, k, v, d_out, kw = _args(*_lengths(name), 8, 4, d, TYPES[type_], seed=d, fused=True, padding=0.2)
    bad = kw["kv_ids"] < 0
    k[bad], v[bad] = 0, 0
    want = _both(layers, q, k, v, d_out, kw)
    assert all(bool(torch.isfinite(t).all()) for t in want[2:]) and not want[3][bad].any() and not want[4][bad].any()
    for in_k, in_v in ((NAN, INF), (INF, NAN), (-INF, NAN)):
        k[bad], v[bad] = in_k, in_v
        _equal(want, _both(layers, q, k, v, d_out, kw))


@every
@types
@dims
def test_a_sequence_of_padding_alone(layers, name, type_, d):
    q, k, v, d_out, kw = _args(*_lengths(name), 8, 4, d, TYPES[type_], seed=d, padding=0.1)
    (a, b), (c, e) = ((int(o[1]), int(o[2])) for o in (kw["q_offsets"], kw["kv_offsets"]))
    kw["kv_ids"][c:e] = -1
    want = _both(layers, q, k, v, d_out, kw)
    assert not want[0][a:b].any() and bool((want[1][a:b] == -INF).all()) and not want[2][a:b].any()
    assert not want[3][c:e].any() and not want[4][c:e].any()
    for value in (NAN, INF):
        q[a:b] = d_out[a:b] = value
        k[c:e] = v[c:e] = value
        _equal(want, _both(layers, q, k, v, d_out, kw))


@every
@types
@dims
def test_another_sequence(layers, name, type_, d):
    q, k, v, d_out, kw = _args(*_lengths(name), 8, 4, d, TYPES[type_], seed=d)
    (a, b), (c, e) = ((int(o[1]), int(o[2])) for o in (kw["q_offsets"], kw["kv_offsets"]))
    want = _both(layers, q, k, v, d_out, kw)
    for value in (NAN, INF):
        q[a:b] = k[c:e] = v[c:e] = d_out[a:b] = value
        got = _both(layers, q, k, v, d_out, kw)
        for new, old, lo, hi in zip(got, want, (a, a, a, c, c), (b, b, b, e, e)):
            assert torch.equal(new[:lo], old[:lo]) and torch.equal(new[hi:], old[hi:])
            assert not torch.isfinite(new[lo:hi]).all()


@every
@types
@dims
def test_equal_calls_give_equal_bits(layers, name, type_, d):
    args = _args(*_lengths(name), 8, 4, d, TYPES[type_], seed=d, padding=0.05)
    want = _both(layers, *args)
    for _ in range(3):
        _equal(want, _both(layers, *args))
