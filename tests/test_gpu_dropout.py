"""Dropout from counted random words: the words of every element against Philox in
Python's whole numbers, values against float64 (tests/tokens_util.py), refusals."""
import pytest

import tokens_util as ref
from layers_util import within

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def ifvs():
    from paper_2607_22922_gb300 import build
    build.build()
    from paper_2607_22922_gb300 import ifvs as mod
    return mod


@pytest.fixture(scope="module")
def layers(ifvs):
    L = ifvs.Layers()
    yield L
    L.close()


def _rand(n, dtype, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(n, generator=g, device="cuda").to(dtype)


@pytest.mark.parametrize("type_", sorted(TYPES))
@pytest.mark.parametrize("n", [1, 3, 4, 7, 8, 9, 511, 4096, 4099, 40_001])
def test_values(layers, type_, n):
    dt = TYPES[type_]
    for p, seed, step in ((0.1, 0, 0), (0.5, -1, 2**63 + 5), (0.0, 3, 1), (0.999, 2**40 + 1, 2**33)):
        x, r = _rand(n, dt, n), _rand(n, dt, n + 1)
        for residual in (None, r):
            within(layers.dropout(x, p, seed, step, residual=residual), *ref.dropout(x, p, seed, step, residual))


@pytest.mark.parametrize("type_", sorted(TYPES))
@pytest.mark.parametrize("shift", [1, 2, 4, 5])
def test_arrays_off_16_bytes(layers, type_, shift):
    dt, n = TYPES[type_], 3001
    x, r = _rand(n + 8, dt, 1)[shift:shift + n], _rand(n, dt, 2)
    within(layers.dropout(x, 0.3, 7, residual=r), *ref.dropout(x, 0.3, 7, 0, r))
    out = torch.full((n + 8,), 7.0, dtype=dt, device="cuda")
    layers.dropout(r, 0.3, 7, out=out[shift:shift + n])
    within(out[shift:shift + n], *ref.dropout(r, 0.3, 7, 0, None))
    assert bool((out[:shift] == 7).all()) and bool((out[shift + n:] == 7).all())


def test_the_gradient_is_the_same_call(layers):
    """d(sum dy out)/dx is dy / (1 - p) where x was kept: by differences of the call
    itself, which is linear, so that they are off by its rounding alone."""
    x, dy = _rand(999, torch.float32, 1), _rand(999, torch.float32, 2)
    dx = layers.dropout(dy, 0.4, 11, 5)
    one = layers.dropout(torch.ones_like(x), 0.4, 11, 5)
    assert torch.equal(dx != 0, one != 0)
    up, down = layers.dropout(x + 1, 0.4, 11, 5), layers.dropout(x - 1, 0.4, 11, 5)
    size = ((x.abs() + 1) / 0.6).double()
    within(((up - down) / 2 * dy).double(), dx.double(), 8 * 2.0 ** -24 * size * dy.abs().double())


def test_what_is_dropped_may_be_anything(layers):
    for dt in TYPES.values():
        x, r = torch.full((4096,), float("nan"), dtype=dt, device="cuda"), _rand(4096, dt, 3)
        x[::2] = float("inf")
        for residual in (None, r):
            out = layers.dropout(x, 0.5, 21, residual=residual)
            kept = (ref.words(0, 4096, 0, 21) >= 2**31).cuda()
            assert torch.equal(out[~kept], (torch.zeros_like(r) if residual is None else r)[~kept])
            assert not bool(torch.isfinite(out[kept]).any())


def test_shares_and_independence(layers):
    """Of n elements the share kept is 1 - p within six of its standard deviations,
    and so are the shares of pairs that two seeds, steps or neighbours keep together."""
    n = 1 << 22
    x = torch.ones(n, device="cuda")
    kept = lambda *a: layers.dropout(x, *a) != 0  # noqa: E731

    def near(flags, share):
        assert abs(float(flags.double().mean()) - share) < 6 * (share * (1 - share) / flags.numel()) ** 0.5

    for p in (0.1, 0.5, 0.9):
        a = kept(p, 1, 0)
        near(a, 1 - p)
        for b in (kept(p, 2, 0), kept(p, 1, 1), kept(p, 1 + 2**32, 0), kept(p, 1, 2**32)):
            near(a & b, (1 - p) ** 2)
        near(a[0::2] & a[1::2], (1 - p) ** 2)


def test_a_replayed_capture_reads_its_step(layers):
    x = _rand(3000, torch.float32, 4)
    step, out = torch.zeros(1, dtype=torch.int64, device="cuda"), torch.empty_like(x)
    s, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        layers.dropout(x, 0.5, 9, step, out=out, stream=s)
        step.add_(1)
    for i in (0, 1, 2):
        graph.replay()
        torch.cuda.synchronize()
        within(out, *ref.dropout(x, 0.5, 9, i, None))
    step.fill_(-3)
    graph.replay()
    torch.cuda.synchronize()
    within(out, *ref.dropout(x, 0.5, 9, 2**64 - 3, None))


def test_far_elements(layers):
    """Elements beyond 2^32: their words have the counter's high half."""
    n = 2**32 + 5000
    x = torch.ones(n, dtype=torch.float16, device="cuda")
    out = layers.dropout(x, 0.5, 13, 2)
    del x
    for first in (0, 2**31 - 100, 2**32 - 100, n - 2000):
        count = min(2000, n - first)
        kept = (ref.words(first, count, 2, 13) >= 2**31).cuda()
        assert torch.equal(out[first:first + count] != 0, kept)


def test_refusals(ifvs, layers):
    x = torch.ones(64, device="cuda")
    for p in (-0.1, 1.0, 1.5, float("nan")):
        with pytest.raises(ifvs.IfvsError) as e:
            layers.dropout(x, p, 1)
        assert e.value.code == ifvs.IFVS_ERR_ARG
    for bad in (dict(step=torch.zeros(1, dtype=torch.int32, device="cuda")), dict(step=torch.zeros(2, dtype=torch.int64, device="cuda")),
                dict(step=torch.zeros(1, dtype=torch.int64)), dict(residual=x[:63]), dict(residual=x.half()), dict(out=x[::2])):
        with pytest.raises(ValueError):
            layers.dropout(x, 0.5, 1, **bad)
    with pytest.raises(TypeError):
        layers.dropout(x.double(), 0.5, 1)
    lib, at = ifvs.lib(), x.data_ptr()
    for args in ((None, None, 64, 0, 0.5, 1, 1, None, at, None), (at, None, -1, 0, 0.5, 1, 1, None, at, None),
                 (at, None, 2**40 + 1, 0, 0.5, 1, 1, None, at, None), (at, None, 4, 3, 0.5, 1, 1, None, at, None),
                 (at + 2, None, 4, 0, 0.5, 1, 1, None, at, None), (at, at + 1, 4, 0, 0.5, 1, 1, None, at, None),
                 (at, None, 4, 0, 0.5, 1, 1, at + 4, at, None), (at, None, 4, 0, 0.5, 1, 1, None, None, None)):
        assert lib.ifvs_dropout(layers.h, *args) == ifvs.IFVS_ERR_ARG
    assert layers.dropout(x[:0], 0.5, 1).shape == (0,)
