"""The encoder's layers at the limits of their ranges and in their steady state,
against float64 with the bounds of tests/layers_util.py."""
import pytest

import layers_util as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
EPS = 1e-5


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


def _rand(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return lambda *shape: torch.randn(*shape, generator=g, device="cuda")


def _check(got, want):
    for a, w in zip(got, want):
        assert (a is None) == (w is None)
        if a is not None:
            ref.within(a, *w)


def test_norm_join_of_as_many_tokens_as_there_can_be(layers):
    """T = 2^31 - 1: the last places of the rings end at the largest int.  A
    token's outputs depend on its row and its sequence's gate alone, so the
    first, some middle and the last tokens are compared."""
    T, D, dt = 2**31 - 1, 1, torch.float16
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB of device memory")
    g = torch.Generator(device="cuda")
    g.manual_seed(31)

    def rows():
        return torch.empty(T, D, dtype=dt, device="cuda").normal_(generator=g)

    x, y, dxo, dn = rows(), rows(), rows(), rows()
    cut = T - 21
    off = torch.tensor([0, cut, T], dtype=torch.int64, device="cuda")
    gate = torch.tensor([[0.5], [-1.5]], dtype=dt, device="cuda")
    w_post, w_pre = torch.full((1,), 1.25, dtype=dt, device="cuda"), torch.full((1,), 0.75, dtype=dt, device="cuda")
    kw = dict(offsets=off, res_scale=0.7, eps=EPS)
    xo, no = layers.norm_join(x, y, gate, w_post, w_pre, **kw)
    dx, dy, _, _, _ = layers.norm_join_grad(x, y, gate, w_post, w_pre, dxo, dn, **kw)
    for lo, hi in ((0, 100), (T // 2, T // 2 + 100), (T - 100, T)):
        s = slice(lo, hi)
        here = torch.tensor([0, min(max(cut - lo, 0), hi - lo), hi - lo], dtype=torch.int64, device="cuda")
        a = (x[s], y[s], gate, w_post, w_pre)
        _check((xo[s], no[s]), ref.norm_join(*a, here, 0.7, EPS))
        _check((dx[s], dy[s]), ref.norm_join_grad(*a, dxo[s], dn[s], here, 0.7, EPS)[:2])


@pytest.mark.parametrize("act", ["silu", "gelu", "relu"])
@pytest.mark.parametrize("T", [1, 4, 7, 200])
def test_ffn_passes_a_nan_gate_on(layers, act, T):
    """A NaN weight of one gate column reaches every output that the column's hidden
    values do: all of y and dx, its own rows of d_w_in and column of d_w_out."""
    D, F, bad = 64, 72, 5
    r = _rand(T)
    x, dy, w_in, w_out = (r(*s).bfloat16() for s in ((T, D), (T, D), (2 * F, D), (D, F)))
    w_in[bad, 3] = float("nan")
    assert layers.ffn(x, w_in, w_out, act=act).isnan().all()
    dx, d_w_in, d_w_out = layers.ffn_grad(x, w_in, w_out, dy, act=act)
    assert dx.isnan().all()
    rows, cols = d_w_in.isnan().all(1), d_w_out.isnan().all(0)
    assert rows[bad] and rows[F + bad] and cols[bad]
    others = [i for i in range(F) if i != bad]
    assert not d_w_in[others].isnan().any() and not d_w_in[F:][others].isnan().any() and not d_w_out[:, others].isnan().any()


@pytest.mark.parametrize("eps", [1e-12, 1e-30, 1e-37])
@pytest.mark.parametrize("type_", ["f32", "bf16"])
def test_norm_join_rows_of_zeros_with_a_small_eps(layers, type_, eps):
    """1 / rms of such a row is eps^(-1/2), whose powers leave float32."""
    r, dt = _rand(9), TYPES[type_]
    T, D = 24, 72
    off = torch.tensor([0, 10, 24], dtype=torch.int64, device="cuda")
    x, y, dxo, dn = (r(T, D).to(dt) for _ in range(4))
    x[3:9], y[5:12] = 0, 0
    dn *= 2.0 ** -30                    # times 1 / rms within the types' range
    dxo *= 2.0 ** -30
    a = (x, y, (1 + 0.3 * r(2, D)).to(dt), (1 + 0.1 * r(D)).to(dt), (1 + 0.1 * r(D)).to(dt))
    kw = dict(offsets=off, res_scale=0.7, eps=eps)
    _check(layers.norm_join(*a, **kw), ref.norm_join(*a, off, 0.7, eps))
    _check(layers.norm_join_grad(*a, dxo, dn, **kw), ref.norm_join_grad(*a, dxo, dn, off, 0.7, eps))
