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


# ---- the steady state: sizes at which every team, warp and CTA has work for many
# rounds of its ring, by the launch rules (asserted here for the device at hand)

def _sms():
    return torch.cuda.get_device_properties(0).multi_processor_count


def _places(T, D, type_, teams):
    """Places of its ring that a team fills."""
    row = D * TYPES[type_].itemsize
    per = 1 if row >= 1024 else (8 if row <= 128 else 1024 // row)
    return -(-T // teams) // per


def _cuts(T, B, seed):
    """Offsets of B sequences: empty ones, single tokens, one of a third of all tokens."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    cuts = torch.randint(T // 3, T + 1, (B + 1,), generator=g, device="cuda").sort().values
    cuts[1:7] = torch.tensor([0, 1, 2, 2, T // 3 - 1, T // 3], device="cuda")
    cuts[0], cuts[B] = 0, T
    return cuts


@pytest.mark.parametrize("type_", sorted(TYPES))
@pytest.mark.parametrize("T,D", [(160_003, 40), (140_001, 97), (60_001, 320), (40_003, 1030), (9_001, 5001)])
def test_norm_join_in_its_steady_state(layers, type_, T, D):
    warps = 1
    while warps * (512 if D <= 4096 else 1024) < D:
        warps *= 2
    assert _places(T, D, type_, 3 * 8 // warps * _sms()) >= 4
    r, dt, off = _rand(D), TYPES[type_], _cuts(T, 1500, D)
    x, y, dxo, dn = ((s * r(T, D)).to(dt) for s in (1.5, 0.5, 1.0, 1.0))
    a = (x, y, (1 + 0.3 * r(1500, D)).to(dt), (1 + 0.1 * r(D)).to(dt), (1 + 0.1 * r(D)).to(dt))
    kw = dict(offsets=off, res_scale=0.7, eps=EPS)
    _check(layers.norm_join(*a, **kw), ref.norm_join(*a, off, 0.7, EPS))
    _check(layers.norm_join_grad(*a, dxo, dn, **kw), ref.norm_join_grad(*a, dxo, dn, off, 0.7, EPS))


@pytest.mark.parametrize("T,D,V,type_", [(400_003, 40, 3_000, "bf16"), (700_001, 64, 50_000, "f32"), (400_003, 520, 9_000, "bf16"),
                                         (700_001, 33, 500, "f16"), (300_007, 260, 2, "f32"), (400_003, 300, 70_000, "f16")])
def test_embed_grad_in_its_steady_state(layers, T, D, V, type_):
    """Parts of more than 32 tokens of the sorted order, aligned rows and others."""
    assert T // 64 >= 16 * _sms()
    g = torch.Generator(device="cuda")
    g.manual_seed(T + D)
    ids = torch.randint(0, V, (T,), generator=g, device="cuda")
    ids = torch.where(torch.rand(T, generator=g, device="cuda") < 0.5, ids % min(V, 12), ids)
    ids[torch.rand(T, generator=g, device="cuda") < 0.03] = -1
    ids = ids.int()
    d_out = _rand(D)(T, D).to(TYPES[type_])
    ref.within(layers.embed_grad(d_out, ids, 1.5, V=V), *ref.embed_grad(d_out, ids, 1.5, V))


def _pairs(rows, cols, K):
    return -(-rows // 256) * -(-cols // 256) >= _sms() // (4 if K >= 1024 else 2)


# tokens, width, hidden width, whether the output product and the gradient's products
# go to pairs of CTAs on the measured device; several tiles of both operands each
@pytest.mark.parametrize("T,D,F,out,grad", [(5_003, 520, 1032, True, True), (9_001, 264, 776, False, True),
                                            (10_001, 264, 776, True, True), (1_100, 776, 1288, False, True),
                                            (300, 520, 1032, False, False), (2_500, 1544, 2056, True, True)])
@pytest.mark.parametrize("act,type_", [("silu", "bf16"), ("gelu", "f16")])
def test_ffn_of_several_tiles(layers, T, D, F, out, grad, act, type_):
    if _sms() == 152:
        assert _pairs(T, D, F) == out
        assert (T > 512 and (_pairs(T, D, 2 * F) or _pairs(2 * F, D, T))) == grad
    r, dt = _rand(T + D), TYPES[type_]
    x, dy = r(T, D).to(dt), r(T, D).to(dt)
    w_in, w_out = (r(2 * F, D) / D ** 0.5).to(dt), (r(D, F) / F ** 0.5).to(dt)
    ref.within(layers.ffn(x, w_in, w_out, act=act), *ref.ffn(x, w_in, w_out, act))
    _check(layers.ffn_grad(x, w_in, w_out, dy, act=act), ref.ffn_grad(x, w_in, w_out, dy, act))


@pytest.mark.parametrize("T,D,F", [(3, 8192, 72), (130, 8192, 64), (3, 64, 65536), (130, 64, 65536), (1, 8192, 8192), (130, 8192, 8192)])
def test_ffn_of_the_largest_widths(layers, T, D, F):
    r, dt = _rand(T + D), torch.bfloat16
    x, dy = r(T, D).to(dt), r(T, D).to(dt)
    w_in, w_out = (r(2 * F, D) / D ** 0.5).to(dt), (r(D, F) / F ** 0.5).to(dt)
    ref.within(layers.ffn(x, w_in, w_out), *ref.ffn(x, w_in, w_out, "silu"))
    _check(layers.ffn_grad(x, w_in, w_out, dy), ref.ffn_grad(x, w_in, w_out, dy, "silu"))
