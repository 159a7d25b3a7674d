"""The linear layer and its gradient against their definitions in float64, at the
sizes where they can go wrong, and their refusals.  Every tolerance is the bound that
tests/tokens_util.py derives for that element."""
import ctypes

import pytest

import tokens_util as ref
from layers_util import within

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
ACTS = ["none", "silu", "gelu", "relu"]


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


def _args(T, D_in, D_out, dtype, seed=None):
    g = torch.Generator(device="cuda")
    g.manual_seed(T * 7 + D_in + D_out if seed is None else seed)
    r = lambda *n: torch.randn(*n, generator=g, device="cuda")  # noqa: E731
    return dict(x=r(T, D_in).to(dtype), w=(r(D_out, D_in) / D_in ** 0.5).to(dtype), bias=r(D_out).to(dtype),
                residual=r(T, D_out).to(dtype), dy=r(T, D_out).to(dtype))


# a few tokens; one tile and ragged ones; sums in parts; pairs of CTAs; several tiles per CTA
SIZES = [(1, 8, 8), (2, 64, 24), (3, 1000, 136), (4, 960, 960), (5, 64, 72), (127, 136, 264), (129, 960, 392), (300, 8, 2056),
         (1000, 4096, 136), (130, 4104, 64), (3001, 72, 1032), (5000, 512, 2560), (20_001, 64, 200)]


@pytest.mark.parametrize("type_", sorted(TYPES))
@pytest.mark.parametrize("size", SIZES)
def test_linear(layers, type_, size):
    a = _args(*size, TYPES[type_])
    for act in ACTS:
        for bias, residual in ((a["bias"], a["residual"]), (None, a["residual"]), (a["bias"], None), (None, None)):
            within(layers.linear(a["x"], a["w"], bias, act=act, residual=residual), *ref.linear(a["x"], a["w"], bias, act, residual))


@pytest.mark.parametrize("type_", sorted(TYPES))
@pytest.mark.parametrize("size", SIZES)
def test_linear_grad(layers, type_, size):
    a = _args(*size, TYPES[type_])
    for act in ACTS:
        for bias in (a["bias"], None):
            got = layers.linear_grad(a["x"], a["w"], a["dy"], bias, act=act)
            want = ref.linear_grad(a["x"], a["w"], a["dy"], bias, act)
            assert (got[2] is None) == (bias is None)
            for p, q in zip(got, want):
                within(p, *q)


@pytest.mark.parametrize("act", ACTS)
def test_gradient_against_differences(layers, act):
    """The loss sum(dy y) along a random direction of every input, in float64 from the
    layer's own definition, against the gradients' sums.  The gradients are off by at
    most their bounds, the central difference by its third-order term (h = 2^-8, third
    derivatives of the activations below 2 and of the product's entries' size) -- for
    ReLU the entries within h of its bend, whose slope it mistakes."""
    a = _args(65, 40, 72, torch.float16)
    g = torch.Generator(device="cuda")
    g.manual_seed(9)
    got = layers.linear_grad(a["x"], a["w"], a["dy"], a["bias"], act=act)
    want = ref.linear_grad(a["x"], a["w"], a["dy"], a["bias"], act)
    p = {k: a[k].double() for k in ("x", "w", "bias", "dy")}
    f = lambda x, w, b: (p["dy"] * ref._act(act, x @ w.t() + b)[0]).sum()  # noqa: E731
    h = 2.0 ** -8
    for i, name in enumerate(("x", "w", "bias")):
        d = torch.randn(p[name].shape, generator=g, device="cuda", dtype=torch.float64)
        at = [{**p, name: p[name] + s * d} for s in (h, -h)]
        difference = (f(at[0]["x"], at[0]["w"], at[0]["bias"]) - f(at[1]["x"], at[1]["w"], at[1]["bias"])) / (2 * h)
        z = p["x"] @ p["w"].t() + p["bias"]
        dz = d @ p["w"].t() if name == "x" else p["x"] @ d.t() if name == "w" else d.expand_as(z)
        third = 2 * h * h / 6 * (p["dy"].abs() * dz.abs() ** 3).sum()
        if act == "relu":
            third = (p["dy"].abs() * dz.abs() * (z.abs() <= h * dz.abs())).sum()
        allowed = (want[i][1] * d.abs()).sum() + third + 1e-9
        assert abs(float((got[i].double() * d).sum() - difference)) <= float(allowed)


def test_no_tokens(layers):
    x, w = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda"), torch.ones(24, 64, dtype=torch.bfloat16, device="cuda")
    assert layers.linear(x, w).shape == (0, 24)
    d_w, d_bias = torch.full_like(w, 7), torch.full((24,), 7.0, dtype=torch.bfloat16, device="cuda")
    layers.linear_grad(x, w, torch.empty(0, 24, dtype=torch.bfloat16, device="cuda"), w[:, 0].contiguous(), act="gelu", d_w=d_w,
                       d_bias=d_bias)
    assert not d_w.any() and not d_bias.any()


@pytest.mark.parametrize("T", [3, 200])
def test_rows_beside_the_output_are_left(layers, T):
    """Tiles are wider and higher than the output."""
    a = _args(T, 72, 72, torch.bfloat16)
    y = torch.full((T + 2, 72), 7.0, dtype=torch.bfloat16, device="cuda")
    layers.linear(a["x"], a["w"], a["bias"], act="silu", y=y[1:T + 1])
    assert bool((y[0] == 7).all()) and bool((y[-1] == 7).all())
    d = [torch.full((n + 2, 72), 7.0, dtype=torch.bfloat16, device="cuda") for n in (T, 72)]
    layers.linear_grad(a["x"], a["w"], a["dy"], act="silu", dx=d[0][1:-1], d_w=d[1][1:-1])
    for t in d:
        assert bool((t[0] == 7).all()) and bool((t[-1] == 7).all())


def test_values_that_are_not_finite(layers):
    """They stay in their rows: every token's row is its own sum."""
    for T in (3, 300):
        a = _args(T, 64, 72, torch.bfloat16)
        a["x"][1, 5], a["x"][2, 0] = float("nan"), float("inf")
        for act in ACTS:
            y = layers.linear(a["x"], a["w"], a["bias"], act=act)
            assert bool(torch.isnan(y[1]).all()) and not bool(torch.isfinite(y[2]).all())
            assert bool(torch.isfinite(y[0]).all()) and bool(torch.isfinite(y[3:]).all())


@pytest.mark.parametrize("size", [(2, 256, 72), (130, 4104, 64), (3001, 72, 1032)])
def test_equal_calls_give_equal_bits(layers, size):
    a = _args(*size, torch.bfloat16)
    y = layers.linear(a["x"], a["w"], a["bias"], act="gelu", residual=a["residual"])
    d = layers.linear_grad(a["x"], a["w"], a["dy"], a["bias"], act="gelu")
    for _ in range(3):
        assert torch.equal(y, layers.linear(a["x"], a["w"], a["bias"], act="gelu", residual=a["residual"]))
        for p, q in zip(d, layers.linear_grad(a["x"], a["w"], a["dy"], a["bias"], act="gelu")):
            assert torch.equal(p, q)


def test_refusals(ifvs, layers):
    a = _args(6, 64, 72, torch.bfloat16)
    x, w, b, dy = a["x"], a["w"], a["bias"], a["dy"]

    def code(*args, f=layers.linear, **kw):
        with pytest.raises(ifvs.IfvsError) as e:
            f(*args, **kw)
        return e.value.code

    assert code(x.float(), w.float()) == ifvs.IFVS_ERR_UNSUPPORTED
    assert code(x[:, :60].contiguous(), w[:, :60].contiguous()) == ifvs.IFVS_ERR_UNSUPPORTED
    assert code(x, w[:70]) == ifvs.IFVS_ERR_UNSUPPORTED
    shifted = torch.empty(6 * 64 + 1, dtype=torch.bfloat16, device="cuda")[1:].view(6, 64)
    assert code(shifted, w) == ifvs.IFVS_ERR_ARG
    for bad in (dict(act="tanh"), dict(bias=b[:64]), dict(residual=a["residual"][:, :64]), dict(y=torch.empty_like(x)),
                dict(residual=a["residual"].t().contiguous().t())):
        with pytest.raises(ValueError):
            layers.linear(x, w, **bad)
    with pytest.raises(ValueError):
        layers.linear(x, w.half())
    with pytest.raises(ValueError):
        layers.linear_grad(x, w, dy[:5])
    with pytest.raises(ifvs.IfvsError):
        layers.linear_grad(x, w, dy, d_bias=torch.empty_like(b))
    for field, value in (("act", 4), ("T", -1), ("T", 2**31), ("D_in", 0), ("D_out", 65_544), ("type", 3), ("w", None)):
        p = ifvs.LinearParams(6, 64, 72, ifvs.IFVS_T_BF16, 0, w.data_ptr(), None, None)
        setattr(p, field, value)
        assert ifvs.lib().ifvs_linear(layers.h, ctypes.byref(p), x.data_ptr(), None, dy.data_ptr()) == ifvs.IFVS_ERR_ARG


def test_widest(layers):
    """65 536 columns in, and out."""
    for D_in, D_out in ((65_536, 16), (16, 65_536)):
        a = _args(33, D_in, D_out, torch.bfloat16)
        within(layers.linear(a["x"], a["w"], a["bias"], act="silu"), *ref.linear(a["x"], a["w"], a["bias"], "silu", None))
        for p, q in zip(layers.linear_grad(a["x"], a["w"], a["dy"], a["bias"], act="silu"),
                        ref.linear_grad(a["x"], a["w"], a["dy"], a["bias"], "silu")):
            within(p, *q)
