"""GELU of the linear layer where it is small: a value far below zero keeps its leading
digits, and a token's row is the same whichever of the layer's kernels makes it.

The inputs make x w^T one exact product, so that the activation alone is off.  Its terms,
for -13 <= z <= 0, with U = 2^-24: the exponent z^2 / 2 log2(e), at most 122, is rounded
three times, the constant among them (122 ln(2) 3 U < 1.6e-5 of the exponential); the
polynomial is within 1.2e-5 of the tail's own value; the exponential, the reciprocal and ten
operations are within 20 U (1.2e-6).  In all below 3e-5 < 2^-15 of each term."""
import math

import pytest

from layers_util import rounded, within

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
REL = 2.0 ** -15


@pytest.fixture(scope="module")
def layers():
    from paper_2607_22922_gb300 import build
    build.build()
    from paper_2607_22922_gb300 import ifvs
    L = ifvs.Layers()
    yield L
    L.close()


def _inputs(T, D_in, D_out, dtype):
    """Row t is z[t] in its first place, weights pick it out"""
    z = torch.linspace(-13, 0, T, device="cuda").to(dtype)
    if T < 5:
        z = torch.tensor([-5.5, -4.25, -6.5, -12.0], device="cuda")[:T].to(dtype)
    x, w = torch.zeros(T, D_in, dtype=dtype, device="cuda"), torch.zeros(D_out, D_in, dtype=dtype, device="cuda")
    x[:, 0], w[:, 0] = z, 1
    return z.double(), x, w


def _phi(z):
    return torch.erfc(-z / math.sqrt(2)) / 2


# a few tokens; single CTAs, pairs, sums in parts
SIZES = [(1, 8, 8), (4, 1000, 72), (5, 8, 8), (300, 64, 136), (130, 8192, 64), (5_000, 72, 2560)]


@pytest.mark.parametrize("type_", sorted(TYPES))
@pytest.mark.parametrize("size", SIZES)
def test_gelu(layers, type_, size):
    z, x, w = _inputs(*size, TYPES[type_])
    want = (z * _phi(z))[:, None].expand(-1, size[2])
    within(layers.linear(x, w, act="gelu"), want, rounded(want, REL * want.abs(), TYPES[type_]))


@pytest.mark.parametrize("type_", sorted(TYPES))
@pytest.mark.parametrize("size", SIZES)
def test_gelu_slope(layers, type_, size):
    """dx's first column is the slope alone where one output has a weight."""
    z, x, w = _inputs(*size, TYPES[type_])
    w[1:] = 0
    dx, _, _ = layers.linear_grad(x, w, torch.ones(size[0], size[2], dtype=TYPES[type_], device="cuda"), act="gelu")
    density = z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    want, dt = _phi(z) + density, TYPES[type_]
    # dz is rounded to the type, then dx, which it equals
    within(dx[:, 0], want, rounded(want, rounded(want, REL * (_phi(z) + density.abs()), dt) - rounded(want, 0 * want, dt), dt))


@pytest.mark.parametrize("type_", sorted(TYPES))
def test_a_row_is_the_same_with_more_tokens(layers, type_):
    z, x, w = _inputs(400, 64, 72, TYPES[type_])
    whole = layers.linear(x, w, act="gelu")
    for t in range(0, 400, 4):
        assert torch.equal(layers.linear(x[t:t + 4], w, act="gelu"), whole[t:t + 4])


def test_far_values(layers):
    """Infinities as g Phi(g) has them: infinity above, no number below (infinity times 0)."""
    for T in (4, 300):
        x = torch.zeros(T, 8, dtype=torch.bfloat16, device="cuda")
        w = torch.zeros(8, 8, dtype=torch.bfloat16, device="cuda")
        w[:, 0] = 1
        x[:4, 0] = torch.tensor([float("inf"), -float("inf"), 300.0, -300.0])
        y = layers.linear(x, w, act="gelu")
        assert bool((y[0] == float("inf")).all()) and bool(torch.isnan(y[1]).all())
        assert bool((y[2] == 300).all()) and not y[3].any()
