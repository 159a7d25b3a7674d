"""Attention and its gradient on both sides of the rules that choose among their kernels:
many sequences with shared heads and several chunks of keys, a few rows with keys in parts
and in a warp's ring, rows beyond one tile among them."""
import pytest

from test_gpu_attend import TYPES, _args, _check, _ragged

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


@pytest.mark.parametrize("type_", sorted(TYPES))
@pytest.mark.parametrize("B,q,k,H,Hk,d", [
    (250, (0, 130), (0, 65), 8, 2, 64),
    (640, (0, 130), (0, 65), 4, 1, 64),
    (700, (1, 3), (1, 40), 64, 1, 40),
    (300, (40, 130), (50, 140), 8, 4, 64),        # chunks of 128 keys
    (500, (60, 70), (0, 200), 4, 4, 32),
    (700, (30, 60), (0, 66), 2, 2, 128),
])
def test_many_sequences(layers, type_, B, q, k, H, Hk, d):
    _check(layers, *_args(_ragged(B, *q, 1), _ragged(B, *k, 2), H, Hk, d, TYPES[type_], seed=B + d, fused=True, padding=0.04))


# keys of one chunk more than k_attend's, of a ring's turns, in parts; groups of 1 to 40
# heads; more rows than a tile in one sequence
@pytest.mark.parametrize("type_", sorted(TYPES))
@pytest.mark.parametrize("lq,lk,H,Hk,d", [
    ([1], [129], 2, 2, 64),
    ([1], [160], 1, 1, 8),
    ([1, 1, 1], [385, 1, 700], 4, 4, 32),
    ([2, 0, 1], [257, 300, 0], 8, 1, 72),
    ([1] * 5, [1_023, 1_024, 1_025, 31, 33], 16, 1, 128),
    ([1] * 40, [300, 0, 290, 600, 1] * 8, 8, 8, 64),
    ([60] + [0] * 9, [500] * 10, 2, 2, 64),
    ([3, 1], [2_050, 4_111], 10, 2, 40),
    ([1], [20_011], 40, 8, 128),
])
def test_a_few_rows(layers, type_, lq, lk, H, Hk, d):
    for padding in (0.0, 0.3):
        _check(layers, *_args(lq, lk, H, Hk, d, TYPES[type_], seed=d, fused=True, padding=padding))


def test_a_few_rows_far_scores(layers):
    """One key far above the others in each of the warps' chunks; a part whose keys are all
    padding."""
    for at in (0, 40, 70, 100, 1_500, 2_999):
        q, k, v, d_out, kw = _args([1], [3_000], 1, 1, 64, torch.bfloat16, seed=2)
        q.fill_(1.0)
        k[at] = 100.0
        assert torch.equal(layers.attend(q, k, v, **kw)[0], v[at].expand_as(q))
    q, k, v, d_out, kw = _args([1, 1], [3_000, 2_900], 4, 2, 64, torch.float16, seed=6, padding=0.02)
    kw["kv_ids"][700:3_000] = -1
    _check(layers, q, k, v, d_out, kw)
