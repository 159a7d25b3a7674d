"""Attention of packed sequences and its gradient against their definitions in float64,
at the lengths, heads, masks and layouts where they can go wrong, and their refusals.
Every tolerance is the bound that tests/tokens_util.py derives for that element."""
import ctypes

import pytest

import tokens_util as ref
from layers_util import within

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}


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


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _offsets(lengths):
    return torch.tensor([0] + lengths, dtype=torch.int64, device="cuda").cumsum(0)


def _args(lq, lk, H, Hk, d, dtype, seed=1, fused=False, padding=0.0):
    """Packed inputs of sequences of these lengths."""
    g = _gen(seed)
    r = lambda *n: torch.randn(*n, generator=g, device="cuda").to(dtype)  # noqa: E731
    Tq, Tk = sum(lq), sum(lk)
    kv = r(Tk, 2, Hk, d)
    k, v = (kv[:, 0], kv[:, 1]) if fused else (kv[:, 0].contiguous(), kv[:, 1].contiguous())
    kw = dict(q_offsets=_offsets(lq), kv_offsets=_offsets(lk))
    if padding:
        kw["kv_ids"] = torch.where(torch.rand(Tk, generator=g, device="cuda") < padding, -1, 5).int()
    return r(Tq, H, d), k, v, r(Tq, H, d), kw


def _reference_kw(kw):
    return dict(q_offsets=kw.get("q_offsets"), kv_offsets=kw.get("kv_offsets"), ids=kw.get("kv_ids"), scale=kw.get("scale"))


def _lse_within(got, want):
    value, bound = want
    assert torch.equal(torch.isinf(got), torch.isinf(value))
    there = torch.isfinite(value)
    within(got[there], value[there], bound[there])


def _check(layers, q, k, v, d_out, kw):
    want = _reference_kw(kw)
    out, lse = layers.attend(q, k, v, lse=True, **kw)
    (o, l), grads = ref.attend(q, k, v, **want), ref.attend_grad(q, k, v, d_out, **want)
    within(out, *o)
    _lse_within(lse, l)
    for got, w in zip(layers.attend_grad(q, k, v, out, lse, d_out, **kw), grads):
        within(got, *w)
    return out, lse


LENGTHS = {
    "one": ([1], [1]),
    "token": ([1], [17]),
    "tiles": ([64, 63, 65, 1, 128], [64, 65, 63, 1, 128]),
    "empty": ([5, 0, 7, 3, 0, 2], [9, 4, 0, 1, 0, 0]),
    "short": ([17, 3, 120, 16, 15, 1], [5, 65, 33, 16, 17, 130]),
    "long": ([300, 1, 129], [700, 513, 2]),
    "many": ([3] * 700, [0, 1, 2, 17, 5] * 140),
}


@pytest.mark.parametrize("type_", sorted(TYPES))
@pytest.mark.parametrize("d", [8, 32, 40, 64, 72, 128])
@pytest.mark.parametrize("name", sorted(LENGTHS))
def test_lengths(layers, type_, d, name):
    lq, lk = LENGTHS[name]
    _check(layers, *_args(lq, lk, 2, 2, d, TYPES[type_], seed=d))


@pytest.mark.parametrize("type_", sorted(TYPES))
@pytest.mark.parametrize("H,Hk", [(1, 1), (4, 1), (6, 2), (8, 4), (40, 1), (65, 1)])
def test_heads_that_share_keys(layers, type_, H, Hk):
    for lq, lk in (([1, 30], [40, 3]), ([64, 0, 5], [90, 7, 130])):
        _check(layers, *_args(lq, lk, H, Hk, 24, TYPES[type_], seed=H))


@pytest.mark.parametrize("type_", sorted(TYPES))
@pytest.mark.parametrize("fused", [False, True])
def test_padding(layers, type_, fused):
    """Keys of padding may hold anything; a sequence may be padding alone."""
    for share in (0.1, 0.9):
        q, k, v, d_out, kw = _args([20, 70, 9, 33], [64, 130, 11, 65], 4, 2, 64, TYPES[type_], seed=3, fused=fused, padding=share)
        kw["kv_ids"][194:205] = -7          # the third sequence
        bad = kw["kv_ids"] < 0
        want = _check(layers, q, k, v, d_out, kw)
        k[bad], v[bad] = float("nan"), float("inf")
        got = layers.attend(q, k, v, lse=True, **kw)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        assert not got[0][90:99].any() and bool((got[1][90:99] == -float("inf")).all())
        k[bad], v[bad] = 0, 0
        clean = layers.attend_grad(q, k, v, *want, d_out, **kw)
        k[bad], v[bad] = float("inf"), float("nan")
        for a, b in zip(clean, layers.attend_grad(q, k, v, *want, d_out, **kw)):
            assert torch.equal(a, b)
        assert not clean[1][bad].any() and not clean[2][bad].any() and not clean[0][90:99].any()


@pytest.mark.parametrize("lengths", [([30, 31, 33], [40, 41, 43]), ([100, 131, 133], [140, 241, 143]), ([200, 331, 133], [340, 541, 243]),
                                     ([60] * 180, [30] * 180)])
def test_sequences_do_not_see_each_other(layers, lengths):
    """Values that are not finite in one sequence stay there."""
    q, k, v, d_out, kw = _args(*lengths, 4, 2, 64, torch.bfloat16, seed=5)
    want = layers.attend(q, k, v, lse=True, **kw)
    grads = layers.attend_grad(q, k, v, *want, d_out, **kw)
    (a, b), (c, d) = ((o[1].item(), o[2].item()) for o in (kw["q_offsets"], kw["kv_offsets"]))
    for t, lo, hi in ((q, a, b), (k, c, d), (v, c, d), (d_out, a, b)):
        t[lo:hi] = float("nan")
    out, lse = layers.attend(q, k, v, lse=True, **kw)
    assert bool(torch.isnan(out[a:b]).all())
    got = layers.attend_grad(q, k, v, out, lse, d_out, **kw)
    for new, old, lo, hi in ((out, want[0], a, b), (lse, want[1], a, b), (got[0], grads[0], a, b), (got[1], grads[1], c, d),
                             (got[2], grads[2], c, d)):
        assert torch.equal(new[:lo], old[:lo]) and torch.equal(new[hi:], old[hi:])


@pytest.mark.parametrize("type_", sorted(TYPES))
def test_rows_with_gaps(layers, type_):
    """Queries, keys, values, outputs and gradients inside wider rows; what lies between
    them is left."""
    dt, T, H, d = TYPES[type_], 77, 2, 40
    g = _gen(8)
    x = torch.randn(T, 5, H, d, generator=g, device="cuda").to(dt)
    q, k, v, d_out = (x[:, i] for i in range(4))
    off = _offsets([7, 70])
    kw = dict(q_offsets=off, kv_offsets=off)
    y = torch.full((T, 7, H, d), 7.0, dtype=dt, device="cuda")
    out, lse = layers.attend(q, k, v, out=y[:, 1], lse=True, **kw)
    assert out.data_ptr() == y[:, 1].data_ptr()
    want = _reference_kw(kw)
    within(out, *ref.attend(q, k, v, **want)[0])
    layers.attend_grad(q, k, v, out, lse, d_out, dq=y[:, 2], dk=y[:, 3], dv=y[:, 5], **kw)
    for i, w in zip((2, 3, 5), ref.attend_grad(q, k, v, d_out, **want)):
        within(y[:, i], *w)
    for i in (0, 4, 6):
        assert bool((y[:, i] == 7).all())


@pytest.mark.parametrize("type_", sorted(TYPES))
@pytest.mark.parametrize("lq,lk,H,Hk,d", [
    ([1], [9_000], 2, 2, 64),                       # one query, its keys in parts
    ([1, 1, 1], [5_001, 40, 3_333], 4, 1, 128),
    ([2, 0, 3], [2_000, 0, 2_001], 2, 2, 32),
    ([3_001], [65], 2, 2, 64),                      # a few keys, the rows in parts
    ([2_000], [17], 8, 1, 40),
    ([1_100, 900], [1_300, 1_000], 2, 1, 128),
    ([700, 60], [2_049, 1_024], 4, 4, 64),
])
def test_long(layers, type_, lq, lk, H, Hk, d):
    _check(layers, *_args(lq, lk, H, Hk, d, TYPES[type_], seed=d + H, padding=0.05))


def _ragged(n, low, high, seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return torch.randint(low, high + 1, (n,), generator=g).tolist()


# many sequences: some without queries or keys, keys of one chunk and of several, groups
# that fill a tile of 128 rows, or do not divide it
@pytest.mark.parametrize("type_", sorted(TYPES))
@pytest.mark.parametrize("B,q,k,H,Hk,d", [
    (160, (0, 130), (0, 65), 4, 1, 64),
    (200, (20, 60), (0, 17), 8, 8, 40),
    (150, (30, 90), (50, 140), 4, 2, 128),
    (120, (60, 70), (40, 300), 6, 2, 72),
    (300, (1, 3), (1, 40), 64, 1, 64),
    (170, (120, 120), (16, 16), 8, 2, 8),
    (418, (64, 64), (20, 20), 8, 8, 64),      # units of a CTA: one more than are found together, in the forward pass
    (500, (32, 40), (16, 16), 8, 8, 64),      # and in the gradient
    (900, (0, 90), (0, 9), 1, 1, 16),
])
def test_many_sequences(layers, type_, B, q, k, H, Hk, d):
    _check(layers, *_args(_ragged(B, *q, 1), _ragged(B, *k, 2), H, Hk, d, TYPES[type_], seed=B, fused=True, padding=0.04))


def test_no_offsets_is_one_sequence(layers):
    q, k, v, d_out, kw = _args([70], [90], 2, 2, 64, torch.bfloat16)
    want = layers.attend(q, k, v, lse=True, **kw)
    got = layers.attend(q, k, v, lse=True)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    for a, b in zip(layers.attend_grad(q, k, v, *want, d_out), layers.attend_grad(q, k, v, *want, d_out, **kw)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("scale", [1e-3, 1.0, 30.0])
def test_scales(layers, scale):
    """Nearly even weights, and weights that one key takes alone."""
    q, k, v, d_out, kw = _args([40, 130], [33, 200], 2, 2, 64, torch.bfloat16, seed=11)
    _check(layers, q, k, v, d_out, dict(kw, scale=scale))


def test_one_key_takes_all(layers):
    """A score far above the others, in the first and in the last tile: the others' weights
    vanish without a NaN, and one key's output is its value."""
    for at in (0, 150):
        q, k, v, d_out, kw = _args([70], [200], 1, 1, 64, torch.bfloat16, seed=2)
        q.fill_(1.0)
        k[at] = 100.0
        out, lse = layers.attend(q, k, v, lse=True, **kw)
        assert torch.equal(out, v[at].expand_as(out))
        dq, dk, dv = layers.attend_grad(q, k, v, out, lse, d_out, **kw)
        assert bool(torch.isfinite(dq).all() and torch.isfinite(dk).all() and torch.isfinite(dv).all())


def test_nothing_to_do(layers):
    bf = torch.bfloat16
    some, none = torch.ones(6, 2, 16, dtype=bf, device="cuda"), torch.empty(0, 2, 16, dtype=bf, device="cuda")
    out, lse = layers.attend(none, some, some, lse=True)
    assert out.shape == (0, 2, 16) and lse.shape == (0, 2)
    for g in layers.attend_grad(none, some, some, out, lse, none)[1:]:
        assert not g.any()
    out, lse = layers.attend(some, none, none, lse=True, out=torch.full_like(some, 7))
    assert not out.any() and bool((lse == -float("inf")).all())
    dq, dk, dv = layers.attend_grad(some, none, none, out, lse, some, dq=torch.full_like(some, 7))
    assert not dq.any() and dk.shape == (0, 2, 16)
    off = torch.zeros(9, dtype=torch.int64, device="cuda")
    assert layers.attend(none, none, none, q_offsets=off, kv_offsets=off)[0].shape == (0, 2, 16)


def test_gradient_against_differences(layers):
    """sum(d_out out) along a random direction of q, k and v, by central differences of
    the definition in float64 (h = 2^-8: off by h^2 times third derivatives, which scores
    of deviation 1 keep below 100 of the gradients' own size)."""
    q, k, v, d_out, kw = _args([9, 70], [21, 90], 4, 2, 16, torch.float16, seed=7)
    out, lse = layers.attend(q, k, v, lse=True, **kw)
    got = layers.attend_grad(q, k, v, out, lse, d_out, **kw)
    bounds = [b for _, b in ref.attend_grad(q, k, v, d_out, **_reference_kw(kw))]
    g, h = _gen(4), 2.0 ** -8
    base = [t.double() for t in (q, k, v)]
    for i in range(3):
        d = torch.randn(base[i].shape, generator=g, device="cuda", dtype=torch.float64)
        moved = [[b + s * h * d if j == i else b for j, b in enumerate(base)] for s in (1, -1)]
        difference = (_loss(moved[0], d_out, kw) - _loss(moved[1], d_out, kw)) / (2 * h)
        allowed = (bounds[i] * d.abs()).sum() + 100 * h * h * (got[i].double() * d).abs().sum()
        assert abs(float((got[i].double() * d).sum() - difference)) <= float(allowed)


def _loss(qkv, d_out, kw):
    q, k, v = qkv
    total, group = 0.0, q.shape[1] // k.shape[1]
    for here, keys in ref._sequences(q.shape[0], k.shape[0], kw["q_offsets"], kw["kv_offsets"], None):
        kk, vv = k[keys.cuda()].repeat_interleave(group, 1), v[keys.cuda()].repeat_interleave(group, 1)
        p = torch.softmax(torch.einsum("qhd,khd->hqk", q[here], kk) * q.shape[2] ** -0.5, -1)
        total = total + (torch.einsum("hqk,khd->qhd", p, vv) * d_out[here].double()).sum()
    return total


@pytest.mark.parametrize("lengths", [([3] * 40, [9] * 40), ([1], [9_000]), ([3_001], [65]), ([500, 400], [600, 1_000]), ([50] * 200, [30] * 200)])
def test_equal_calls_give_equal_bits(layers, lengths):
    q, k, v, d_out, kw = _args(*lengths, 4, 2, 64, torch.bfloat16)
    out, lse = layers.attend(q, k, v, lse=True, **kw)
    grads = layers.attend_grad(q, k, v, out, lse, d_out, **kw)
    for _ in range(3):
        again = layers.attend(q, k, v, lse=True, **kw)
        assert torch.equal(again[0], out) and torch.equal(again[1], lse)
        for a, b in zip(grads, layers.attend_grad(q, k, v, out, lse, d_out, **kw)):
            assert torch.equal(a, b)


@pytest.mark.parametrize("bad", [[5, 40, 60], [0, 40, 59], [0, 61, 60], [-1, 3, 60], [0, -7, 60], [0, 2**40, 60], [60, 0, 0]])
@pytest.mark.parametrize("of", ["q_offsets", "kv_offsets"])
def test_offsets_that_break_their_rules_are_reported(ifvs, layers, bad, of):
    """Nothing outside the arrays is written (guards around the outputs), and the next
    call is right."""
    q, k, v, d_out, kw = _args([20, 40], [10, 50], 2, 2, 64, torch.bfloat16)
    want = layers.attend(q, k, v, lse=True, **kw)
    guard = torch.full((5, 64, 2, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    to = [g[2:62] for g in guard]
    broken = dict(kw, **{of: torch.tensor(bad, dtype=torch.int64, device="cuda")})
    for call in (lambda: layers.attend(q, k, v, out=to[0], **broken),
                 lambda: layers.attend_grad(q, k, v, *want, d_out, dq=to[1], dk=to[2], dv=to[3], **broken)):
        with pytest.raises(ifvs.IfvsError) as e:
            call()
        assert e.value.code == ifvs.IFVS_ERR_ARG and "offsets" in str(e.value)
    assert bool((guard[:, :2] == 7).all()) and bool((guard[:, 62:] == 7).all())
    assert torch.equal(layers.attend(q, k, v, **kw)[0], want[0])


def test_far_keys(layers):
    """Keys whose elements lie beyond 2^32: all but the last few are padding."""
    Tk, H, d = 4_300_000, 8, 128
    k = torch.full((Tk, H, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    g = _gen(3)
    n = 100
    k[-n:] = torch.randn(n, H, d, generator=g, device="cuda").bfloat16()
    q, d_out = (torch.randn(3, H, d, generator=g, device="cuda").bfloat16() for _ in range(2))
    ids = torch.full((Tk,), -1, dtype=torch.int32, device="cuda")
    ids[-n:] = 1
    last = k[-n:].clone()
    out, lse = layers.attend(q, k, k, kv_ids=ids, lse=True)
    (o, l) = ref.attend(q, last, last)
    within(out, *o)
    _lse_within(lse, l)
    dq, dk, dv = layers.attend_grad(q, k, k, out, lse, d_out, kv_ids=ids)
    for got, w in zip((dq, dk[-n:], dv[-n:]), ref.attend_grad(q, last, last, d_out)):
        within(got, *w)
    assert not dk[:-n].any() and not dv[:-n].any()


def test_refusals(ifvs, layers):
    q, k, v, d_out, kw = _args([20, 40], [10, 50], 4, 2, 64, torch.bfloat16)

    def code(*args, f=layers.attend, **more):
        with pytest.raises(ifvs.IfvsError) as e:
            f(*args, **more)
        return e.value.code

    assert code(q.float(), k.float(), v.float()) == ifvs.IFVS_ERR_UNSUPPORTED
    assert code(q[..., :60].contiguous(), k[..., :60].contiguous(), v[..., :60].contiguous()) == ifvs.IFVS_ERR_UNSUPPORTED
    big = torch.ones(2, 1, 136, dtype=torch.bfloat16, device="cuda")
    assert code(big, big, big) == ifvs.IFVS_ERR_ARG
    assert code(q[:, :3].contiguous(), k, v) == ifvs.IFVS_ERR_ARG              # 2 does not divide 3
    for scale in (0.0, -1.0, float("inf"), float("nan")):
        assert code(q, k, v, scale=scale) == ifvs.IFVS_ERR_ARG
    shifted = torch.empty(60 * 4 * 64 + 1, dtype=torch.bfloat16, device="cuda")[1:].view(60, 4, 64)
    assert code(shifted, k, v) == ifvs.IFVS_ERR_ARG
    odd = torch.empty(60, 4 * 64 + 4, dtype=torch.bfloat16, device="cuda")[:, :256].unflatten(1, (4, 64))
    for bad in (dict(kv_ids=torch.zeros(59, dtype=torch.int32, device="cuda")), dict(kv_ids=torch.zeros(60, device="cuda")),
                dict(q_offsets=kw["q_offsets"]), dict(q_offsets=kw["q_offsets"], kv_offsets=kw["kv_offsets"][:2]),
                dict(q_offsets=kw["q_offsets"].int(), kv_offsets=kw["kv_offsets"]), dict(out=q[:, :, :32]), dict(out=odd),
                dict(out=q.half()), dict(lse=torch.empty(60, 4, dtype=torch.bfloat16, device="cuda")),
                dict(lse=torch.empty(60, 3, device="cuda"))):
        with pytest.raises(ValueError):
            layers.attend(q, k, v, **bad)
    for args in ((q, k, v[:59]), (q, k.half(), v), (q, k[..., :32], v[..., :32]), (q[:, 0], k[:, 0], v[:, 0]), (odd, k, v),
                 (q.transpose(0, 1).contiguous().transpose(0, 1), k, v)):
        with pytest.raises(ValueError):
            layers.attend(*args)
    out, lse = layers.attend(q, k, v, lse=True)
    with pytest.raises(ifvs.IfvsError):
        layers.attend_grad(q, k, v, out, None, d_out)
    with pytest.raises(ValueError):
        layers.attend_grad(q, k, v, out, lse, d_out[:59])
    at = q.data_ptr()
    for field, value in (("Tq", -1), ("Tk", 2**31), ("heads", 0), ("kv_heads", 3), ("dh", 0), ("dh", 136), ("heads", 256), ("type", 7),
                         ("n_seq", 0), ("n_seq", 2), ("ld_q", 248), ("ld_k", 132), ("ld_out", 260)):
        p = ifvs.AttendParams(60, 60, 4, 2, 64, ifvs.IFVS_T_BF16, 1)
        p.scale = 1.0
        setattr(p, field, value)
        assert ifvs.lib().ifvs_attend(layers.h, ctypes.byref(p), at, at, at, at, None) == ifvs.IFVS_ERR_ARG, field
