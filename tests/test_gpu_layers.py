"""The encoder's layers against their definitions in float64, at the sizes and
sequences where they can go wrong, and their refusals.  Every tolerance is the
bound that tests/layers_util.py derives for that element."""
import os

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


def _ids(kind, T, V, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    if kind == "one":
        return torch.full((T,), V - 1, dtype=torch.int32, device="cuda")
    if kind == "padding":
        return torch.full((T,), -1, dtype=torch.int32, device="cuda")
    ids = torch.randint(0, V, (T,), generator=g, device="cuda")
    if kind == "hot":
        ids = torch.where(torch.rand(T, generator=g, device="cuda") < 0.6, ids % min(V, 3), ids)
    ids[torch.rand(T, generator=g, device="cuda") < 0.1] = -1
    return ids.int()


# ------------------------------------------------------------------ embedding

WIDTHS = [1, 7, 33, 96, 100, 128, 257, 960]


@pytest.mark.parametrize("type_", sorted(TYPES))
@pytest.mark.parametrize("D", WIDTHS)
def test_embed(layers, type_, D):
    for T, V in ((1, 1), (17, 300), (1021, 40)):
        r = _rand(D + T)
        table = r(V, D).to(TYPES[type_])
        ids = _ids("any", T, V, T)
        ref.within(layers.embed(table, ids, 11.3), *ref.embed(table, ids, 11.3))


@pytest.mark.parametrize("type_", sorted(TYPES))
@pytest.mark.parametrize("D", WIDTHS)
def test_embed_grad(layers, type_, D):
    for T, V, kind in ((1, 1, "one"), (17, 300, "any"), (1021, 40, "hot"), (64, 70, "padding"), (513, 5, "one")):
        d_out = _rand(D + T)(T, D).to(TYPES[type_])
        ids = _ids(kind, T, V, T + V)
        ref.within(layers.embed_grad(d_out, ids, 0.7, V=V), *ref.embed_grad(d_out, ids, 0.7, V))


@pytest.mark.parametrize("T,V,kind", [(40_007, 70_001, "hot"), (40_007, 3, "any"), (9_001, 1_200_000, "any"),
                                      (150_001, 255, "hot"), (150_001, 257, "any"), (33_333, 33_333, "one")])
def test_embed_grad_of_many_tokens(layers, T, V, kind):
    """More tokens than one pass of a sort sees at once, tables of one to three
    bytes of ids, runs over many parts of the sorted order."""
    for D, type_ in ((20, "f32"), (24, "bf16")):
        d_out = _rand(T)(T, D).to(TYPES[type_])
        ids = _ids(kind, T, V, V)
        ref.within(layers.embed_grad(d_out, ids, 1.5, V=V), *ref.embed_grad(d_out, ids, 1.5, V))


def test_embed_grad_sums_in_a_fixed_order(layers):
    d_out = _rand(3)(70_001, 36)
    ids = _ids("hot", 70_001, 999, 3)
    a = layers.embed_grad(d_out, ids, V=999)
    for _ in range(3):
        assert torch.equal(a, layers.embed_grad(d_out, ids, V=999))


def test_embed_without_tokens(layers):
    ids = torch.empty(0, dtype=torch.int32, device="cuda")
    assert layers.embed(torch.ones(4, 8, device="cuda"), ids).shape == (0, 8)
    g = torch.full((5, 8), 7.0, device="cuda")
    layers.embed_grad(torch.empty(0, 8, device="cuda"), ids, d_table=g)
    assert not g.any()


def test_embed_reports_ids_out_of_range(ifvs, layers):
    """The rows are zeros, nothing is read or added, and the error arrives: from
    the waiting call itself, else from status()."""
    table = torch.ones(4, 24, device="cuda")
    for bad in (4, -2, 2**31 - 1, -2**31):
        ids = torch.tensor([0, bad, 3], dtype=torch.int32, device="cuda")
        out = torch.full((3, 24), 9.0, device="cuda")
        with pytest.raises(ifvs.IfvsError) as e:
            layers.embed(table, ids, out=out)
        assert e.value.code == ifvs.IFVS_ERR_ARG and "id" in str(e.value)
        assert out.tolist() == [[1.0] * 24, [0.0] * 24, [1.0] * 24]
        d = torch.full((4, 24), 9.0, device="cuda")
        layers.embed_grad(out + 1, ids, d_table=d, stream=torch.cuda.current_stream())
        with pytest.raises(ifvs.IfvsError):
            layers.status()
        layers.status()
        assert d[:, 0].tolist() == [2.0, 0.0, 0.0, 2.0]


# ------------------------------------------------------------------ norm, gate, residual

def _join_inputs(T, D, type_, offsets, seed):
    r, dt = _rand(seed), TYPES[type_]
    B = 1 if offsets is None else len(offsets) - 1
    off = None if offsets is None else torch.tensor(offsets, dtype=torch.int64, device="cuda")
    return dict(x=(1.5 * r(T, D)).to(dt), y=(0.5 * r(T, D)).to(dt), gate=(1 + 0.3 * r(B, D)).to(dt),
                w_post=(1 + 0.1 * r(D)).to(dt), w_pre=(1 + 0.1 * r(D)).to(dt), dxo=r(T, D).to(dt), dn=r(T, D).to(dt)), off


def _join_both(layers, v, off, gate=True, pre=True, d_x=True, rho=0.7):
    gate_, w_pre = v["gate"] if gate else None, v["w_pre"] if pre else None
    kw = dict(offsets=off, res_scale=rho, eps=EPS)
    _check(layers.norm_join(v["x"], v["y"], gate_, v["w_post"], w_pre, **kw),
           ref.norm_join(v["x"], v["y"], gate_, v["w_post"], w_pre, off, rho, EPS))
    dxo, dn = v["dxo"] if d_x or not pre else None, v["dn"] if pre else None
    _check(layers.norm_join_grad(v["x"], v["y"], gate_, v["w_post"], w_pre, dxo, dn, **kw),
           ref.norm_join_grad(v["x"], v["y"], gate_, v["w_post"], w_pre, dxo, dn, off, rho, EPS))


@pytest.mark.parametrize("type_", sorted(TYPES))
@pytest.mark.parametrize("D", WIDTHS + [513, 1024, 1536, 2050, 4096, 8192])
def test_norm_join(layers, type_, D):
    for T, offsets in ((1, None), (37, [0, 0, 1, 17, 17, 37, 37]), (260, [0, 260])):
        v, off = _join_inputs(T, D, type_, offsets, D + T)
        _join_both(layers, v, off)


@pytest.mark.parametrize("lengths", [[5000], [1] * 700, [0, 3, 0, 0, 2500, 1, 0, 40, 0], [0] * 50 + [7] + [0] * 50,
                                     [17] * 60 + [3000] + [17] * 60])
def test_norm_join_sequences(layers, lengths):
    """Sequences of none to thousands of tokens: their gates' gradients join
    parts of a sequence that different warps sum."""
    offsets = [0]
    for n in lengths:
        offsets.append(offsets[-1] + n)
    for D, type_ in ((40, "f32"), (97, "f16"), (320, "bf16")):
        v, off = _join_inputs(offsets[-1], D, type_, offsets, len(lengths))
        _join_both(layers, v, off)


@pytest.mark.parametrize("D,type_", [(64, "f32"), (51, "bf16"), (128, "f16")])
def test_norm_join_parts_left_out(layers, D, type_):
    v, off = _join_inputs(90, D, type_, [0, 40, 90], 5)
    _join_both(layers, v, off, gate=False)
    _join_both(layers, v, off, pre=False)
    _join_both(layers, v, off, d_x=False)
    v, _ = _join_inputs(90, D, type_, None, 6)
    _join_both(layers, v, None, gate=False, rho=0.0)
    # the first norm of an encoder: no block before it
    x_out, n = layers.norm_join(v["x"], w_pre=v["w_pre"], eps=EPS)
    assert x_out is None
    ref.within(n, *ref.norm_join(v["x"], None, None, None, v["w_pre"], None, 1.0, EPS)[1])
    for dxo in (v["dxo"], None):
        _check(layers.norm_join_grad(v["x"], w_pre=v["w_pre"], d_x_out=dxo, d_n=v["dn"], eps=EPS),
               ref.norm_join_grad(v["x"], None, None, None, v["w_pre"], dxo, v["dn"], None, 1.0, EPS))


def test_norm_join_rows_of_zeros(layers):
    """mean square 0: eps alone keeps the norms finite."""
    v, off = _join_inputs(24, 72, "f32", [0, 10, 24], 9)
    v["x"][3:9], v["y"][5:12] = 0, 0
    _join_both(layers, v, off)


def test_norm_join_not_finite_stays_in_its_row(layers):
    v, off = _join_inputs(40, 128, "bf16", [0, 20, 40], 10)
    kw = dict(offsets=off, res_scale=0.7, eps=EPS)
    a = (v["y"], v["gate"], v["w_post"], v["w_pre"])
    clean = layers.norm_join(v["x"], *a, **kw)
    v["x"][7, 3], v["x"][21, 0] = float("nan"), float("inf")
    got = layers.norm_join(v["x"], *a, **kw)
    rows = [i for i in range(40) if i not in (7, 21)]
    for c, g in zip(clean, got):
        assert torch.equal(c[rows], g[rows])
    assert got[1][7].isnan().all()


def test_norm_join_without_tokens(layers):
    v, _ = _join_inputs(0, 16, "f32", None, 1)
    off = torch.zeros(4, dtype=torch.int64, device="cuda")
    gate = torch.ones(3, 16, device="cuda")
    a = (v["y"], gate, v["w_post"], v["w_pre"])
    xo, n = layers.norm_join(v["x"], *a, offsets=off)
    assert xo.shape == n.shape == (0, 16)
    got = layers.norm_join_grad(v["x"], *a, v["dxo"], v["dn"], offsets=off)
    assert not got[2].any() and not got[3].any() and not got[4].any()


def test_norm_join_grad_in_a_fixed_order(layers):
    v, off = _join_inputs(9_001, 130, "f32", [0, 8000, 8001, 9001], 4)
    a = (v["x"], v["y"], v["gate"], v["w_post"], v["w_pre"], v["dxo"], v["dn"])
    first = layers.norm_join_grad(*a, offsets=off)
    for _ in range(3):
        for p, q in zip(first, layers.norm_join_grad(*a, offsets=off)):
            assert torch.equal(p, q)


def test_norm_join_reports_offsets(ifvs, layers):
    """Offsets that break their rules are reported, and no row beyond the arrays is touched."""
    T, D = 50, 64
    v, _ = _join_inputs(T, D, "f32", [0, 20, 50], 11)
    for bad in ([0, 20, 40], [0, 60, 50], [5, 20, 50], [0, -7, 50], [0, 2**40, 50], [30, 20, 10]):
        off = torch.tensor(bad, dtype=torch.int64, device="cuda")
        guard = torch.full((4 + 2 + 4, D), 3.0, device="cuda")
        with pytest.raises(ifvs.IfvsError) as e:
            layers.norm_join(v["x"], v["y"], v["gate"], v["w_post"], v["w_pre"], offsets=off)
        assert e.value.code == ifvs.IFVS_ERR_ARG and "offsets" in str(e.value)
        with pytest.raises(ifvs.IfvsError):
            layers.norm_join_grad(v["x"], v["y"], v["gate"], v["w_post"], v["w_pre"], v["dxo"], v["dn"], offsets=off,
                                  d_gate=guard[4:6])
        assert bool((guard[:4] == 3).all()) and bool((guard[6:] == 3).all())


# ------------------------------------------------------------------ feed-forward

FFN_SHAPES = [(1, 8, 8), (1, 960, 264), (3, 104, 520), (8, 64, 128), (9, 128, 136), (16, 256, 344), (17, 40, 1000),
              (128, 64, 64), (129, 136, 200), (300, 96, 256), (513, 128, 344), (1000, 320, 136)]


def _ffn_inputs(T, D, F, type_, seed):
    r, dt = _rand(seed), TYPES[type_]
    return (r(T, D).to(dt), (r(2 * F, D) / D ** 0.5).to(dt), (r(D, F) / F ** 0.5).to(dt)), r(T, D).to(dt)


@pytest.mark.parametrize("type_", ["f16", "bf16"])
@pytest.mark.parametrize("act", ["silu", "gelu", "relu"])
@pytest.mark.parametrize("T,D,F", FFN_SHAPES)
def test_ffn(layers, T, D, F, act, type_):
    a, dy = _ffn_inputs(T, D, F, type_, T + D + F)
    ref.within(layers.ffn(*a, act=act), *ref.ffn(*a, act))
    _check(layers.ffn_grad(*a, dy, act=act), ref.ffn_grad(*a, dy, act))


def test_ffn_of_many_tokens(layers):
    """More tiles of tokens than SMs, sums over thousands of tokens."""
    a, dy = _ffn_inputs(20_011, 72, 136, "bf16", 8)
    ref.within(layers.ffn(*a), *ref.ffn(*a, "silu"))
    _check(layers.ffn_grad(*a, dy), ref.ffn_grad(*a, dy, "silu"))


def test_ffn_large_gate_values(layers):
    """Gates far from 0: exponentials that overflow or vanish."""
    for act in ("silu", "gelu"):
        (x, w_in, w_out), dy = _ffn_inputs(70, 64, 64, "bf16", 3)
        w_in[:64] *= 40
        ref.within(layers.ffn(x, w_in, w_out, act=act), *ref.ffn(x, w_in, w_out, act))
        _check(layers.ffn_grad(x, w_in, w_out, dy, act=act), ref.ffn_grad(x, w_in, w_out, dy, act))


def test_ffn_not_finite_stays_in_its_row(layers):
    for T in (5, 200):
        (x, w_in, w_out), dy = _ffn_inputs(T, 128, 192, "bf16", 4)
        clean, clean_dx = layers.ffn(x, w_in, w_out), layers.ffn_grad(x, w_in, w_out, dy)[0]
        x[3, 5] = float("inf")
        rows = [i for i in range(T) if i != 3]
        assert torch.equal(clean[rows], layers.ffn(x, w_in, w_out)[rows])
        assert torch.equal(clean_dx[rows], layers.ffn_grad(x, w_in, w_out, dy)[0][rows])


def test_ffn_without_tokens(layers):
    (x, w_in, w_out), dy = _ffn_inputs(0, 64, 72, "f16", 1)
    assert layers.ffn(x, w_in, w_out).shape == (0, 64)
    dx, a, b = layers.ffn_grad(x, w_in, w_out, dy, d_w_in=torch.ones_like(w_in), d_w_out=torch.ones_like(w_out))
    assert dx.shape == (0, 64) and not a.any() and not b.any()


def test_ffn_grad_in_a_fixed_order(layers):
    for T in (7, 3001):
        a, dy = _ffn_inputs(T, 128, 264, "bf16", T)
        y, first = layers.ffn(*a), layers.ffn_grad(*a, dy)
        for _ in range(3):
            assert torch.equal(y, layers.ffn(*a))
            for p, q in zip(first, layers.ffn_grad(*a, dy)):
                assert torch.equal(p, q)


# ------------------------------------------------------------------ differences

def _slope(f, v, d, h):
    return float(f(v + h * d) - f(v - h * d)) / (2 * h)


def test_gradients_against_differences():
    """Every gradient along a random direction against central differences of
    the definition in float64.  The difference's own error, h^2/6 of the third
    derivative, is below 1e-6 of the gradient's size at h = 1e-4; the rest is
    the bound of the elements along the direction."""
    from paper_2607_22922_gb300 import ifvs as mod
    L = mod.Layers()

    def agree(f, v, got, bound, seed):
        d = _rand(seed)(*v.shape).double()
        want = _slope(f, v.double(), d, 1e-4)
        assert abs(want - float((got.double() * d).sum())) <= float((bound * d.abs()).sum()) + 1e-6 * float(
            (got.double().abs() * d.abs()).sum())

    # embedding
    ids = _ids("hot", 300, 20, 1)
    r = _rand(21)
    table, w = r(20, 24), r(300, 24)
    agree(lambda v: (ref.embed(v, ids, 3.0)[0] * w).sum() if v.dtype != torch.float64 else _embed64(v, ids, 3.0, w),
          table, L.embed_grad(w, ids, 3.0, V=20), ref.embed_grad(w, ids, 3.0, 20)[1], 1)

    # norm, gate, residual
    v, off = _join_inputs(60, 48, "f32", [0, 13, 13, 60], 22)
    names = ("x", "y", "gate", "w_post", "w_pre")
    p = {k: v[k].double() for k in names}
    xo = _join64(p, off)[0].float()
    grads = L.norm_join_grad(xo, v["y"], v["gate"], v["w_post"], v["w_pre"], v["dxo"], v["dn"], offsets=off, res_scale=0.7,
                             eps=EPS)
    bounds = ref.norm_join_grad(xo, v["y"], v["gate"], v["w_post"], v["w_pre"], v["dxo"], v["dn"], off, 0.7, EPS)
    for i, k in enumerate(names):
        def f(t, k=k):
            a, n = _join64({**p, k: t}, off)
            return (a * v["dxo"].double()).sum() + (n * v["dn"].double()).sum()
        # x_out was rounded to float32 on its way in: 2^-24 of every term
        agree(f, p[k], grads[i], bounds[i][1] + 2 ** -20 * bounds[i][0].abs(), 30 + i)

    # feed-forward
    for act in ("silu", "gelu"):
        a, dy = _ffn_inputs(50, 64, 72, "f16", 23)
        got, bounds = L.ffn_grad(*a, dy, act=act), ref.ffn_grad(*a, dy, act)
        q = [t.double() for t in a]
        for i in range(3):
            def f(t, i=i):
                z = list(q)
                z[i] = t
                g, u = (z[0] @ z[1].t()).chunk(2, 1)
                return ((ref.activation(act, g)[0] * u) @ z[2].t() * dy.double()).sum()
            agree(f, q[i], got[i], bounds[i][1], 40 + i)
    L.close()


def _embed64(table, ids, scale, w):
    keep = ids >= 0
    return (scale * table[ids[keep].long()] * w[keep].double()).sum()


def _join64(p, off, rho=0.7):
    def norm(v):
        return v / torch.sqrt((v * v).mean(1, keepdim=True) + EPS)
    xo = rho * p["x"] + p["gate"][ref.sequences(off, len(p["x"]), "cuda")] * p["w_post"] * norm(p["y"])
    return xo, p["w_pre"] * norm(xo)


# ------------------------------------------------------------------ streams, workspace, refusals

def test_calls_on_several_streams_share_the_workspace(layers):
    """Calls that use the workspace, enqueued on two streams in turn without any
    synchronisation by the caller, on inputs made on their own stream."""
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    a, dy = _ffn_inputs(700, 128, 264, "bf16", 5)
    d_out, ids = _rand(6)(30_000, 64), _ids("hot", 30_000, 500, 6)
    want_f, want_e = layers.ffn_grad(*a, dy), layers.embed_grad(d_out, ids, V=500)
    torch.cuda.synchronize()
    got = []
    for i in range(12):
        s = streams[i % 2]
        with torch.cuda.stream(s):
            if i % 3 == 0:
                got.append((layers.embed_grad(d_out * 1, ids, V=500, stream=s), want_e))
            else:
                got.append((layers.ffn_grad(*a, dy * 1, stream=s)[i % 3], want_f[i % 3]))
    torch.cuda.synchronize()
    layers.status()
    for g, w in got:
        assert torch.equal(g, w)


def test_calls_in_a_graph(layers):
    """Captured once the workspace has its size, replayed on new inputs."""
    a, dy = _ffn_inputs(40, 64, 136, "bf16", 7)
    y, dx = torch.empty_like(a[0]), torch.empty_like(a[0])
    s = torch.cuda.Stream()
    layers.ffn_grad(*a, dy)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        layers.ffn(*a, y=y, stream=s)
        layers.ffn_grad(*a, dy, dx=dx, stream=s)
    a[0].copy_(_ffn_inputs(40, 64, 136, "bf16", 8)[0][0])
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, layers.ffn(*a)) and torch.equal(dx, layers.ffn_grad(*a, dy)[0])


def test_a_captured_workspace_outlives_its_growth(ifvs):
    L = ifvs.Layers()
    d_out, ids = _rand(14)(900, 40), _ids("hot", 900, 64, 14)
    out = torch.empty(64, 40, device="cuda")
    want = L.embed_grad(d_out, ids, V=64)
    s, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        L.embed_grad(d_out, ids, d_table=out, stream=s)
        with pytest.raises(ifvs.IfvsError) as e:     # nothing grows in a capture
            L.embed_grad(torch.empty(300_000, 40, device="cuda"), torch.empty(300_000, dtype=torch.int32, device="cuda"),
                         d_table=out, stream=s)
        assert e.value.code == ifvs.IFVS_ERR_STATE
    L.embed_grad(_rand(15)(300_000, 40), _ids("any", 300_000, 64, 15), V=64)       # grows
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    del graph
    L.close()


@pytest.mark.parametrize("act,type_", [("silu", "f16"), ("gelu", "bf16"), ("gelu", "f16"), ("relu", "bf16")])
def test_ffn_pairs_of_ctas(layers, act, type_):
    """Tiles of 256 tokens in the hidden layer, of 128 in the products."""
    a, dy = _ffn_inputs(12_001, 136, 392, type_, 16)
    ref.within(layers.ffn(*a, act=act), *ref.ffn(*a, act))
    _check(layers.ffn_grad(*a, dy, act=act), ref.ffn_grad(*a, dy, act))


@pytest.mark.parametrize("T,V", [(33_000, 5000), (65_537, 600_000), (65_536, 511), (8_193, 512)])
def test_embed_grad_around_the_sorts_limits(layers, T, V):
    """One cluster of 16 or 32 warps a CTA, tiles beyond; one, two and three digits."""
    d_out, ids = _rand(T)(T, 12), _ids("hot", T, V, V)
    ref.within(layers.embed_grad(d_out, ids, V=V), *ref.embed_grad(d_out, ids, 1.0, V))


def test_failed_workspace_leaves_the_handle_usable(ifvs):
    L = ifvs.Layers()
    a, dy = _ffn_inputs(40, 64, 136, "bf16", 7)
    try:
        os.environ["IFVS_FAIL_ALLOC"] = "1"
        with pytest.raises(ifvs.IfvsError) as e:
            L.ffn_grad(*a, dy)
        assert e.value.code == ifvs.IFVS_ERR_OOM
    finally:
        os.environ.pop("IFVS_FAIL_ALLOC", None)
    _check(L.ffn_grad(*a, dy), ref.ffn_grad(*a, dy, "silu"))
    L.close()


def test_unaligned_arrays(ifvs, layers):
    """Rows that start between vectors: the same results for embedding and
    norms, a refusal from the feed-forward block."""
    T, D, V = 60, 64, 30
    r = _rand(12)

    def off(t):
        flat = torch.empty(t.numel() + 1, dtype=t.dtype, device="cuda")[1:]
        return flat.view(t.shape).copy_(t)

    for type_ in sorted(TYPES):
        dt = TYPES[type_]
        table, d_out, ids = r(V, D).to(dt), r(T, D).to(dt), _ids("any", T, V, 3)
        ref.within(layers.embed(off(table), ids, out=off(d_out)), *ref.embed(table, ids, 1.0))
        ref.within(layers.embed_grad(off(d_out), ids, d_table=off(table)), *ref.embed_grad(d_out, ids, 1.0, V))
        v, o = _join_inputs(T, D, type_, [0, 20, 60], 13)
        _join_both(layers, {k: off(t) for k, t in v.items()}, o)
    (x, w_in, w_out), _ = _ffn_inputs(5, 64, 64, "f16", 1)
    with pytest.raises(ifvs.IfvsError) as e:
        layers.ffn(off(x), w_in, w_out)
    assert e.value.code == ifvs.IFVS_ERR_ARG and "aligned" in str(e.value)


def test_refusals(ifvs, layers):
    L = ifvs.lib()
    t = torch.ones(4, 16, device="cuda")
    ids = torch.zeros(4, dtype=torch.int32, device="cuda")
    p, i, o = t.data_ptr(), ids.data_ptr(), torch.empty_like(t).data_ptr()

    def refused(rc, code=ifvs.IFVS_ERR_ARG):
        assert rc == code and ifvs.ifvs_last_error()

    ok = dict(h=layers.h, table=p, V=4, D=16, type=0, ids=i, T=4, scale=1.0, out=o)

    def embed(**kw):
        a = {**ok, **kw}
        return L.ifvs_embed(a["h"], a["table"], a["V"], a["D"], a["type"], a["ids"], a["T"], a["scale"], a["out"], None)

    assert embed() == 0
    for kw in (dict(h=None), dict(table=None), dict(out=None), dict(ids=None), dict(V=0), dict(V=2**31), dict(D=0),
               dict(D=8193), dict(type=3), dict(type=-1), dict(T=-1), dict(T=2**31), dict(scale=float("nan")),
               dict(scale=float("inf")), dict(table=p + 2), dict(ids=i + 1)):
        refused(embed(**kw))

    jp = ifvs._join_params(t, None, t[0].clone(), None, None, 1.0, 1e-5, None)[0]

    def join(xp=p, yp=p, xo=o, no=None, **kw):
        q = ifvs.JoinParams()
        for f, _ in ifvs.JoinParams._fields_:
            setattr(q, f, kw.get(f, getattr(jp, f)))
        return L.ifvs_norm_join(layers.h, ifvs.C.byref(q), xp, yp, xo, no)

    assert join() == 0
    for kw in (dict(xp=None), dict(yp=None), dict(xo=None), dict(no=o), dict(w_post=None), dict(w_pre=p), dict(D=0),
               dict(T=-1), dict(n_seq=0), dict(n_seq=2), dict(eps=0.0), dict(eps=float("nan")),
               dict(res_scale=float("inf")), dict(type=9), dict(offsets=p + 4, n_seq=2)):
        refused(join(**kw))
    refused(L.ifvs_norm_join(None, ifvs.C.byref(jp), p, p, o, None))
    refused(L.ifvs_norm_join(layers.h, None, p, p, o, None))
    refused(L.ifvs_norm_join_grad(layers.h, ifvs.C.byref(jp), p, p, None, None, o, o, None, o, None))
    refused(L.ifvs_norm_join_grad(layers.h, ifvs.C.byref(jp), p, p, p, p, o, o, None, o, o))       # d_n without w_pre
    refused(L.ifvs_norm_join_grad(layers.h, ifvs.C.byref(jp), p, p, p, None, o, o, o, o, None))    # d_gate without gate
    refused(L.ifvs_norm_join_grad(layers.h, ifvs.C.byref(jp), p, p, p, None, o, None, None, o, None))

    (x, w_in, w_out), _ = _ffn_inputs(4, 16, 24, "bf16", 1)
    y = torch.empty_like(x)
    fp = ifvs._ffn_params(x, w_in, w_out, "silu", None)[0]

    def ffn(xp=x.data_ptr(), yp=y.data_ptr(), **kw):
        q = ifvs.FfnParams()
        for f, _ in ifvs.FfnParams._fields_:
            setattr(q, f, kw.get(f, getattr(fp, f)))
        return L.ifvs_ffn(layers.h, ifvs.C.byref(q), xp, yp)

    assert ffn() == 0
    for kw in (dict(xp=None), dict(yp=None), dict(w_in=None), dict(w_out=None), dict(T=-1), dict(D=0), dict(F=0),
               dict(F=65544), dict(act=3), dict(type=5), dict(xp=x.data_ptr() + 2)):
        refused(ffn(**kw))
    for kw in (dict(type=0), dict(D=12), dict(F=20)):
        refused(ffn(**kw), ifvs.IFVS_ERR_UNSUPPORTED)
    refused(L.ifvs_layers_status(None))
    h = ifvs.C.c_void_p()
    refused(L.ifvs_layers_create(ifvs.C.byref(h), 10_000))

    # the binding's own
    with pytest.raises(TypeError):
        layers.embed(t.double(), ids)
    with pytest.raises(ValueError):
        layers.embed(t, ids.long())
    with pytest.raises(ValueError):
        layers.embed(t.t(), ids)
    with pytest.raises(ValueError):
        layers.embed(t, ids, out=torch.empty(3, 16, device="cuda"))
    with pytest.raises(ValueError):
        layers.embed_grad(t, ids[:3], V=4)
    with pytest.raises(ValueError):
        layers.ffn(x, w_in[:24], w_out)
    with pytest.raises(ValueError):
        layers.ffn(x, w_in, w_out, act="tanh")
    with pytest.raises(ValueError):
        layers.norm_join(t, t, w_post=t[0].half())
