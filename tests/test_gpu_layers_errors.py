"""What the encoder's layers do when a call finds an error or fails on its way:
which error is reported, and that the handle's later calls are right."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
EPS = 1e-5


@pytest.fixture(scope="module")
def ifvs():
    from paper_2607_22922_gb300 import build
    build.build()
    from paper_2607_22922_gb300 import ifvs as mod
    return mod


@pytest.fixture
def layers(ifvs, monkeypatch):
    monkeypatch.setenv("IFVS_TEST_STALL_COPIES", "0")      # a handle that looks at them
    monkeypatch.setenv("IFVS_FAIL_LAUNCH", "0")
    L = ifvs.Layers()
    yield L
    L.close()


def _rand(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return lambda *shape: torch.randn(*shape, generator=g, device="cuda")


def _bad_id(layers, stream):
    layers.embed(torch.ones(4, 8, device="cuda"), torch.tensor([0, 9], dtype=torch.int32, device="cuda"), stream=stream)


def _bad_offsets(layers, stream):
    x, w = torch.ones(6, 8, device="cuda"), torch.ones(8, device="cuda")
    layers.norm_join(x, x, torch.ones(2, 8, device="cuda"), w, w, offsets=torch.tensor([0, 3, 5], device="cuda"), stream=stream)


def test_a_later_error_does_not_hide_an_earlier_one(ifvs, layers):
    s = torch.cuda.current_stream()
    for calls in ((_bad_id, _bad_offsets), (_bad_offsets, _bad_id)):
        for call in calls:
            call(layers, s)
        with pytest.raises(ifvs.IfvsError) as e:
            layers.status()
        assert e.value.code == ifvs.IFVS_ERR_ARG and "id" in str(e.value)
        layers.status()
    _bad_offsets(layers, s)
    with pytest.raises(ifvs.IfvsError) as e:
        layers.status()
    assert "offsets" in str(e.value)


# ---- waits that run out.  While IFVS_TEST_STALL_COPIES is 1 the barriers expect
# more bytes than the copies deliver: every wait runs out after its bound, the call
# reports it, and the same call is right again once it is 0.

def _same(a, b):
    for p, q in zip(a, b):
        assert (p is None and q is None) or torch.equal(p, q)


def _runs_out(ifvs, monkeypatch, call):
    want = call()
    monkeypatch.setenv("IFVS_TEST_STALL_COPIES", "1")
    for _ in range(2):
        with pytest.raises(ifvs.IfvsError) as e:
            call()
        assert e.value.code == ifvs.IFVS_ERR_TIMEOUT
    monkeypatch.setenv("IFVS_TEST_STALL_COPIES", "0")
    _same(want, call())


def _join_args(T, D, dtype, seed=1):
    r = _rand(seed)
    off = torch.tensor([0, T // 3, T // 3, T], dtype=torch.int64, device="cuda")
    v = [r(T, D).to(dtype), r(T, D).to(dtype), r(3, D).to(dtype), r(D).to(dtype), r(D).to(dtype)]
    return v, [r(T, D).to(dtype), r(T, D).to(dtype)], off


# rows on 16 bytes and between them, one warp a team and many, few tokens a team and
# many, a ring of one place (float32 rows beyond 4096 in the gradient)
@pytest.mark.parametrize("T,D,dtype", [(1, 64, torch.float32), (5, 128, torch.bfloat16), (20_000, 96, torch.float16),
                                       (20_000, 97, torch.bfloat16), (3_000, 1030, torch.bfloat16), (700, 8192, torch.float32)])
def test_norm_join_wait_runs_out(ifvs, layers, monkeypatch, T, D, dtype):
    v, d, off = _join_args(T, D, dtype)
    _runs_out(ifvs, monkeypatch, lambda: layers.norm_join(*v, offsets=off, eps=EPS))
    _runs_out(ifvs, monkeypatch, lambda: layers.norm_join(v[0], w_pre=v[4], eps=EPS))
    _runs_out(ifvs, monkeypatch, lambda: layers.norm_join_grad(*v, *d, offsets=off, eps=EPS))
    _runs_out(ifvs, monkeypatch, lambda: layers.norm_join_grad(v[0], w_pre=v[4], d_n=d[1], eps=EPS))


def test_a_bad_argument_does_not_hide_a_wait_that_ran_out(ifvs, layers, monkeypatch):
    v, _, off = _join_args(50, 64, torch.float32)
    s = torch.cuda.current_stream()
    monkeypatch.setenv("IFVS_TEST_STALL_COPIES", "1")
    layers.norm_join(*v, offsets=off, eps=EPS, stream=s)
    monkeypatch.setenv("IFVS_TEST_STALL_COPIES", "0")
    _bad_offsets(layers, s)
    _bad_id(layers, s)
    with pytest.raises(ifvs.IfvsError) as e:
        layers.status()
    assert e.value.code == ifvs.IFVS_ERR_TIMEOUT
    layers.status()


# rows of one slice and of several, tokens of one part and of many, padding
@pytest.mark.parametrize("T,D,V,dtype", [(1, 8, 3, torch.float32), (31, 128, 3, torch.bfloat16), (5_000, 64, 700, torch.float32),
                                         (90_001, 960, 400, torch.float16), (400_000, 256, 9_000, torch.bfloat16)])
def test_embed_grad_wait_runs_out(ifvs, layers, monkeypatch, T, D, V, dtype):
    r = _rand(T)
    d_out = r(T, D).to(dtype)
    ids = torch.randint(-1, V, (T,), dtype=torch.int32, device="cuda", generator=torch.Generator("cuda").manual_seed(T))
    ids[0] = V - 1
    _runs_out(ifvs, monkeypatch, lambda: (layers.embed_grad(d_out, ids, V=V),))


# single CTAs and pairs, sums whole and in parts, few tiles and many
@pytest.mark.parametrize("T,D,F,act,dtype", [(5, 64, 72, "silu", torch.float16), (129, 960, 264, "gelu", torch.bfloat16),
                                             (3_000, 128, 344, "relu", torch.float16), (12_001, 136, 392, "silu", torch.bfloat16)])
def test_ffn_wait_runs_out(ifvs, layers, monkeypatch, T, D, F, act, dtype):
    r = _rand(T)
    x, dy, w_in, w_out = (r(*s).to(dtype) for s in ((T, D), (T, D), (2 * F, D), (D, F)))
    _runs_out(ifvs, monkeypatch, lambda: (layers.ffn(x, w_in, w_out, act=act),))
    _runs_out(ifvs, monkeypatch, lambda: layers.ffn_grad(x, w_in, w_out, dy, act=act))


# ---- calls that fail between their launches.  While IFVS_FAIL_LAUNCH is n the n-th
# launch of a call is not made and fails.

def _calls(layers):
    v, d, off = _join_args(3_000, 64, torch.float32)
    r = _rand(7)
    x, dy, w_in, w_out = (r(*s).to(torch.bfloat16) for s in ((40, 64), (40, 64), (272, 64), (64, 136)))
    x1 = x[:1].clone()
    grads = {}
    for T, V in ((30_000, 500), (90_000, 600)):      # one cluster's sort; two passes of three launches
        ids = torch.randint(-1, V, (T,), dtype=torch.int32, device="cuda", generator=torch.Generator("cuda").manual_seed(T))
        rows = r(T, 20)
        grads["embed_grad %d" % T] = lambda s, ids=ids, rows=rows, V=V: (layers.embed_grad(rows, ids, V=V, stream=s),)
    return {**grads,
            "norm_join": lambda s: layers.norm_join(*v, offsets=off, eps=EPS, stream=s),
            "norm_join_grad": lambda s: layers.norm_join_grad(*v, *d, offsets=off, eps=EPS, stream=s),
            "ffn, one token": lambda s: (layers.ffn(x1, w_in, w_out, stream=s),),
            "ffn": lambda s: (layers.ffn(x, w_in, w_out, stream=s),),
            "ffn_grad": lambda s: layers.ffn_grad(x, w_in, w_out, dy, stream=s)}


LAUNCHES = {"embed_grad 30000": 3, "embed_grad 90000": 8, "norm_join": 1, "norm_join_grad": 2, "ffn, one token": 2, "ffn": 2,
            "ffn_grad": 2}


@pytest.mark.parametrize("name", sorted(LAUNCHES))
def test_no_launch_follows_one_that_failed(ifvs, layers, monkeypatch, name):
    """A kernel whose input was not made would go by what the workspace holds from
    earlier calls: the sort's scatter writes where the counts say."""
    call = _calls(layers)[name]
    want = call(None)
    for n in range(1, LAUNCHES[name] + 1):
        monkeypatch.setenv("IFVS_FAIL_LAUNCH", str(n))
        with pytest.raises(ifvs.IfvsError) as e:
            call(None)
        assert e.value.code == ifvs.IFVS_ERR_CUDA
        monkeypatch.setenv("IFVS_FAIL_LAUNCH", "0")
        torch.cuda.synchronize()
        _same(want, call(None))
    monkeypatch.setenv("IFVS_FAIL_LAUNCH", str(LAUNCHES[name] + 1))
    _same(want, call(None))


@pytest.mark.parametrize("name", sorted(LAUNCHES))
def test_a_call_that_fails_on_its_way_keeps_its_place(ifvs, layers, monkeypatch, name):
    """What such a call had enqueued (behind 50 ms of other work here) is waited for
    by the next call that uses the workspace, on another stream, and by the call
    itself where it has no stream."""
    call = _calls(layers)[name]
    want = call(None)
    made = LAUNCHES[name]
    for n in range(1, made + 1):
        first, second = torch.cuda.Stream(), torch.cuda.Stream()
        torch.cuda.synchronize()
        for s in (first, None):
            here = first if s is first else torch.cuda.default_stream()
            with torch.cuda.stream(here):
                torch.cuda._sleep(100_000_000)
                slept = torch.cuda.Event()
                slept.record(here)
                monkeypatch.setenv("IFVS_FAIL_LAUNCH", str(n))
                with pytest.raises(ifvs.IfvsError) as e:
                    call(s)
                monkeypatch.setenv("IFVS_FAIL_LAUNCH", "0")
            assert e.value.code == ifvs.IFVS_ERR_CUDA
            if s is None:
                assert n == 1 or slept.query()
            else:
                assert not slept.query()
                with torch.cuda.stream(second):
                    got = call(second)
                    done = torch.cuda.Event()
                    done.record(second)
                done.synchronize()
                # calls without workspace have no place in the order
                assert slept.query() or name == "norm_join"
                _same(want, got)
            torch.cuda.synchronize()
    monkeypatch.setenv("IFVS_FAIL_LAUNCH", str(made + 1))
    _same(want, call(None))
    layers.status()


# ---- offsets that break their rules are reported whatever their number

@pytest.mark.parametrize("T,bad", [(50, [5, 40]), (50, [0, 49]), (50, [0, 51]), (50, [-1, 50]), (50, [50, 0]), (0, [0, 1]),
                                   (0, [-1, 0]), (0, [0, 0, 5]), (0, [0, 3, 0])])
def test_offsets_of_one_sequence_and_of_no_tokens_are_checked(ifvs, layers, T, bad):
    x, w = torch.ones(T, 24, device="cuda"), torch.ones(24, device="cuda")
    gate, good = torch.ones(len(bad) - 1, 24, device="cuda"), [0] * (len(bad) - 1) + [T]
    for offsets in (bad, good):
        off = torch.tensor(offsets, dtype=torch.int64, device="cuda")
        for call in (lambda: layers.norm_join(x, x, gate, w, w, offsets=off),
                     lambda: layers.norm_join_grad(x, x, gate, w, w, x, x, offsets=off)):
            if offsets is good:
                call()
                continue
            with pytest.raises(ifvs.IfvsError) as e:
                call()
            assert e.value.code == ifvs.IFVS_ERR_ARG and "offsets" in str(e.value)
