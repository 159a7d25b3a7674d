"""What projections and attention do when a wait runs out or a launch fails: which error is
reported, and that the handle's later calls are right."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


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


def _same(a, b):
    for p, q in zip(a, b):
        assert (p is None and q is None) or torch.equal(p, q)


def _linear(layers, T, D_in, D_out, act, dtype):
    g = torch.Generator(device="cuda")
    g.manual_seed(T)
    r = lambda *n: torch.randn(*n, generator=g, device="cuda").to(dtype)  # noqa: E731
    x, w, b, res = r(T, D_in), r(D_out, D_in) / D_in ** 0.5, r(D_out), r(T, D_out)
    return (lambda s=None: (layers.linear(x, w, b, act=act, residual=res, stream=s),),
            lambda s=None: layers.linear_grad(x, w, res, b, act=act, stream=s))


def _attend(layers, lq, lk, H, Hk, d, dtype):
    g = torch.Generator(device="cuda")
    g.manual_seed(len(lq))
    r = lambda *n: torch.randn(*n, generator=g, device="cuda").to(dtype)  # noqa: E731
    q, d_out, k, v = r(sum(lq), H, d), r(sum(lq), H, d), r(sum(lk), Hk, d), r(sum(lk), Hk, d)
    kw = dict(q_offsets=torch.tensor([0] + lq, device="cuda").cumsum(0), kv_offsets=torch.tensor([0] + lk, device="cuda").cumsum(0))
    out, lse = layers.attend(q, k, v, lse=True, **kw)
    return (lambda s=None: layers.attend(q, k, v, lse=True, stream=s, **kw),
            lambda s=None: layers.attend_grad(q, k, v, out, lse, d_out, stream=s, **kw))


# ---- waits that run out.  While IFVS_TEST_STALL_COPIES is 1 the barriers expect more bytes
# than the copies deliver: every wait runs out after its bound, the call reports it, and the
# same call is right again once it is 0.

def _runs_out(ifvs, monkeypatch, call):
    want = call()
    monkeypatch.setenv("IFVS_TEST_STALL_COPIES", "1")
    with pytest.raises(ifvs.IfvsError) as e:
        call()
    assert e.value.code == ifvs.IFVS_ERR_TIMEOUT
    monkeypatch.setenv("IFVS_TEST_STALL_COPIES", "0")
    _same(want, call())


# single CTAs and pairs, sums whole and in parts, with an activation and without
@pytest.mark.parametrize("T,D_in,D_out,act,dtype", [(5, 64, 72, "silu", torch.float16), (300, 4096, 136, "none", torch.bfloat16),
                                                    (5_000, 512, 2560, "gelu", torch.bfloat16)])
def test_linear_wait_runs_out(ifvs, layers, monkeypatch, T, D_in, D_out, act, dtype):
    for call in _linear(layers, T, D_in, D_out, act, dtype):
        _runs_out(ifvs, monkeypatch, call)


# long sequences, whole and in parts; many short ones, of one chunk of keys and of several
@pytest.mark.parametrize("lq,lk,H,Hk,d,dtype", [([300, 200], [400, 700], 2, 1, 128, torch.bfloat16), ([130], [3_000], 2, 2, 64, torch.float16),
                                                ([50] * 400, [30] * 400, 8, 4, 64, torch.bfloat16),
                                                ([40] * 200, [60] * 200, 4, 4, 128, torch.float16)])
def test_attend_wait_runs_out(ifvs, layers, monkeypatch, lq, lk, H, Hk, d, dtype):
    for call in _attend(layers, lq, lk, H, Hk, d, dtype):
        _runs_out(ifvs, monkeypatch, call)


# ---- calls that fail between their launches.  While IFVS_FAIL_LAUNCH is n the n-th launch
# of a call is not made and fails.

def _calls(layers):
    """name: call, whether it uses the workspace"""
    some, many = _linear(layers, 130, 4104, 64, "silu", torch.bfloat16), _attend(layers, [2, 3], [2_000, 2_001], 2, 2, 64, torch.bfloat16)
    long, parts = (_attend(layers, *n, 2, 2, 64, torch.bfloat16) for n in (([300, 400], [500, 600]), ([3_001], [65])))
    return {"linear": some[0], "linear_grad": some[1], "attend, parts": many[0], "attend_grad, long": long[1], "attend_grad, parts": parts[1]}


@pytest.mark.parametrize("name", ["linear", "linear_grad", "attend, parts", "attend_grad, long", "attend_grad, parts"])
def test_a_launch_fails(ifvs, layers, monkeypatch, name):
    """The call reports it, no launch follows, the next call that uses the workspace waits
    for what was enqueued (behind 50 ms of other work here), on another stream."""
    call = _calls(layers)[name]
    want = call()
    n = 0
    while True:
        n += 1
        assert n < 10
        first, second = torch.cuda.Stream(), torch.cuda.Stream()
        torch.cuda.synchronize()
        with torch.cuda.stream(first):
            torch.cuda._sleep(100_000_000)
            slept = torch.cuda.Event()
            slept.record(first)
            monkeypatch.setenv("IFVS_FAIL_LAUNCH", str(n))
            try:
                got = call(first)
                break                   # the call has n - 1 launches
            except ifvs.IfvsError as e:
                assert e.code == ifvs.IFVS_ERR_CUDA
            monkeypatch.setenv("IFVS_FAIL_LAUNCH", "0")
        with torch.cuda.stream(second):
            got = call(second)
            done = torch.cuda.Event()
            done.record(second)
        done.synchronize()
        assert slept.query()
        _same(want, got)
    torch.cuda.synchronize()
    _same(want, got)
    assert n > 2                        # there was a second launch to fail
    layers.status()
