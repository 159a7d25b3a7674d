"""The layers on streams other than the tensors' own: what a call without a stream
waits for, and whose memory the outputs are."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
LONG = 100_000_000          # clocks: about 50 ms


@pytest.fixture(scope="module")
def layers():
    from paper_2607_22922_gb300 import build
    build.build()
    from paper_2607_22922_gb300 import ifvs
    L = ifvs.Layers()
    yield L
    L.close()


def _operators(layers):
    """name: (input, call of it)"""
    T, D, F, bf = 40, 64, 72, torch.bfloat16
    ids = torch.arange(T, dtype=torch.int32, device="cuda") % 7
    w, w_in, w_out = torch.ones(D, dtype=bf, device="cuda"), torch.ones(2 * F, D, dtype=bf, device="cuda"), torch.ones(D, F, dtype=bf, device="cuda")
    y = torch.ones(T, D, dtype=bf, device="cuda")
    return {"embed": (7, lambda x, **s: [layers.embed(x, ids, **s)]),
            "embed_grad": (T, lambda x, **s: [layers.embed_grad(x, ids, V=7, **s)]),
            "norm_join": (T, lambda x, **s: layers.norm_join(x, y, None, w, w, **s)),
            "norm_join_grad": (T, lambda x, **s: [t for t in layers.norm_join_grad(x, y, None, w, w, x, y, **s) if t is not None]),
            "ffn": (T, lambda x, **s: [layers.ffn(x, w_in, w_out, **s)]),
            "ffn_grad": (T, lambda x, **s: layers.ffn_grad(x, w_in, w_out, y, **s))}


NAMES = ["embed", "embed_grad", "norm_join", "norm_join_grad", "ffn", "ffn_grad"]


@pytest.mark.parametrize("name", NAMES)
def test_a_call_without_a_stream_follows_the_current_one(layers, name):
    rows, call = _operators(layers)[name]
    x = torch.zeros(rows, 64, dtype=torch.bfloat16, device="cuda")
    want = call(torch.full_like(x, 1.5))
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(LONG)
        x.fill_(1.5)
        got = call(x)
    for p, q in zip(want, got):
        assert torch.equal(p, q)


@pytest.mark.parametrize("raw", [False, True])
@pytest.mark.parametrize("name", NAMES)
def test_outputs_are_the_memory_of_the_calls_stream(layers, name, raw):
    """An output that is dropped before its kernel has run: its memory may not go
    to a tensor of the current stream, where the kernel would overwrite it."""
    rows, call = _operators(layers)[name]
    x = torch.full((rows, 64), 1.5, dtype=torch.bfloat16, device="cuda")
    call(x)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(LONG)
    out = call(x, stream=s.cuda_stream if raw else s)
    shapes = [t.shape for t in out]
    del out
    mine = [torch.full(tuple(n), 7.0, dtype=torch.bfloat16, device="cuda") for n in shapes for _ in range(4)]
    torch.cuda.synchronize()
    for t in mine:
        assert bool((t == 7).all())


def test_the_default_stream_by_each_of_its_names(layers):
    rows, call = _operators(layers)["ffn"]
    x = torch.full((rows, 64), 1.5, dtype=torch.bfloat16, device="cuda")
    want = call(x)[0]
    s = torch.cuda.Stream()
    for stream in (None, 0, 1, torch.cuda.default_stream()):
        for here in (torch.cuda.default_stream(), s):
            with torch.cuda.stream(here):
                got = call(x, stream=stream)[0]
            torch.cuda.synchronize()
            assert torch.equal(got, want)


def test_a_call_without_a_stream_is_refused_in_a_capture(layers):
    rows, call = _operators(layers)["embed"]
    x = torch.full((rows, 64), 1.5, dtype=torch.bfloat16, device="cuda")
    y, s, graph = torch.zeros_like(x), torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        y.copy_(x)
        with pytest.raises(ValueError, match="capture"):
            call(x)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(x, y)
