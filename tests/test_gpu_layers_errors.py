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
def layers(ifvs):
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
