"""Attention and its gradient without any key: every query has zeros and lse = -infinity,
every gradient is zero, at as many queries as the kernels for many short sequences take
(twice their rules' rows and sequences on the device at hand) and at fewer."""
import pytest

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


def _sms():
    return torch.cuda.get_device_properties(0).multi_processor_count


# sequences, queries of each, heads, of keys
FORMS = {"many": (lambda n: n, 40, 8, 8), "many, shared": (lambda n: 2 * n, 33, 8, 4), "one": (lambda n: 1, 16_000, 8, 8),
         "few": (lambda n: 3, 7, 8, 2)}


@pytest.mark.parametrize("type_", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("d", [8, 64, 128])
@pytest.mark.parametrize("name", sorted(FORMS))
def test_no_keys_at_all(layers, type_, d, name):
    count, n, H, Hk = FORMS[name]
    B = count(2 * _sms())
    g = torch.Generator(device="cuda")
    g.manual_seed(d)
    q, d_out = (torch.randn(B * n, H, d, generator=g, device="cuda").to(type_) for _ in range(2))
    none = torch.empty(0, Hk, d, dtype=type_, device="cuda")
    kws = [dict(q_offsets=torch.arange(B + 1, device="cuda") * n, kv_offsets=torch.zeros(B + 1, dtype=torch.int64, device="cuda"))]
    kws.append(dict(kws[0], kv_ids=torch.empty(0, dtype=torch.int32, device="cuda")))
    if B == 1:
        kws.append({})
    for kw in kws:
        out, lse = layers.attend(q, none, none, out=torch.full_like(q, 7), lse=torch.zeros(B * n, H, device="cuda"), **kw)
        assert not out.any() and bool((lse == -float("inf")).all())
        dq, dk, dv = layers.attend_grad(q, none, none, out, lse, d_out, dq=torch.full_like(q, 7), **kw)
        assert not dq.any() and dk.shape == dv.shape == (0, Hk, d)
