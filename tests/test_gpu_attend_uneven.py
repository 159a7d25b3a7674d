"""One sequence that is longer than all the others together, among many short ones: what
waits behind its tiles for a second or more is not taken for a wait that ran out.  The
batches are those of the kernels for many short sequences on the device at hand."""
import pytest

import tokens_util as ref
from layers_util import within

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
BF = torch.bfloat16


@pytest.fixture(scope="module")
def layers():
    from paper_2607_22922_gb300 import build
    build.build()
    from paper_2607_22922_gb300 import ifvs
    L = ifvs.Layers()
    yield L
    L.close()


def _sequences():
    return 5 * torch.cuda.get_device_properties(0).multi_processor_count


def _offsets(lengths):
    return torch.tensor([0] + lengths, dtype=torch.int64, device="cuda").cumsum(0)


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def test_many_keys_in_one_sequence(layers):
    """80 million keys of which 200 are no padding, the others' values no numbers."""
    B, H, d, n, many = _sequences(), 8, 8, 12, 80_000_000
    g = _gen(1)
    lk = [many] + [30] * (B - 1)
    live = torch.cat([torch.randint(0, 2_000, (97,), generator=g, device="cuda"),
                      many - 1 - torch.randint(0, 2_000, (103,), generator=g, device="cuda")]).unique()
    k, v = (torch.full((sum(lk), 1, d), float("nan"), dtype=BF, device="cuda") for _ in range(2))
    ids = torch.full((sum(lk),), -1, dtype=torch.int32, device="cuda")
    at = torch.cat([live, torch.arange(many, sum(lk), device="cuda")])
    k[at], v[at] = (torch.randn(len(at), 1, d, generator=g, device="cuda").to(BF) for _ in range(2))
    ids[at] = 3
    q = torch.randn(B * n, H, d, generator=g, device="cuda").to(BF)
    qo = _offsets([n] * B)
    out, lse = layers.attend(q, k, v, q_offsets=qo, kv_offsets=_offsets(lk), kv_ids=ids, lse=True)
    o, l = ref.attend(q, k[at], v[at], q_offsets=qo, kv_offsets=_offsets([len(live)] + lk[1:]))
    within(out, *o)
    within(lse, *l)


@pytest.mark.parametrize("keys", [4, 0])
def test_many_rows_in_one_sequence(layers, keys):
    """40 million rows of a group, the gradients of all but a few of them zeros, so that the
    sums over them are of those few."""
    B, H, d, many = _sequences(), 64, 8, 625_000
    g = _gen(2)
    lq, lk = [many] + [1] * (B - 1), [keys] + [4] * (B - 1)
    Tq, Tk = sum(lq), sum(lk)
    at = torch.cat([torch.tensor([0, 1, 2, 70_001, 311_111, many - 2, many - 1], device="cuda"), torch.arange(many, Tq, device="cuda")])
    q = torch.randn(Tq, H, d, generator=g, device="cuda", dtype=BF)
    k, v = (torch.randn(Tk, 1, d, generator=g, device="cuda").to(BF) for _ in range(2))
    d_out = torch.zeros_like(q)
    d_out[at] = torch.randn(len(at), H, d, generator=g, device="cuda").to(BF)
    kw = dict(q_offsets=_offsets(lq), kv_offsets=_offsets(lk))
    out, lse = layers.attend(q, k, v, lse=True, **kw)
    dq, dk, dv = layers.attend_grad(q, k, v, out, lse, d_out, dq=torch.full_like(q, 7), **kw)
    some, of = at[:7 + 20], keys + 20 * 4            # and the first twenty of the others
    few = dict(q_offsets=_offsets([7] + lq[1:21]), kv_offsets=_offsets(lk[:21]))
    for got, want in zip((dq[some], dk[:of], dv[:of]), ref.attend_grad(q[some], k[:of], v[:of], d_out[some], **few)):
        within(got, *want)
    within(out[some], *ref.attend(q[some], k[:of], v[:of], **few)[0])
    dq[at] = 0
    assert not dq.any()
