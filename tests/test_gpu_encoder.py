"""The predicate encoder (paper_2607_22922_gb300/encoder.py) as a whole, against
the same network in float64 with gradients by differentiation, and with the
index it serves.

Tolerance.  A block rounds to bfloat16 (relative 2^-8) its normed input, hidden
values, output and residual, the gates and the weights: eight roundings, the
embedding and the mean three more.  The norms keep relative errors, the
projections of random weights keep them on average and at most double them: by
row norm w_z is within 2 (8 blocks + 3) 2^-8 of its spread, a gradient, which
passes the same places twice, within twice that."""
import math

import numpy as np
import pytest

from paper_2607_22922_gb300 import synth
from parity_util import check_topk

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
BLOCKS = 2
TOL = 2 * (8 * BLOCKS + 3) * 2.0 ** -8


@pytest.fixture(scope="module")
def env():
    from paper_2607_22922_gb300 import build
    build.build()
    from paper_2607_22922_gb300 import encoder, ifvs
    return ifvs, encoder


def _predicates(n, seed):
    rng = np.random.default_rng(seed)
    p = synth.empty_predicates(n)
    for i in range(n):
        k = int(rng.integers(0, 5))          # none to four clauses
        p[i]["n_clauses"] = k
        for j in range(k):
            lo = int(rng.integers(0, 900))
            synth.set_clause(p[i], j, int(rng.integers(0, 2)), int(rng.integers(0, 6)), lo, lo + 50)
    return p


def _plain(enc, params, preds, context):
    ids, offsets = enc.tokens(preds)
    ids, seq = torch.from_numpy(ids).long().cuda(), torch.from_numpy(np.repeat(np.arange(len(preds)), np.diff(offsets))).cuda()

    def norm(v):
        return v / torch.sqrt((v * v).mean(1, keepdim=True) + enc.eps)

    x = params["table"][ids] * math.sqrt(enc.D)
    n = params["pre_0"] * norm(x)
    for i in range(enc.blocks):
        g, u = (n @ params["in_%d" % i].t()).chunk(2, 1)
        y = (g * torch.sigmoid(g) * u) @ params["out_%d" % i].t()
        gate = 1 + context @ params["ctx_%d" % i].t()
        x = enc.rho * x + gate[seq] * params["post_%d" % i] * norm(y)
        n = params["pre_%d" % (i + 1)] * norm(x)
    counts = torch.bincount(seq, minlength=len(preds))[:, None]
    mean = torch.zeros(len(preds), enc.D, dtype=torch.float64, device="cuda").index_add(0, seq, n) / counts
    return math.log(math.e - 1) + params["head"] * mean


def test_tokens(env):
    ifvs, encoder = env
    enc = encoder.PredicateEncoder([(0, 1000), (0, 1000)], 64, 64, blocks=1, buckets=10)
    p = synth.empty_predicates(3)
    p["n_clauses"] = [0, 1, 2]
    synth.set_clause(p[1], 0, 1, synth.OP_EQ, 999)
    synth.set_clause(p[2], 0, 0, synth.OP_RANGE, 100, 350)
    synth.set_clause(p[2], 1, 1, synth.OP_LE, -5)
    ids, offsets = enc.tokens(p)
    per = 6 + 20                         # tokens of a column: operators, lower, upper bounds
    assert offsets.tolist() == [0, 1, 4, 10]
    assert ids.tolist() == [0,
                            0, 1 + per, 1 + per + 6 + 9,
                            0, 1 + 1, 1 + 6 + 1, 1 + 16 + 3, 1 + per + 5, 1 + per + 6]
    enc.close()


def test_encoder_against_float64(env):
    ifvs, encoder = env
    enc = encoder.PredicateEncoder([(0, 1000), (0, 1000)], 96, 200, blocks=BLOCKS, seed=3)
    preds = _predicates(300, 4)
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    for k in ("ctx_0", "ctx_1"):
        enc.params[k] = 0.02 * torch.randn(96, 96, generator=g, device="cuda")
    context, d_wz = (torch.randn(300, 96, generator=g, device="cuda") for _ in range(2))
    wz = enc.forward(preds, context)
    grads = enc.backward(d_wz)
    enc.layers.status()
    p = {k: v.double().requires_grad_() for k, v in enc.params.items()}
    want = _plain(enc, p, preds, context.double())
    spread = (want - math.log(math.e - 1)).norm()
    assert float((wz.double() - want.detach()).norm() / spread.detach()) <= TOL
    want.backward(d_wz.double())
    assert set(grads) == set(p)
    for k, v in grads.items():
        assert float((v.double() - p[k].grad).norm() / p[k].grad.norm()) <= 2 * TOL, k
    enc.close()


def test_training_lowers_the_loss_and_search_takes_the_vectors(env, orc):
    ifvs, encoder = env
    w = synth.scaled(synth.WORKLOADS["gmm10k-d128-m16"], N=4000)
    ix = synth.pq_space_index(w)
    cond = synth.make_conditioning(ix)
    index = ifvs.Index(ix.codes, ix.attrs, D=w.D, K=w.K)
    index.load_codebooks(ix.codebook, bank=cond.bank, W=cond.W, hash_seeds=cond.seeds)
    enc = encoder.PredicateEncoder([(a.lo, a.hi) for a in w.attrs], w.D, hidden=128, seed=1)
    qs = synth.make_queries(ix, 0.2, nq=16)
    preds = np.repeat(qs.preds[:1], 16)
    X, n_pos = synth.raw_vectors(ix), 8
    cand = np.empty((16, 32), np.int64)
    for i in range(16):
        bm, _ = orc.filter_bitmap(ix.attrs, preds[i])
        cand[i], _ = orc.exact_topk(X, qs.q[i], bm, 32)
    context = torch.from_numpy(qs.q.mean(0, keepdims=True)).cuda()
    losses = []
    for _ in range(12):
        wz = enc.forward(preds[:1], context)
        loss, _, _, g_wz = index.train_grad(qs.q, preds, wz[0].cpu().numpy(), cand, n_pos, 8.0, 0.0)
        losses.append(loss)
        enc.step(enc.backward(torch.from_numpy(g_wz).cuda()[None]), 0.01)
    assert losses[-1] < losses[0]
    # each query's own vector, through the search path
    wz = enc.forward(qs.preds, torch.from_numpy(qs.q).cuda()).cpu().numpy()
    ids, d, _ = index.search(qs.q, qs.preds, 10, wz=wz)
    oi, od, _, st = orc.search(ix.codes, ix.attrs, ix.codebook, qs.q, qs.preds, 10, bank=cond.bank, W=cond.W,
                               seeds=cond.seeds, wz=wz, want_stages=True)
    for i in range(16):
        bm, _ = orc.filter_bitmap(ix.attrs, qs.preds[i])
        passing = np.unpackbits(bm.view(np.uint8), bitorder="little")[:w.N].astype(bool)
        check_topk(ids[i], d[i], oi[i], od[i], orc.adc_all(st["lut"][i], ix.codes), passing)
    enc.close()
    index.close()
