"""A predicate encoder on the library's layers: clause tokens -> w_z.

The method takes the filter weights' vector w_z (w_f = softplus(w_z)) from a
learned encoder of the predicate whose architecture the paper does not give.
This one is an example of the layers in ``ifvs.Layers`` at work, forward and
backward, and a stand-in that can be trained: a conjunction is a set of
clauses, so its tokens (column, operator, bounds, each with the clause's column)
pass through gated feed-forward blocks and are averaged:

    x_0 = sqrt(D) table[ids]                                     embed
    n_0 = w_pre * x_0 / rms(x_0)                                 norm_join
    y_l = ffn_l(n_l)                                             ffn
    x_{l+1} = rho x_l + gate_l * w_post * y_l / rms(y_l),
    n_{l+1} = w_pre * x_{l+1} / rms(x_{l+1})                     norm_join
    w_z = ln(e - 1) + head * mean over the tokens of n_L

gate_l = 1 + G_l c conditions each block on a vector c of the predicate's query
(G starts at zero, head at a small constant: w_f starts near the method's
initial 1).  Torch holds the memory and the two products with c; parameters are
float32, the layers run in bfloat16.

``python -m paper_2607_22922_gb300.encoder`` trains one on a small synthetic
index (dL/dw_z from ``ifvs_train_grad``) and searches with its w_z.
"""
from __future__ import annotations

import math

import numpy as np
import torch

from . import ifvs

N_OPS = 6
WZ_IDENTITY = math.log(math.e - 1)     # softplus of it is 1


class PredicateEncoder:
    """spans: (lo, hi) of every attribute column's values, for the bounds'
    buckets; D: the index's dimension."""

    def __init__(self, spans, D, hidden, blocks=2, buckets=64, rho=0.7071, eps=1e-5, seed=0, device=0):
        self.spans, self.D, self.buckets, self.rho, self.eps = list(spans), D, buckets, rho, eps
        self.layers = ifvs.Layers(device)
        self.device = torch.device("cuda", device)
        g = torch.Generator(device=self.device)
        g.manual_seed(seed)

        def normal(*shape):
            return torch.randn(*shape, generator=g, device=self.device)

        # token 0 begins a predicate; then per column: operators, lower and upper bounds' buckets
        self.V = 1 + len(self.spans) * (N_OPS + 2 * buckets)
        ones = lambda: torch.ones(D, device=self.device)  # noqa: E731
        self.params = {"table": normal(self.V, D) / math.sqrt(D), "pre_0": ones(),
                       "head": 0.1 * ones()}
        self.blocks = blocks
        for i in range(blocks):
            self.params.update({"in_%d" % i: normal(2 * hidden, D) / math.sqrt(D),
                                "out_%d" % i: normal(D, hidden) / math.sqrt(hidden),
                                "post_%d" % i: ones(), "pre_%d" % (i + 1): ones(),
                                "ctx_%d" % i: torch.zeros(D, D, device=self.device)})

    def tokens(self, preds):
        """ids int32 [T], offsets int64 [B + 1]: the tokens of every predicate's
        clauses (ifvs_predicate records)."""
        n = preds["n_clauses"].astype(np.int64)
        c = preds["c"]
        per_col = N_OPS + 2 * self.buckets
        lo, hi = (np.array([s[k] for s in self.spans], np.float64) for k in (0, 1))
        col, op = c["col"].astype(np.int64) % len(self.spans), c["op"].astype(np.int64)

        def bucket(v):
            x = (v.astype(np.float64) - lo[col]) / np.maximum(hi[col] - lo[col], 1.0)
            return np.clip((x * self.buckets).astype(np.int64), 0, self.buckets - 1)

        base = 1 + col * per_col
        three = np.stack([base + op, base + N_OPS + bucket(c["lo"]),
                          np.where(op == ifvs.IFVS_OP_RANGE, base + N_OPS + self.buckets + bucket(c["hi"]), -1)], -1)
        used = (np.arange(c.shape[1])[None, :, None] < n[:, None, None]) & (three >= 0)
        ids = np.concatenate([np.zeros((len(n), 1), np.int64), np.where(used, three, -1).reshape(len(n), -1)], 1)
        lengths = (ids >= 0).sum(1)
        return ids[ids >= 0].astype(np.int32), np.concatenate([[0], np.cumsum(lengths)]).astype(np.int64)

    def forward(self, preds, context=None):
        """w_z [B][D] float32; context [B][D] float32 or None.  Keeps what backward needs."""
        L, stream = self.layers, torch.cuda.current_stream(self.device)
        ids, offsets = self.tokens(preds)
        B = len(offsets) - 1
        seq = np.repeat(np.arange(B, dtype=np.int32), np.diff(offsets))
        s = {"ids": torch.from_numpy(ids).to(self.device), "offsets": torch.from_numpy(offsets).to(self.device),
             "seq": torch.from_numpy(seq).to(self.device), "context": context,
             "w": {k: v.bfloat16() for k, v in self.params.items()}}
        w = s["w"]
        s["lengths"] = (s["offsets"][1:] - s["offsets"][:-1]).float()[:, None]
        x = L.embed(w["table"], s["ids"], math.sqrt(self.D), stream=stream)
        _, n = L.norm_join(x, w_pre=w["pre_0"], eps=self.eps, stream=stream)
        s["x"], s["n"], s["y"], s["gate"] = [x], [n], [], []
        for i in range(self.blocks):
            y = L.ffn(n, w["in_%d" % i], w["out_%d" % i], stream=stream)
            gate = torch.ones(B, self.D, device=self.device)
            if context is not None:
                gate += context @ self.params["ctx_%d" % i].t()
            gate = gate.bfloat16()
            x, n = L.norm_join(x, y, gate, w["post_%d" % i], w["pre_%d" % (i + 1)], offsets=s["offsets"],
                               res_scale=self.rho, eps=self.eps, stream=stream)
            for k, v in zip(("x", "n", "y", "gate"), (x, n, y, gate)):
                s[k].append(v)
        # the sum over a predicate's tokens is the embedding's gradient by their predicate
        s["mean"] = L.embed_grad(n, s["seq"], V=B, stream=stream).float() / s["lengths"]
        self.saved = s
        return WZ_IDENTITY + self.params["head"] * s["mean"]

    def backward(self, d_wz):
        """Gradients of the parameters of the last forward call from dL/dw_z [B][D]."""
        L, stream, s = self.layers, torch.cuda.current_stream(self.device), self.saved
        w, g = s["w"], {"head": (d_wz * s["mean"]).sum(0)}
        d_mean = (d_wz * self.params["head"] / s["lengths"]).bfloat16()
        dn, dx = L.embed(d_mean, s["seq"], stream=stream), None
        for i in reversed(range(self.blocks)):
            dx, dy, d_gate, g["post_%d" % i], g["pre_%d" % (i + 1)] = L.norm_join_grad(
                s["x"][i + 1], s["y"][i], s["gate"][i], w["post_%d" % i], w["pre_%d" % (i + 1)], d_x_out=dx, d_n=dn,
                offsets=s["offsets"], res_scale=self.rho, eps=self.eps, stream=stream)
            if s["context"] is not None:
                g["ctx_%d" % i] = d_gate.float().t() @ s["context"]
            dn, g["in_%d" % i], g["out_%d" % i] = L.ffn_grad(s["n"][i], w["in_%d" % i], w["out_%d" % i], dy,
                                                             stream=stream)
        dx, _, _, _, g["pre_0"] = L.norm_join_grad(s["x"][0], w_pre=w["pre_0"], d_x_out=dx, d_n=dn, eps=self.eps,
                                                   stream=stream)
        g["table"] = L.embed_grad(dx, s["ids"], math.sqrt(self.D), V=self.V, stream=stream)
        return {k: v.float() for k, v in g.items()}

    def step(self, grads, lr):
        for k, v in grads.items():
            self.params[k] -= lr * v

    def close(self):
        self.layers.status()
        self.layers.close()


def main():
    from . import synth
    w = synth.scaled(synth.WORKLOADS["gmm10k-d128-m16"], N=10_000)
    ix = synth.pq_space_index(w)
    cond = synth.make_conditioning(ix)
    index = ifvs.Index(ix.codes, ix.attrs, vectors=synth.raw_vectors(ix), D=w.D, K=w.K)
    index.load_codebooks(ix.codebook, bank=cond.bank, W=cond.W, hash_seeds=cond.seeds)
    enc = PredicateEncoder([(a.lo, a.hi) for a in w.attrs], w.D, hidden=256)
    # mini-batches of queries under one predicate: its w_z is theirs
    batches, n_pos, n_neg = [], 10, 32
    for i in range(8):
        qs = synth.make_queries(ix, 0.1, nq=16, salt=i)
        preds = np.repeat(qs.preds[:1], 16)
        near, _, _ = index.search(qs.q, preds, 128, rerank=128)      # exact distances: positives first
        batches.append((qs.q, preds, near[:, :n_pos + n_neg].copy()))
    for epoch in range(5):
        total = 0.0
        for q, preds, cand in batches:
            context = torch.from_numpy(q.mean(0, keepdims=True)).cuda()
            wz = enc.forward(preds[:1], context)
            loss, _, _, g_wz = index.train_grad(q, preds, wz[0].cpu().numpy(), cand, n_pos, 8.0, 0.0)
            enc.step(enc.backward(torch.from_numpy(g_wz).cuda()[None]), 0.01)
            total += loss / len(batches)
        print("epoch %d: mean loss %.4f" % (epoch, total))
    qs = synth.make_queries(ix, 0.1, nq=64, salt=99)
    wz = enc.forward(qs.preds, torch.from_numpy(qs.q).cuda())
    ids, dists, passing = index.search(qs.q, qs.preds, w.k, wz=wz.cpu().numpy())
    print("searched %d queries: %d of %d places filled, first distance %.3f" % (
        len(ids), int((ids >= 0).sum()), ids.size, float(dists[0, 0])))
    enc.close()
    index.close()


if __name__ == "__main__":
    main()
