"""A query encoder on the library's operators: from an upstream embedding to a vector of an index's space and to the
labels to filter by, its training step, and the search with what it says.

    h = x + W2 gelu(W1 norm(x) + b1) + b2;   g = norm(h);   vector = Wv g + bv;   label logits = Wl g + bl

``python -m paper_2506_00812_amd.query_encoder`` trains one on a synthetic table and searches with it.

Everything runs on the current stream; ``train_step`` waits for nothing, ``search`` only for the labels of its
queries, which ``binding.search`` takes from host memory.
"""
from __future__ import annotations

import torch

from . import binding as vf

__all__ = ["QueryEncoder"]


class QueryEncoder:
    """width: of the upstream embedding; dim: of the index's vectors; n_labels: its vocabulary.  dtype: of weights and
    activations; below float32 every weight has a float32 master.  state_bits: of the optimiser's moments (32 or 8).
    absent: ids of labels that no vector carries; they are never predicted (their logits are -inf).

    float16 reaches down to 6e-8, above most entries of the logits' gradient (p / queries: a third of it and more would be lost at 10,000 queries
    and labels).  There the backward pass carries everything times `scale`, a power of two in device memory; the weights' gradients are
    divided by it in float32.  A step whose gradients are not finite is left out (it still counts for the bias corrections) and
    halves the scale, GROWTH_STEPS good ones in a row double it."""

    FIRST_SCALE, GROWTH_STEPS = 1024.0, 500

    def __init__(self, width, dim, n_labels, hidden=None, dtype=torch.bfloat16, state_bits=32, absent=None, seed=0, device="cuda"):
        hidden = hidden or 4 * width
        g = torch.Generator(device=device)
        g.manual_seed(seed)

        def weight(n, k):
            return torch.randn((n, k), generator=g, device=device) * k ** -0.5

        def const(n, value):
            return torch.full((n,), value, device=device)

        start = dict(n1w=const(width, 1.0), n1b=const(width, 0.0), w1=weight(hidden, width), b1=const(hidden, 0.0),
                     w2=weight(width, hidden), b2=const(width, 0.0), n2w=const(width, 1.0), n2b=const(width, 0.0),
                     wv=weight(dim, width), bv=const(dim, 0.0), wl=weight(n_labels, width), bl=const(n_labels, 0.0))
        gone = torch.as_tensor(() if absent is None else absent, device=device)
        if gone.numel():     # (an empty list makes a tensor of floats, which is no index)
            start["bl"][gone] = -torch.inf
        self.params = {k: v.to(dtype) for k, v in start.items()}
        self.names = list(start)
        self._masters = [start[k] for k in self.names] if dtype != torch.float32 else None
        state = [vf.adamw_state(p, state_bits) for p in self.params.values()]
        self._m, self._v = [s[0] for s in state], [s[1] for s in state]
        self._ms, self._vs = ([s[2] for s in state], [s[3] for s in state]) if state_bits == 8 else (None, None)
        # no decay for biases and norms
        self._decayed = [k.startswith("w") for k in self.names]
        self.dtype, self.steps = dtype, 0
        self.scale = torch.full((1,), self.FIRST_SCALE, device=device) if dtype == torch.float16 else None
        self._good = torch.zeros(1, dtype=torch.int32, device=device)     # steps since the scale changed

    # ------------------------------------------------------------------ forward and backward

    def _body(self, x, save=False):
        p = self.params
        if not save:
            h = vf.linear(vf.layer_norm(x, p["n1w"], p["n1b"]), p["w1"], p["b1"], activation="gelu")
            return vf.layer_norm(vf.linear(h, p["w2"], p["b2"], residual=x), p["n2w"], p["n2b"])
        a, mean1, rstd1 = vf.layer_norm(x, p["n1w"], p["n1b"], save=True)
        h, z = vf.linear(a, p["w1"], p["b1"], activation="gelu", save=True)
        r = vf.linear(h, p["w2"], p["b2"], residual=x)
        g, mean2, rstd2 = vf.layer_norm(r, p["n2w"], p["n2b"], save=True)
        return g, (x, a, mean1, rstd1, h, z, r, mean2, rstd2)

    def encode(self, x, top=1):
        """(vectors [m, dim], label ids int32 [m, top], their log probabilities, entropy [m]) of embeddings x [m, width]."""
        p = self.params
        g = self._body(x)
        vectors = vf.linear(g, p["wv"], p["bv"])
        _, entropy, _, *labels = vf.log_probs(vf.linear(g, p["wl"], p["bl"]), top=top)
        ids, logp = labels or (entropy.new_empty((len(x), 0), dtype=torch.int32), entropy.new_empty((len(x), 0)))     # (none were asked for)
        return vectors, ids, logp, entropy

    def gradients(self, x, vectors, labels, label_weight=1.0, entropy_weight=0.0):
        """(loss, {name: gradient}) of mean |vector - target|^2 - label_weight mean log p(label) - entropy_weight mean
        entropy.  vectors [m, dim]; labels int32 [m], -1 for a query without one.  Of no queries at all everything is 0.  Gradients
        are of the encoder's dtype, for float16 in float32."""
        return self._gradients(x, vectors, labels, label_weight, entropy_weight)[:2]

    def _gradients(self, x, vectors, labels, label_weight=1.0, entropy_weight=0.0):
        """The same, and for float16 the one tensor that holds all gradients."""
        p, m = self.params, max(x.shape[0], 1)
        g, (x, a, mean1, rstd1, h, z, r, mean2, rstd2) = self._body(x, save=True)
        out = vf.linear(g, p["wv"], p["bv"])
        logits = vf.linear(g, p["wl"], p["bl"])
        logp, entropy, lse = vf.log_probs(logits, labels)
        off = out.float() - vectors.float()
        loss = off.square().sum(1).mean() - label_weight * logp.mean() - entropy_weight * entropy.mean() if len(x) else off.sum()
        grads = {}
        d_logp = torch.full_like(logp, -label_weight / m)
        d_entropy = torch.full_like(entropy, -entropy_weight / m) if entropy_weight else None
        d_out = off * (2.0 / m)
        if self.scale is not None:
            for d in (d_logp, d_out) + ((d_entropy,) if entropy_weight else ()):
                d.mul_(self.scale)
        d_logits = vf.log_probs_backward(logits, lse, labels, d_logp, entropy=entropy if entropy_weight else None,
                                         d_entropy=d_entropy, out=logits)
        dg, grads["wl"], grads["bl"] = vf.linear_backward(d_logits, g, p["wl"])
        dg2, grads["wv"], grads["bv"] = vf.linear_backward(d_out.to(self.dtype), g, p["wv"])
        dr, grads["n2w"], grads["n2b"] = vf.layer_norm_backward(dg.add_(dg2), r, mean2, rstd2, p["n2w"])
        dh, grads["w2"], grads["b2"] = vf.linear_backward(dr, h, p["w2"])
        da, grads["w1"], grads["b1"] = vf.linear_backward(dh, a, p["w1"], z=z, activation="gelu")
        # x is an input: only the weights' gradients are wanted of its norm
        _, grads["n1w"], grads["n1b"] = vf.layer_norm_backward(da, x, mean1, rstd1, p["n1w"], dx=False)
        if self.scale is None:
            return loss, grads, None
        flat = torch.cat([t.flatten() for t in grads.values()]).float().div_(self.scale)
        parts = flat.split([t.numel() for t in grads.values()])
        return loss, {k: part.view_as(t) for (k, t), part in zip(grads.items(), parts)}, flat

    def _adapt_scale(self, flat):
        """int32 [1]: whether a gradient is not finite; moves the scale.  Nothing waits for the device."""
        bad = ~torch.isfinite(flat).all().reshape(1)
        self._good.add_(1).masked_fill_(bad, 0)
        grow = self._good >= self.GROWTH_STEPS
        self._good.masked_fill_(grow, 0)
        self.scale.mul_(torch.where(bad, 0.5, torch.where(grow, 2.0, 1.0))).clamp_(1.0, 2.0 ** 24)
        return bad.int()

    def train_step(self, x, vectors, labels, lr=1e-3, weight_decay=0.01, **weights):
        """One step of AdamW on the loss of `gradients`; returns the loss (a CUDA tensor)."""
        loss, grads, flat = self._gradients(x, vectors, labels, **weights)
        self.steps += 1
        skip = None if flat is None else self._adapt_scale(flat)
        vf.adamw_step([self.params[k] for k in self.names], [grads[k] for k in self.names], self._m, self._v, step=self.steps,
                      lr=lr, weight_decay=[weight_decay if d else 0.0 for d in self._decayed], masters=self._masters,
                      m_scales=self._ms, v_scales=self._vs, skip=skip)
        return loss

    # ------------------------------------------------------------------ search

    def search(self, index, x, k, **params):
        """(ids, distances, labels): the k nearest vectors that carry each query's most probable label.  `index`: a
        binding.Index of float32 vectors; `params` as in binding.search."""
        vectors, labels, _, _ = self.encode(x, top=1)
        host = labels[:, 0].cpu().numpy()
        ids, dists = vf.search(index, vectors.float(), range(len(host) + 1), host, k, **params)
        return ids, dists, labels[:, 0]


def _demo(n=20_000, steps=200, batch=512, width=256):
    from .workloads import make_workload
    w = make_workload("c2", n=n, n_labels=100, T=500, n_clusters=64, nq=1000)
    s = w.spec
    X = torch.from_numpy(w.vectors).cuda()
    index = vf.build_index(X, w.label_offsets, w.label_ids, s.n_labels, s.T, s.graph_degree)
    # a stand-in for an upstream model: a fixed random map of the vector, plus a direction for the label
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    lift = torch.randn((s.dim, width), generator=g, device="cuda") * s.dim ** -0.5
    mark = torch.randn((s.n_labels, width), generator=g, device="cuda")

    def embed(v, labels):
        return (v @ lift + mark[labels.long()]).bfloat16()

    sizes = torch.from_numpy(index.export("S"))
    enc = QueryEncoder(width, s.dim, s.n_labels, state_bits=8, absent=torch.nonzero(sizes == 0)[:, 0])
    first = torch.from_numpy(w.label_ids[w.label_offsets[:-1]]).cuda()
    for t in range(steps):
        at = torch.randint(0, n, (batch,), generator=g, device="cuda")
        loss = enc.train_step(embed(X[at], first[at]), X[at], first[at], lr=2e-3)
        if t % 50 == 0 or t == steps - 1:
            print(f"step {t}: loss {loss.item():.2f}", flush=True)
    Q = torch.from_numpy(w.queries).cuda()
    asked = torch.from_numpy(w.qlabel_ids).cuda()
    ids, _, labels = enc.search(index, embed(Q, asked), 10, itopk=32, width=1, iters=8, n_seeds=2048)
    want, _ = vf.search_exact(index, Q, w.qlabel_offsets, w.qlabel_ids, 10)
    hit = (ids[:, :, None] == want[:, None, :]).any(2) & (ids >= 0)
    print(f"labels predicted: {(labels == asked).float().mean().item():.3f}; of the 10 nearest with the true vector and label "
          f"found: {hit.float().sum().item() / (want >= 0).float().sum().item():.3f}")


if __name__ == "__main__":
    _demo()
