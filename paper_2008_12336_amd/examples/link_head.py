"""A link predictor on an embedding, trained with 8-bit activations: embeds a synthetic graph, trains a small head on
products of the rows of vertex pairs, and says how well it tells held-out edges from pairs that are none.

    python -m paper_2008_12336_amd.examples.link_head [--scale 14] [--dim 64] [--steps 200] [--bits 32]

The head is layer norm (rows of hubs are orders of magnitude longer than others), a linear layer with GELU to four
times the width, one back with the features added, and one to a single logit.  Between the passes it keeps the normalised
rows, the layers' inputs and the pre-activations in 8 bits, a byte an entry, of which the backward calls read them.  The
optimiser keeps its moments in 32 bits, or in 8 with --bits 8, and writes the weights' 16-bit copies, which the layers read.  torch
holds the parameters and takes the loss; every operator of the head and its optimiser is one of the library's kernels."""
from __future__ import annotations

import argparse

import torch

import graphgen
import paper_2008_12336_amd as G

DEV = "cuda"


class LinkHead:
    """Parameters in 32 bits, activations in `dtype`; buffers for batches of `rows` pairs are made once."""

    def __init__(self, dim: int, rows: int, dtype=torch.bfloat16, seed: int = 0):
        g = torch.Generator(device=DEV).manual_seed(seed)
        wide = 4 * dim
        init = lambda n, k: torch.randn(n, k, generator=g, device=DEV) / k ** 0.5  # noqa: E731
        zeros = lambda *s: torch.zeros(*s, device=DEV)  # noqa: E731
        self.dtype, self.rows = dtype, rows
        self.params = dict(gamma=torch.ones(dim, device=DEV), beta=zeros(dim), w1=init(wide, dim), b1=zeros(wide),
                           w2=0.1 * init(dim, wide), b2=zeros(dim), w3=init(1, dim), b3=zeros(1))
        self.grads = {name: torch.empty_like(p) for name, p in self.params.items()}
        self.copies = self.weights()  # of float32: the parameters themselves
        act = lambda n: torch.empty(rows, n, dtype=dtype, device=DEV)  # noqa: E731
        eight = lambda n: G.Packed8(rows, n, dtype, DEV)  # noqa: E731
        self.h, self.a, self.o, self.s = act(dim), act(wide), act(dim), act(1)
        self.dh, self.da, self.do = act(dim), act(wide), act(dim)
        self.rstd = torch.empty(rows, device=DEV)
        self.xhat8, self.h8, self.z8, self.a8 = eight(dim), eight(dim), eight(wide), eight(wide)

    def weights(self) -> dict:
        """The weights as the layers read them, from the parameters as they are."""
        return {name: self.params[name].to(self.dtype) for name in ("w1", "w2", "w3")}

    def optimiser(self, bits: int = 32):
        """AdamW over all parameters, moments in 32 or 8 bits, which keeps the copies up to date from here on: with every step it
        takes."""
        names = list(self.params)
        for name, w in self.weights().items():
            self.copies[name].copy_(w)
        copies = None if self.dtype == torch.float32 else [self.copies.get(n) for n in names]
        return G.gosh_adamw_create([self.params[n] for n in names], [self.grads[n] for n in names], bits=bits, copies=copies)

    def forward(self, x: torch.Tensor, w: dict) -> torch.Tensor:
        """The logits of `rows` pairs' features."""
        p = self.params
        G.gosh_layer_norm(x, p["gamma"], p["beta"], self.h, rstd=self.rstd, xhat8=self.xhat8, y8=self.h8)
        G.gosh_linear(self.h, w["w1"], self.a, bias=p["b1"], act=G.GOSH_ACT_GELU, z=self.z8, y8=self.a8)
        G.gosh_linear(self.a, w["w2"], self.o, bias=p["b2"], residual=x)
        G.gosh_linear(self.o, w["w3"], self.s, bias=p["b3"])
        return self.s[:, 0]

    def backward(self, ds: torch.Tensor, w: dict) -> dict:
        """The parameters' gradients from that of the logits, out of the 8-bit forms."""
        p, g = self.params, self.grads
        G.gosh_linear_backward(ds[:, None], self.o, w["w3"], None, dx=self.do, dw=g["w3"], db=g["b3"])
        G.gosh_linear_backward(self.do, self.a8, w["w2"], None, dx=self.da, dw=g["w2"], db=g["b2"])
        G.gosh_linear_backward(self.da, self.h8, w["w1"], self.z8, G.GOSH_ACT_GELU, dx=self.dh, dw=g["w1"], db=g["b1"])
        G.gosh_layer_norm_backward(self.dh, self.xhat8, p["gamma"], None, self.rstd, None, dgamma=g["gamma"], dbeta=g["beta"])
        return g

    def score(self, x: torch.Tensor) -> torch.Tensor:
        """Logits of any number of pairs, nothing kept."""
        p, w, n = self.params, self.weights(), x.shape[0]
        new = lambda k: torch.empty(n, k, dtype=self.dtype, device=DEV)  # noqa: E731
        h, a, o, s = new(x.shape[1]), new(4 * x.shape[1]), new(x.shape[1]), new(1)
        G.gosh_layer_norm(x, p["gamma"], p["beta"], h)
        G.gosh_linear(h, w["w1"], a, bias=p["b1"], act=G.GOSH_ACT_GELU)
        G.gosh_linear(a, w["w2"], o, bias=p["b2"], residual=x)
        G.gosh_linear(o, w["w3"], s, bias=p["b3"])
        return s[:, 0].float()


def features(M: torch.Tensor, pairs: torch.Tensor, scale: float, dtype) -> torch.Tensor:
    return (M[pairs[:, 0]] * M[pairs[:, 1]] * scale).to(dtype)


def auc(pos: torch.Tensor, neg: torch.Tensor) -> float:
    """The share of (edge, non-edge) pairs that are ordered rightly, equal scores counted half."""
    order = torch.sort(neg).values
    below = torch.searchsorted(order, pos) + torch.searchsorted(order, pos, right=True)
    return float(below.double().mean() / (2 * neg.numel()))


def train(scale: int = 14, dim: int = 64, steps: int = 200, rows: int = 16384, seed: int = 1, bits: int = 32):
    """(held-out AUC before training, after it, the loss of every step); bits: of the optimiser's moments."""
    n = 1 << scale
    edges = graphgen.rmat(scale, 16 << scale, seed=seed)
    kept, held = (e.long() for e in graphgen.holdout_split(edges, 0.1, seed + 1000))
    csr = graphgen.to_csr(n, kept).to(DEV)
    M = torch.empty(n, dim, dtype=torch.float32, device=DEV)
    h = G.gosh_coarsen_device(n, csr.xadj, csr.adj, threshold=100, min_shrink=0.8)
    G.gosh_embed(h, M, 3, 300, 0.3, 0.035, seed)
    h.free()

    gen = torch.Generator(device=DEV).manual_seed(seed)
    kept, held = kept.to(DEV), held.to(DEV)
    busy = torch.nonzero(csr.xadj.diff() > 0)[:, 0]
    held = held[torch.isin(held, busy).all(dim=1)]
    none = lambda count: busy[torch.randint(busy.numel(), (count, 2), generator=gen, device=DEV)]  # noqa: E731
    unit = 1.0 / float((M[kept[:, 0]] * M[kept[:, 1]]).std())
    head = LinkHead(dim, rows, seed=seed)
    test_pos, test_neg = (features(M, p, unit, head.dtype) for p in (held, none(held.shape[0])))
    before = auc(head.score(test_pos), head.score(test_neg))
    optimiser = head.optimiser(bits)
    target = torch.cat((torch.ones(rows // 2, device=DEV), torch.zeros(rows - rows // 2, device=DEV)))
    losses = []
    for step in range(1, steps + 1):
        some = kept[torch.randint(kept.shape[0], (rows // 2,), generator=gen, device=DEV)]
        x = features(M, torch.cat((some, none(rows - rows // 2))), unit, head.dtype)
        logits = head.forward(x, head.copies).float()
        losses.append(torch.nn.functional.softplus(torch.where(target > 0, -logits, logits)).mean())
        head.backward(((torch.sigmoid(logits) - target) / rows).to(head.dtype), head.copies)
        G.gosh_adamw_step(optimiser, lr=2e-3, step=step)
    return before, auc(head.score(test_pos), head.score(test_neg)), [float(v) for v in losses]


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--scale", type=int, default=14, help="2^scale vertices")
    ap.add_argument("--dim", type=int, default=64)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--bits", type=int, default=32, choices=(8, 32), help="of the optimiser's moments")
    args = ap.parse_args()
    before, after, losses = train(args.scale, args.dim, args.steps, bits=args.bits)
    print(f"held-out AUC {before:.3f} before, {after:.3f} after {args.steps} steps; loss {losses[0]:.3f} -> {losses[-1]:.3f}")
