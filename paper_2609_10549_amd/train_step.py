"""A training step of a small model through the library's operators: embedding,
layer norm, the fused MLP pair, layer norm, cross entropy over a split
vocabulary, and back.

    python -m paper_2609_10549_amd.train_step [--steps N] [--tokens M] [--hidden K] [--vocab V] [--shards S]

The model is one (linear) MLP layer with a residual between a tied embedding:

    x0 = scale E[ids]                      compass_embed_forward
    x1 = x0 + W2 (W1 norm(x0))             compass_norm_forward, compass_ag_gemm, compass_gemm_rs
    loss = mean xent(norm(x1) E^T, next)   compass_norm_forward, compass_xent_forward, compass_xent_join

with one rank in the tensor-parallel group (its shard is the whole activation;
the residual enters as the incoming fp32 partial sum of the ReduceScatter) and
the vocabulary in `shards` pieces, as that many ranks would hold it. The
gradient of E is written by the cross entropy and added to by the embedding.
The learned task: token t is followed by (a t + b) mod V.
"""
from __future__ import annotations

import argparse
import math


class Model:
    def __init__(self, tokens: int, hidden: int, vocab: int, shards: int, seed: int = 0):
        import torch

        from . import compass as C
        if vocab % shards:
            raise ValueError(f"vocab = {vocab} must split into {shards} shards")
        self.C, self.torch, self.M, self.K, self.V, self.S = C, torch, tokens, hidden, vocab, shards
        self.F = 2 * hidden
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        bf = torch.bfloat16

        def normal(*shape, std=1.0):
            return std * torch.randn(*shape, generator=g, device="cuda")

        # fp32 master weights, bf16 copies for the products
        self.master = {"E": normal(vocab, hidden, std=hidden ** -0.5), "W1": normal(self.F, hidden, std=hidden ** -0.5),
                       "W2": normal(hidden, self.F, std=0.1 * self.F ** -0.5),
                       "g1": torch.ones(hidden, device="cuda"), "b1": torch.zeros(hidden, device="cuda"),
                       "g2": torch.ones(hidden, device="cuda"), "b2": torch.zeros(hidden, device="cuda")}
        self.momentum = {k: torch.zeros_like(v) for k, v in self.master.items()}
        self.bf16 = {k: self.master[k].to(bf) for k in ("E", "W1", "W2")}
        self.scale = math.sqrt(hidden)

        def empty(*shape, dtype=torch.float32):
            return torch.empty(shape, dtype=dtype, device="cuda")

        M, K, V, S = tokens, hidden, vocab, shards
        self.x0, self.h, self.x1, self.y = (empty(M, K, dtype=bf) for _ in range(4))
        self.gathered, self.u = empty(M, K, dtype=bf), empty(M, self.F, dtype=bf)
        self.stats = {k: empty(M) for k in ("mean1", "rstd1", "mean2", "rstd2", "lse", "loss")}
        self.lse_parts, self.tlogit_parts = empty(S, M), empty(S, M)
        self.dy, self.dx1, self.dh, self.dx0 = (empty(M, K, dtype=bf) for _ in range(4))
        self.du = empty(M, self.F, dtype=bf)
        self.grad = {"E": empty(V, K, dtype=bf), "W1": empty(self.F, K, dtype=bf), "W2": empty(K, self.F, dtype=bf),
                     "g1": empty(K), "b1": empty(K), "g2": empty(K), "b2": empty(K)}
        self.residual, self.stage = empty(M, K), empty(M, K)
        need = max(C.compass_xent_workspace(M, V // S, K), C.compass_xent_workspace(M, V // S, K, backward=True),
                   C.compass_norm_workspace(M, K), C.compass_embed_workspace(M, V, K))
        self.ws = torch.empty(need, dtype=torch.uint8, device="cuda")   # one stream: every call may use the same
        self.ag = C.ag_problem([self.h], self.gathered, self.bf16["W1"], self.u, 0, "single")
        self.rs = C.rs_problem(self.u, self.bf16["W2"], [self.residual], self.stage, self.x1, None, 0, "single")

    def shard(self, x, q: int):
        n = self.V // self.S
        return x[q * n:(q + 1) * n]

    def forward(self, ids, target):
        """Losses of the tokens (M, fp32)."""
        C, w, s = self.C, self.master, self.stats
        C.compass_embed_forward(ids, self.bf16["E"], self.x0, scale=self.scale)
        C.compass_norm_forward(self.x0, w["g1"], w["b1"], self.h, s["mean1"], s["rstd1"])
        C.compass_ag_gemm(self.ag)
        self.residual.copy_(self.x0)
        C.compass_gemm_rs(self.rs)
        C.compass_norm_forward(self.x1, w["g2"], w["b2"], self.y, s["mean2"], s["rstd2"])
        n = self.V // self.S
        for q in range(self.S):
            C.compass_xent_forward(self.y, self.shard(self.bf16["E"], q), target, self.lse_parts[q], self.tlogit_parts[q],
                                   None, self.ws, v0=q * n)
        C.compass_xent_join(self.lse_parts, self.tlogit_parts, target, s["lse"], s["loss"])
        return s["loss"]

    def backward(self, ids, target):
        """Gradients of the mean loss over the tokens that have a target."""
        C, torch, w, s, g, b = self.C, self.torch, self.master, self.stats, self.grad, self.bf16
        kept = target >= 0
        weight = kept.float() / kept.sum().clamp(min=1)
        n = self.V // self.S
        total = torch.zeros(self.M, self.K, device="cuda")
        for q in range(self.S):   # every rank's share of dH, summed (over the ranks, by the ReduceScatter)
            C.compass_xent_backward(self.y, self.shard(b["E"], q), target, s["lse"], weight, self.dy,
                                    self.shard(g["E"], q), self.ws, v0=q * n)
            total += self.dy
        self.dy.copy_(total)
        C.compass_norm_backward(self.dy, self.x1, w["g2"], s["mean2"], s["rstd2"], self.dx1, g["g2"], g["b2"], self.ws)
        C.compass_gemm(self.dx1, b["W2"].T.contiguous(), self.du)
        C.compass_gemm(self.dx1.T.contiguous(), self.u.T.contiguous(), g["W2"])
        C.compass_gemm(self.du, b["W1"].T.contiguous(), self.dh)
        C.compass_gemm(self.du.T.contiguous(), self.h.T.contiguous(), g["W1"])
        C.compass_norm_backward(self.dh, self.x0, w["g1"], s["mean1"], s["rstd1"], self.dx0, g["g1"], g["b1"], self.ws)
        self.dx0 += self.dx1
        C.compass_embed_backward(ids, self.dx0, g["E"], self.ws, scale=self.scale, accumulate=True)
        return g

    def step(self, ids, target, lr: float):
        """One update; the mean loss before it, on the GPU."""
        loss = self.forward(ids, target).sum() / (target >= 0).sum().clamp(min=1)
        for k, d in self.backward(ids, target).items():
            self.momentum[k].mul_(0.9).add_(d.float())
            self.master[k].sub_(lr * self.momentum[k])
        for k, v in self.bf16.items():
            v.copy_(self.master[k])
        return loss


def batch(model: Model, seed: int):
    """Random tokens, each with its successor as the target; one in 16 has none."""
    torch = model.torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    ids = torch.randint(0, model.V, (model.M,), generator=g, device="cuda")
    target = (5 * ids + 17) % model.V
    return ids, torch.where(torch.arange(model.M, device="cuda") % 16 == 5, -100, target)


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--tokens", type=int, default=2048)
    ap.add_argument("--hidden", type=int, default=256)
    ap.add_argument("--vocab", type=int, default=1000)
    ap.add_argument("--shards", type=int, default=2)
    ap.add_argument("--lr", type=float, default=0.2)
    a = ap.parse_args()
    model = Model(a.tokens, a.hidden, a.vocab, a.shards)
    for i in range(a.steps):
        loss = model.step(*batch(model, i), a.lr)
        if i % 10 == 0 or i + 1 == a.steps:
            print(f"step {i:4d}  loss {float(loss):.4f}", flush=True)


if __name__ == "__main__":
    main()
