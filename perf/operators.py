"""The language-model operators whose speed is measured: the two ends of a
model around the fused tensor-parallel MLP, and the layer norms between.

  xent_fwd   softmax cross entropy of one rank's share of the vocabulary from
             hidden states and output weight: per row the log-sum-exp, the
             target's logit and the loss
  xent_bwd   its gradients for the hidden states and the weight
  norm_fwd   layer norm with its row statistics
  norm_bwd   its gradients: input, weight and bias
  embed_fwd  embedding lookup with a scale
  embed_bwd  the table's gradient

Rows are tokens of one tensor-parallel rank. Hidden states are bf16 (layer
norm and embedding: bf16 or fp32); statistics, losses and the gradients of the
norm's parameters are fp32. Targets below zero carry no loss; ids outside the
table look up zeros.
"""
from __future__ import annotations

import math

import torch

own = False   # True: the framework's kernels, False: the plain form

EPS = 1e-5


def _xent(name, kind, M, V, K):
    return {"name": name, "kind": kind, "M": M, "V": V, "K": K}


def _norm(name, kind, M, N, dtype):
    return {"name": name, "kind": kind, "M": M, "N": N, "dtype": dtype}


def _embed(name, kind, T, V, K, dtype, v0=0):
    return {"name": name, "kind": kind, "T": T, "V": V, "K": K, "dtype": dtype, "v0": v0}


def listed():
    return [
        # scoring the last tokens of eight prompts: the weight is read for a few rows
        _xent("xent_fwd_few_tokens", "xent_fwd", 8, 32000, 4096),
        # one of eight ranks' share of a 50 k vocabulary at the largest hidden size
        _xent("xent_fwd_shard", "xent_fwd", 8192, 6283, 12288),
        # a short batch, no dimension a multiple of a tile
        _xent("xent_bwd_ragged", "xent_bwd", 777, 10007, 1544),
        # a step's whole vocabulary on one rank: the largest call
        _xent("xent_bwd_vocab", "xent_bwd", 8192, 50257, 4096),
        # four single tokens of a serving step at the largest hidden size
        _norm("norm_fwd_tokens", "norm_fwd", 4, 12288, "bf16"),
        # a long batch's activations
        _norm("norm_fwd_batch", "norm_fwd", 32768, 8192, "bf16"),
        # an odd row length, fp32 residual stream
        _norm("norm_bwd_odd_f32", "norm_bwd", 1000, 4097, "f32"),
        # the norm before the largest MLP pair
        _norm("norm_bwd_batch", "norm_bwd", 8192, 12288, "bf16"),
        # single tokens of a serving step, one rank's share of the table
        _embed("embed_fwd_tokens", "embed_fwd", 16, 6283, 4096, "bf16", 6283),
        # a long batch from the whole table
        _embed("embed_fwd_batch", "embed_fwd", 32768, 50257, 4096, "bf16"),
        # a short batch into one rank's share, odd row length, fp32
        _embed("embed_bwd_short_f32", "embed_bwd", 500, 6283, 1031, "f32"),
        # a long batch into the whole table
        _embed("embed_bwd_batch", "embed_bwd", 32768, 50257, 4096, "bf16"),
    ]


_XENT_FLOPS_MAX = 6.0 * 8192 * 50257 * 4096      # the largest listed call
_ROW_BYTES_MAX = 1.2e9                           # the largest norm and embedding


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _int(rng, lo, hi):
    return int(round(_log(rng, lo, hi)))


def draw(rng):
    kind = rng.choice(("xent_fwd", "xent_fwd", "xent_bwd", "xent_bwd", "norm_fwd", "norm_bwd", "embed_fwd", "embed_bwd"))
    while True:
        if kind.startswith("xent"):
            c = {"kind": kind, "M": _int(rng, 1, 8192), "V": _int(rng, 1000, 131072), "K": 8 * _int(rng, 64, 1536)}
            if work(c)["flops"] <= _XENT_FLOPS_MAX and c["V"] * c["K"] * 2 <= _ROW_BYTES_MAX:
                return c
        elif kind.startswith("norm"):
            c = {"kind": kind, "M": _int(rng, 1, 32768), "N": _int(rng, 64, 16384), "dtype": rng.choice(("bf16", "f32"))}
            if rng.random() < 0.5:
                c["N"] = max(64, c["N"] // 64 * 64)
            if work(c)["bytes"] <= _ROW_BYTES_MAX and c["N"] != 3072:
                return c
        else:
            c = {"kind": kind, "T": _int(rng, 1, 65536), "V": _int(rng, 1000, 131072), "K": _int(rng, 64, 12288),
                 "dtype": rng.choice(("bf16", "f32")), "v0": 0}
            if rng.random() < 0.5:
                c["K"] = max(64, c["K"] // 64 * 64)
            if rng.random() < 0.3:
                c["v0"] = c["V"]
            if c["T"] * c["K"] * 4 <= _ROW_BYTES_MAX and c["V"] * c["K"] * 4 <= _ROW_BYTES_MAX and c["K"] != 3072:
                return c


def _type(case):
    return torch.bfloat16 if case.get("dtype", "bf16") == "bf16" else torch.float32


def _seeded(case, seed):
    """The inputs alone, from the seed."""
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed))

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=dev)

    def uniform(*shape):
        return torch.rand(*shape, generator=g, device=dev)

    kind, dt = case["kind"], _type(case)
    if kind.startswith("xent"):
        M, V, K = case["M"], case["V"], case["K"]
        W = (0.02 * normal(V, K)).to(torch.bfloat16)
        target = (uniform(M) * V).long().clamp_(max=V - 1)
        # normalised hidden states that lean to their target, some rows more
        # than others: its logit rises by 0 to 8
        lean = 8.0 * uniform(M, 1) / (4e-4 * K)
        H = (normal(M, K) + lean * W[target].float()).to(torch.bfloat16)
        # prompt and padding tokens carry no loss
        target = torch.where(uniform(M) < 0.06, torch.full_like(target, -100), target)
        s = {"H": H, "W": W, "target": target}
        if kind == "xent_bwd":
            z = H.float() @ W.float().T
            top = z.amax(1, keepdim=True)
            s["lse"] = (top + (z - top).exp_().sum(1, keepdim=True).log()).squeeze(1)
            kept = target >= 0
            s["grad"] = torch.where(kept, 1.0 / kept.sum().clamp(min=1), 0.0).float()
        return s
    if kind.startswith("norm"):
        M, N = case["M"], case["N"]
        # a residual stream: rows of different size, a common offset
        x = ((0.5 + uniform(M, 1)) * normal(M, N) + 0.3).to(dt)
        s = {"x": x, "gamma": (1.0 + 0.1 * normal(N)).to(dt), "beta": (0.1 * normal(N)).to(dt)}
        if kind == "norm_bwd":
            xf = x.float()
            mean = xf.mean(1)
            s["mean"] = mean
            s["rstd"] = ((xf - mean[:, None]).square().mean(1) + EPS).rsqrt()
            s["dy"] = (1e-3 * normal(M, N)).to(dt)
        return s
    T, V, K = case["T"], case["V"], case["K"]
    # token frequencies fall as 1 / rank; with an offset, ids of the other
    # ranks' shares too, and some padding
    span = V + 2 * case["v0"]
    ids = torch.exp(uniform(T) * math.log(span)).long().sub_(1).clamp_(0, span - 1)
    if case["v0"]:
        ids = (ids * 7919) % span
    ids = torch.where(uniform(T) < 0.03, torch.full_like(ids, -1), ids)
    s = {"ids": ids}
    if kind == "embed_fwd":
        s["table"] = (0.02 * normal(V, K)).to(dt)
    else:
        s["dy"] = (1e-3 * normal(T, K)).to(dt)
    return s


def prepare(case, seed):
    s = _seeded(case, seed)
    s["case"] = case
    return s


# ------------------------------------------------------- the framework's calls
def _buffers(s):
    """Outputs and workspaces, which a program allocates once and keeps."""
    from paper_2609_10549_amd import compass as C
    case, dev = s["case"], torch.device("cuda")
    kind, dt = case["kind"], _type(case)

    def empty(*shape, dtype=torch.float32):
        return torch.empty(shape, dtype=dtype, device=dev)

    def scratch(nbytes):
        return torch.empty(max(nbytes, 16), dtype=torch.uint8, device=dev)

    if kind.startswith("xent"):
        M, V, K = case["M"], case["V"], case["K"]
        if kind == "xent_fwd":
            return {"C": C, "lse": empty(M), "tlogit": empty(M), "loss": empty(M),
                    "ws": scratch(C.compass_xent_workspace(M, V, K))}
        return {"C": C, "dH": empty(M, K, dtype=torch.bfloat16), "dW": empty(V, K, dtype=torch.bfloat16),
                "ws": scratch(C.compass_xent_workspace(M, V, K, backward=True))}
    if kind.startswith("norm"):
        M, N = case["M"], case["N"]
        if kind == "norm_fwd":
            return {"C": C, "y": empty(M, N, dtype=dt), "mean": empty(M), "rstd": empty(M)}
        return {"C": C, "dx": empty(M, N, dtype=dt), "dgamma": empty(N), "dbeta": empty(N),
                "ws": scratch(C.compass_norm_workspace(M, N))}
    T, V, K = case["T"], case["V"], case["K"]
    if kind == "embed_fwd":
        return {"C": C, "y": empty(T, K, dtype=dt)}
    return {"C": C, "dtable": empty(V, K, dtype=dt), "ws": scratch(C.compass_embed_workspace(T, V, K))}


def _scale(case):
    return math.sqrt(case["K"])


def _own(s):
    b = s.get("buffers")
    if b is None:
        b = s["buffers"] = _buffers(s)
    C, case = b["C"], s["case"]
    kind = case["kind"]
    if kind == "xent_fwd":
        C.compass_xent_forward(s["H"], s["W"], s["target"], b["lse"], b["tlogit"], b["loss"], b["ws"])
        return {"lse": b["lse"], "tlogit": b["tlogit"], "loss": b["loss"]}
    if kind == "xent_bwd":
        C.compass_xent_backward(s["H"], s["W"], s["target"], s["lse"], s["grad"], b["dH"], b["dW"], b["ws"])
        return {"dH": b["dH"], "dW": b["dW"]}
    if kind == "norm_fwd":
        C.compass_norm_forward(s["x"], s["gamma"], s["beta"], b["y"], b["mean"], b["rstd"], eps=EPS)
        return {"y": b["y"], "mean": b["mean"], "rstd": b["rstd"]}
    if kind == "norm_bwd":
        C.compass_norm_backward(s["dy"], s["x"], s["gamma"], s["mean"], s["rstd"], b["dx"], b["dgamma"], b["dbeta"],
                                b["ws"])
        return {"dx": b["dx"], "dgamma": b["dgamma"], "dbeta": b["dbeta"]}
    if kind == "embed_fwd":
        C.compass_embed_forward(s["ids"], s["table"], b["y"], scale=_scale(case), v0=case["v0"])
        return {"y": b["y"]}
    C.compass_embed_backward(s["ids"], s["dy"], b["dtable"], b["ws"], scale=_scale(case), v0=case["v0"])
    return {"dtable": b["dtable"]}


# ------------------------------------------------------------- the plain form
def _plain(s):
    case = s["case"]
    kind, dt = case["kind"], _type(case)
    if kind == "xent_fwd":
        z = s["H"].float() @ s["W"].float().T
        top = z.amax(1, keepdim=True)
        t = s["target"]
        tlogit = torch.where(t >= 0, z.gather(1, t.clamp(min=0)[:, None])[:, 0], 0.0)
        lse = top[:, 0] + (z - top).exp_().sum(1).log()
        return {"lse": lse, "tlogit": tlogit, "loss": torch.where(t >= 0, lse - tlogit, 0.0)}
    if kind == "xent_bwd":
        H, W, t = s["H"].float(), s["W"].float(), s["target"]
        p = (H @ W.T).sub_(s["lse"][:, None]).exp_()
        p.scatter_add_(1, t.clamp(min=0)[:, None], -(t >= 0).float()[:, None])
        p.mul_(torch.where(t >= 0, s["grad"], 0.0)[:, None])
        return {"dH": (p @ W).to(torch.bfloat16), "dW": (p.T @ H).to(torch.bfloat16)}
    if kind == "norm_fwd":
        x = s["x"].float()
        mean = x.mean(1)
        xc = x - mean[:, None]
        rstd = (xc.square().mean(1) + EPS).rsqrt()
        y = xc * rstd[:, None] * s["gamma"].float() + s["beta"].float()
        return {"y": y.to(dt), "mean": mean, "rstd": rstd}
    if kind == "norm_bwd":
        dy = s["dy"].float()
        xh = (s["x"].float() - s["mean"][:, None]) * s["rstd"][:, None]
        a = dy * s["gamma"].float()
        dx = (a - a.mean(1, keepdim=True) - xh * (a * xh).mean(1, keepdim=True)) * s["rstd"][:, None]
        return {"dx": dx.to(dt), "dgamma": (dy * xh).sum(0), "dbeta": dy.sum(0)}
    local = s["ids"] - case["v0"]
    inside = (local >= 0) & (local < case["V"])
    row = torch.where(inside, local, 0)
    if kind == "embed_fwd":
        y = s["table"][row].float() * _scale(case)
        return {"y": torch.where(inside[:, None], y, 0.0).to(dt)}
    dy = s["dy"].float() * _scale(case)
    dt32 = torch.zeros(case["V"], case["K"], device=dy.device)
    dt32.index_add_(0, row, torch.where(inside[:, None], dy, 0.0))
    return {"dtable": dt32.to(dt)}


def run(state):
    return _own(state) if own else _plain(state)


def work(case):
    kind = case["kind"]
    if kind.startswith("xent"):
        M, V, K = case["M"], case["V"], case["K"]
        operands = 2.0 * K * (M + V)
        if kind == "xent_fwd":
            return {"bytes": operands + 20.0 * M, "flops": 2.0 * M * V * K}
        return {"bytes": 2.0 * operands + 16.0 * M, "flops": 6.0 * M * V * K}
    size = 2.0 if case["dtype"] == "bf16" else 4.0
    if kind.startswith("norm"):
        M, N = case["M"], case["N"]
        if kind == "norm_fwd":
            return {"bytes": size * (2.0 * M * N + 2.0 * N) + 8.0 * M, "flops": 8.0 * M * N}
        return {"bytes": size * (3.0 * M * N + N) + 8.0 * M + 8.0 * N, "flops": 15.0 * M * N}
    T, V, K = case["T"], case["V"], case["K"]
    if kind == "embed_fwd":
        # each table row that is looked up read once: at most the whole table
        return {"bytes": size * K * (T + min(T, V)) + 8.0 * T, "flops": 1.0 * T * K}
    return {"bytes": size * K * (T + V) + 8.0 * T, "flops": 2.0 * T * K}


# ------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    s = _seeded(case, seed)
    kind = case["kind"]
    if kind.startswith("xent"):
        H, W, t = s["H"].double(), s["W"].double(), s["target"]
        kept = t >= 0
        rows = torch.nonzero(kept)[:, 0]
        z = torch.mm(H, W.t())
        if kind == "xent_fwd":
            lse = torch.logsumexp(z, dim=1)
            tlogit = torch.zeros_like(lse)
            tlogit[rows] = z[rows, t[rows]]
            return {"lse": lse, "tlogit": tlogit, "loss": (lse - tlogit) * kept.double()}
        # the log-sum-exp is an input, as is each row's weight
        dz = torch.exp(z - s["lse"].double().unsqueeze(1))
        del z
        dz[rows, t[rows]] -= 1.0
        dz *= (s["grad"].double() * kept.double()).unsqueeze(1)
        return {"dH": torch.mm(dz, W), "dW": torch.mm(dz.t(), H)}
    if kind == "norm_fwd":
        x = s["x"].double()
        var, mean = torch.var_mean(x, dim=1, correction=0)
        rstd = 1.0 / torch.sqrt(var + EPS)
        y = (x - mean.unsqueeze(1)).mul_(rstd.unsqueeze(1))
        return {"y": torch.addcmul(s["beta"].double(), y, s["gamma"].double()), "mean": mean, "rstd": rstd}
    if kind == "norm_bwd":
        dy, r = s["dy"].double(), s["rstd"].double().unsqueeze(1)
        xh = (s["x"].double() - s["mean"].double().unsqueeze(1)) * r
        N = float(case["N"])
        dgamma, dbeta = torch.einsum("mn,mn->n", dy, xh), dy.sum(dim=0)
        dxh = dy * s["gamma"].double()
        c1, c2 = dxh.sum(dim=1, keepdim=True), torch.einsum("mn,mn->m", dxh, xh).unsqueeze(1)
        return {"dx": r / N * (N * dxh - c1 - xh * c2), "dgamma": dgamma, "dbeta": dbeta}
    V, K, f = case["V"], case["K"], math.sqrt(case["K"])
    local = s["ids"] - case["v0"]
    keep = torch.nonzero((local >= 0) & (local < V))[:, 0]
    if kind == "embed_fwd":
        y = torch.zeros(case["T"], K, dtype=torch.float64, device=local.device)
        y[keep] = s["table"].double()[local[keep]] * f
        return {"y": y}
    d = torch.zeros(V, K, dtype=torch.float64, device=local.device)
    d.index_put_((local[keep],), s["dy"].double()[keep] * f, accumulate=True)
    return {"dtable": d}
