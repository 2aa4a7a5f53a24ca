"""Ids and targets at the ends of 64 bits, over shards that begin at 0, at the
middle and at the last place: none but the shard's own count, however far away."""
from __future__ import annotations

import pytest

from paper_2609_10549_amd import compass as C

pytestmark = pytest.mark.gpu

LAST = 2 ** 63 - 1
V = 70


def _torch():
    import torch
    return torch


def _ids(v0):
    """Far and near, inside and out: the shard's ends, 64 bits' ends, and what
    differs from an id inside by 2^63 or 2^64."""
    out = [v0, v0 + V - 1, v0 + 3, v0 - 1, v0 + V, -LAST - 1, -LAST, -1, -100, 0, LAST, 2 ** 62, -2 ** 62, v0 - 2 ** 62]
    out += [x for v in (v0 + 1, v0 + V - 2) for d in (2 ** 32, 2 ** 63) for x in (v + d, v - d)]
    return [x for x in out if -LAST - 1 <= x <= LAST]


@pytest.mark.parametrize("v0", [0, 5, 2 ** 40, 2 ** 62, LAST - V])
def test_embedding(v0):
    torch = _torch()
    K = 40
    ids = _ids(v0)
    table = torch.randint(-64, 65, (V, K), device="cuda").float()
    dev = torch.tensor(ids, dtype=torch.int64).cuda()
    y = torch.full((len(ids), K), float("nan"), device="cuda")
    C.compass_embed_forward(dev, table, y, scale=2.0, v0=v0)
    d = torch.full((V, K), float("nan"), device="cuda")
    ws = torch.empty(C.compass_embed_workspace(len(ids), V, K), dtype=torch.uint8, device="cuda")
    C.compass_embed_backward(dev, y, d, ws, v0=v0)
    want = torch.zeros_like(d)
    for i, v in enumerate(ids):
        at = v - v0 if 0 <= v - v0 < V else None
        assert torch.equal(y[i], torch.zeros(K, device="cuda") if at is None else 2.0 * table[at]), v
        if at is not None:
            want[at] += y[i]
    assert torch.equal(d, want)


@pytest.mark.parametrize("v0", [0, 5, 2 ** 40, 2 ** 62, LAST - V])
@pytest.mark.parametrize("piece", [0, 33])
def test_cross_entropy(v0, piece):
    """One logit of 8, at one column, else 0: lse is the same for all rows."""
    torch = _torch()
    K = 64
    targets = _ids(v0)
    M = len(targets)
    H, W = torch.zeros(M, K, dtype=torch.bfloat16), torch.zeros(V, K, dtype=torch.bfloat16)
    H[:, 0], W[V - 1, 0] = 8.0, 1.0
    W[:, 1] = torch.arange(V) - 35.0            # tells the rows of W apart
    H, W, t = H.cuda(), W.cuda(), torch.tensor(targets, dtype=torch.int64).cuda()
    lse, tl, loss = (torch.full((M,), float("nan"), device="cuda") for _ in range(3))
    ws = torch.empty(C.compass_xent_workspace(M, V, K), dtype=torch.uint8, device="cuda")
    C.compass_xent_forward(H, W, t, lse, tl, loss, ws, v0=v0)
    for i, v in enumerate(targets):
        z = 8.0 if v - v0 == V - 1 else 0.0
        assert float(tl[i]) == z and float(loss[i]) == (0.0 if v < 0 else float(lse[i]) - z), v
    dH, dW = torch.empty_like(H), torch.empty_like(W)
    ws = torch.empty(C.compass_xent_workspace(M, V, K, backward=True, piece=piece), dtype=torch.uint8, device="cuda")
    C.compass_xent_backward(H, W, t, lse, torch.ones(M, device="cuda"), dH, dW, ws, v0=v0, piece=piece)
    p = torch.full((V,), 1.0, dtype=torch.float64)
    p[V - 1] = torch.tensor(8.0, dtype=torch.float64).exp()
    p /= p.sum()
    w = W.double().cpu()
    for i, v in enumerate(targets):
        dz = p.clone() if v >= 0 else torch.zeros(V, dtype=torch.float64)
        if 0 <= v - v0 < V and v >= 0:
            dz[v - v0] -= 1.0
        # dz and dH are rounded to bf16, p is good to fp32
        assert ((dH[i].double().cpu() - dz @ w).abs() <= 2 ** -7 * (dz.abs() @ w.abs()) + 1e-6).all(), v
