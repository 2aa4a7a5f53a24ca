"""The vocabulary cross entropy on logits that fp32 holds exactly, where the
result's own properties are exact too: a loss is never negative and is zero
where the target's probability rounds to one."""
from __future__ import annotations

import numpy as np
import pytest

from oracle import model_ends as E
from paper_2609_10549_amd import compass as C

pytestmark = pytest.mark.gpu

U24 = 2.0 ** -24


def _torch():
    import torch
    return torch


def _np(t):
    return t.double().cpu().numpy()


def _nan(*shape, dtype=None):
    torch = _torch()
    return torch.full(shape, float("nan"), dtype=dtype or torch.float32, device="cuda")


def _scratch(n):
    torch = _torch()
    return torch.full((max(n, 16),), 0xFF, dtype=torch.uint8, device="cuda")   # NaN patterns


def _dominated(M, V, K, at, seed, lo=1.0, hi=64.0):
    """H, W and targets, all of them `at`, whose logit s (1 + r / 256) (s in [lo, hi),
    r in [1/2, 1)) is the row's largest by s or more: the others are s (a + b r / 256)
    with a in [-1, 0] and b = +-1. In bf16 the two terms have 16 and 8 bits, their
    sum at most 19."""
    torch = _torch()
    g = torch.Generator().manual_seed(seed)
    W, H = torch.zeros(V, K), torch.zeros(M, K)
    W[:, 0] = -torch.randint(0, 257, (V,), generator=g) / 256
    W[:, 1] = 1.0 - 2.0 * torch.randint(0, 2, (V,), generator=g)
    W[at, 0] = W[at, 1] = 1.0
    H[:, 0] = lo + (hi - lo) * torch.rand(M, generator=g)
    H[:, 1] = H[:, 0] * (0.5 + 0.5 * torch.rand(M, generator=g)) / 256
    bf = torch.bfloat16
    return H.to(bf).cuda(), W.to(bf).cuda(), torch.full((M,), at).cuda()


# one column; columns within a tile, over several and at the last tile's edge;
# few rows (a workgroup each in the join) and many
DOMINATED = [(1, 1, 8, 0), (300, 1, 64, 0), (8, 1000, 72, 999), (97, 64, 64, 0), (300, 4099, 72, 2050), (700, 130, 136, 129),
             (2000, 20011, 72, 7)]


@pytest.mark.parametrize("M,V,K,at", DOMINATED)
def test_loss_is_never_negative_and_zero_for_certain_rows(M, V, K, at):
    print(f"xent dominated {M} {V} {K}", flush=True)
    torch = _torch()
    H, W, t = _dominated(M, V, K, at, 71)
    lse, tl, loss = _nan(M), _nan(M), _nan(M)
    C.compass_xent_forward(H, W, t, lse, tl, loss, _scratch(C.compass_xent_workspace(M, V, K)))
    r_lse, r_tl, r_loss = E.xent_forward(_np(H), _np(W), t.cpu().numpy())
    assert np.array_equal(_np(tl), r_tl)
    assert (loss >= 0).all(), f"{int((loss < 0).sum())} of {M} losses below 0, down to {float(loss.min())}"
    assert (lse >= tl).all()
    # e^-32 times 20011 others is below half a step of fp32 at 1
    certain = (H[:, 0] >= 32) | (V == 1)
    assert not loss[certain].any()
    # 64 terms in a lane, at most 79 of 256 workgroup parts one after another
    # (three roundings each), a tree; then lse's own rounding
    assert (np.abs(_np(loss) - r_loss) <= U24 * (r_lse + r_loss) + 400 * U24).all()
    assert torch.equal(loss, lse - tl)


def test_loss_of_a_split_vocabulary_is_never_negative():
    M, n, V, K = 500, 4, 33, 72
    H, W, t = _dominated(M, n * V, K, 2 * V + 5, 72)
    lse_p, tl_p, lse, loss = _nan(n, M), _nan(n, M), _nan(M), _nan(M)
    for q in range(n):
        C.compass_xent_forward(H, W[q * V:(q + 1) * V], t, lse_p[q], tl_p[q], None,
                               _scratch(C.compass_xent_workspace(M, V, K)), v0=q * V)
    C.compass_xent_join(lse_p, tl_p, t, lse, loss)
    assert (loss >= 0).all() and not loss[H[:, 0] >= 32].any()


@pytest.mark.parametrize("size", [8000.0, 2.0 ** 60, 2.0 ** 127])
def test_one_column_is_certain_at_any_size(size):
    torch = _torch()
    M, K = 70, 64
    H, W, t = _dominated(M, 1, K, 0, 73, lo=size, hi=1.9 * size)
    H[::2] *= -1
    lse, tl, loss = _nan(M), _nan(M), _nan(M)
    C.compass_xent_forward(H, W, t, lse, tl, loss, _scratch(C.compass_xent_workspace(M, 1, K)))
    z = H[:, 0].double() + H[:, 1].double()
    assert torch.equal(lse, z.float()) and torch.equal(tl, z.float()) and not loss.any()


def _backward(H, W, t, lse, grad):
    torch = _torch()
    (M, K), V = H.shape, W.shape[0]
    dH, dW = _nan(M, K, dtype=torch.bfloat16), _nan(V, K, dtype=torch.bfloat16)
    C.compass_xent_backward(H, W, t, lse, grad, dH, dW, _scratch(C.compass_xent_workspace(M, V, K, backward=True)))
    return dH, dW


@pytest.mark.parametrize("M,V,K,at", DOMINATED)
def test_certain_rows_have_no_gradient(M, V, K, at):
    """exp(z - lse) is 1 where lse is z: what is left of a certain row are the
    other columns, e^-31 or less each."""
    print(f"xent dominated backward {M} {V} {K}", flush=True)
    torch = _torch()
    H, W, t = _dominated(M, V, K, at, 74, lo=1.0 if V == 1 else 32.0)
    lse = torch.from_numpy(E.xent_forward(_np(H), _np(W), t.cpu().numpy())[0]).float().cuda()
    grad = torch.randn(M, generator=torch.Generator().manual_seed(75)).cuda()
    dH, dW = _backward(H, W, t, lse, grad)
    if V == 1:
        assert not dH.any() and not dW.any()
    left = (V - 1) * float(np.exp(-31.0))
    assert (dH.abs().amax(1) <= grad.abs() * left).all()
    assert float(dW.abs().max()) <= float((grad.abs() * H[:, 0]).sum()) * left


@pytest.mark.parametrize("size", [8000.0, 2.0 ** 60, 2.0 ** 127])
def test_one_column_has_no_gradient_at_any_size(size):
    torch = _torch()
    M, K = 70, 64
    H, W, t = _dominated(M, 1, K, 0, 76, lo=size, hi=1.9 * size)
    H[::2] *= -1
    lse = (H[:, 0].double() + H[:, 1].double()).float()
    dH, dW = _backward(H, W, t, lse, torch.ones(M, device="cuda"))
    assert not dH.any() and not dW.any()
