"""The row weights of the cross entropy's gradient. dz is held in bf16 as a
multiple of the largest weight, so a weight that all rows share, or that one row
alone has, costs no rounding: with logits that make every dz / weight a multiple
of 1/8, dH and dW are the exact sums times the weight, rounded to bf16. A weight
that is no power of two shows a missed largest one: its dz would be rounded."""
from __future__ import annotations

import pytest

from paper_2609_10549_amd import compass as C

pytestmark = pytest.mark.gpu

V, K = 8, 64


def _torch():
    import torch
    return torch


def _case(M, seed):
    """8 equal logits (H is zero where W is not, and the reverse), targets at all
    of them: dz is the row's weight times 1/8, or -7/8 at the target."""
    torch = _torch()
    g = torch.Generator().manual_seed(seed)
    H, W = torch.zeros(M, K), torch.zeros(V, K)
    H[:, :32] = torch.randint(-4, 5, (M, 32), generator=g).float()
    W[:, 32:] = torch.randint(-4, 5, (V, 32), generator=g).float()
    t = torch.randint(0, V, (M,), generator=g)
    unit = torch.full((M, V), 0.125)
    unit[torch.arange(M), t] -= 1.0
    lse = torch.full((M,), 3 * 0.6931471805599453)
    bf = torch.bfloat16
    return H.to(bf).cuda(), W.to(bf).cuda(), t.cuda(), unit.cuda(), lse.cuda()


def _check(H, W, t, unit, lse, weight, rows):
    """The weight is `weight` in `rows` (a truth value per row), else 0."""
    torch = _torch()
    M = H.shape[0]
    grad = torch.where(rows, weight, 0.0).float().cuda()
    dH = torch.full((M, K), float("nan"), dtype=torch.bfloat16, device="cuda")
    dW = torch.full((V, K), float("nan"), dtype=torch.bfloat16, device="cuda")
    ws = torch.full((C.compass_xent_workspace(M, V, K, backward=True),), 0xFF, dtype=torch.uint8, device="cuda")
    C.compass_xent_backward(H, W, t, lse, grad, dH, dW, ws)
    u = torch.where(rows.cuda()[:, None], unit, 0.0).double()
    w = torch.tensor(weight, dtype=torch.float32, device="cuda")
    for name, got, s in (("dH", dH, u @ W.double()), ("dW", dW, u.T.contiguous() @ H.double())):
        # the sums are multiples of 1/8 below 2^13: exact in fp32, then times the weight
        want = (s.float() * w).to(torch.bfloat16)
        assert torch.equal(got, want), f"{name}: {int((got != want).sum())} of {got.numel()} differ"


# both sides of where the search for the largest weight takes a launch of its own
# (256 rows), by values of four digits that bf16 cannot hold
@pytest.mark.parametrize("M", [1, 3, 64, 250, 256, 257, 300, 1500])
@pytest.mark.parametrize("weight", ["mean", -0.7071, 1.234e-5, 8765.0])
def test_a_shared_weight_costs_no_rounding(M, weight):
    torch = _torch()
    w = float(torch.tensor(1.0 / M if weight == "mean" else weight, dtype=torch.float32))
    _check(*_case(M, 81), w, torch.ones(M, dtype=torch.bool))


@pytest.mark.parametrize("M", [1, 64, 65, 250, 256, 257, 300, 1024, 1500])
def test_the_largest_weight_is_found_in_any_row(M):
    torch = _torch()
    for row in sorted({0, 1, 63, 64, 127, 128, 191, 192, 255, 256, 1023, 1024, M // 2, M - 1}):
        if row < M:
            _check(*_case(M, 82), float(torch.tensor(-0.00137)), torch.arange(M) == row)


@pytest.mark.parametrize("M", [250, 300])
def test_the_weight_of_a_row_without_a_target_is_not_looked_at(M):
    torch = _torch()
    H, W, t, unit, lse = _case(M, 83)
    t[5::9] = -100
    kept = (t >= 0).cpu()
    w = float(torch.tensor(0.3))
    # of the largest size, infinite and NaN in rows without a target
    for other in (1e30, float("inf"), float("nan")):
        grad = torch.where(kept, w, other).float().cuda()
        outs = []
        for g in (grad, torch.where(kept, w, 0.0).float().cuda()):
            dH = torch.full((M, K), float("nan"), dtype=torch.bfloat16, device="cuda")
            dW = torch.full((V, K), float("nan"), dtype=torch.bfloat16, device="cuda")
            ws = torch.full((C.compass_xent_workspace(M, V, K, backward=True),), 0xFF, dtype=torch.uint8, device="cuda")
            C.compass_xent_backward(H, W, t, lse, g, dH, dW, ws)
            outs.append((dH, dW))
        assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])
        assert not outs[0][0][~kept.cuda()].any()
    _check(H, W, t, unit, lse, w, kept)
