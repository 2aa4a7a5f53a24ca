"""The vocabulary cross entropy over long reductions, where element-wise worst
cases (every rounding in one direction) would let errors of a tenth pass: the
errors' sizes over all rows, and each probability by itself.

Bounds. A logit is a sum of K products whose roundings (at most 2^-23 of a partial
sum, which a matrix core may truncate) are taken as independent: sqrt(K) 2^-23 of
the largest logit, which bounds the partial sums. dz, dH and dW are rounded to
bf16, at most 2^-8 of each element, independently and to both sides: the root of
the sum of their squares."""
from __future__ import annotations

import pytest

from paper_2609_10549_amd import compass as C
from tests.test_gpu_model_ends import _backward, _nan, _scratch, _xent_inputs

pytestmark = pytest.mark.gpu

U8, U23 = 2.0 ** -8, 2.0 ** -23
DEEP = [(300, 4099, 12288), (1100, 130, 16384), (409, 57510, 952), (37, 20011, 8200), (2100, 3001, 4088)]


@pytest.mark.parametrize("M,V,K", DEEP)
def test_errors_over_long_reductions(M, V, K):
    print(f"xent depth {M} {V} {K}", flush=True)
    import torch
    H, W, t = _xent_inputs(M, V, K, 61)
    h, w = H.double(), W.double()
    z = h @ w.T
    kept = t >= 0
    at = t.clamp(min=0)[:, None]
    r_lse = torch.logsumexp(z, 1)
    z_err = U23 * K ** 0.5 * float(z.abs().max())
    lse, tl, loss = _nan(M), _nan(M), _nan(M)
    C.compass_xent_forward(H, W, t, lse, tl, loss, _scratch(C.compass_xent_workspace(M, V, K)))
    r_tl = torch.where(kept, z.gather(1, at)[:, 0], 0.0)
    # a row's sum: chains of at most 64 + V / 1024 + 16 roundings; the lse's own
    lse_err = z_err + U23 * (80 + V / 1024 + float(r_lse.abs().max()))
    for name, got, ref, tol in (("lse", lse, r_lse, lse_err), ("tlogit", tl, r_tl, z_err),
                                ("loss", loss, torch.where(kept, r_lse - r_tl, 0.0), lse_err + z_err)):
        rms = float((got.double() - ref).square().mean().sqrt())
        print(f"{name}: {rms:.3g} of {tol:.3g}", flush=True)
        assert rms <= tol, name

    lse = r_lse.float()
    grad = (torch.arange(M, device="cuda") % 13 + 1.0) / (7 * M)
    dH, dW = _backward(H, W, t, lse, grad)
    g = torch.where(kept, grad.double(), 0.0)[:, None]
    p = g * (z - lse.double()[:, None]).exp()       # what the probabilities bring in
    dz = p.clone().scatter_add_(1, at, -g)
    del z
    for name, got, left, soft, right in (("dH", dH, dz, p, w), ("dW", dW, dz.T.contiguous(), p.T.contiguous(), h)):
        ref = left @ right
        # dz's rounding and the result's, and the exponents' errors
        square = U8 ** 2 * (left.square() @ right.square() + ref.square()) \
            + (z_err + 128 * U23) ** 2 * (soft.square() @ right.square())
        err = got.double() - ref
        print(f"{name}: {float(err.norm() / ref.norm()):.3g} of {float(square.sum().sqrt() / ref.norm()):.3g}", flush=True)
        assert float(err.square().sum()) <= float(square.sum()), name


def test_each_probability():
    """W the unit matrix: logits are H itself and dH is dz, element by element, held
    to the two roundings to bf16 that it takes (of dz and of dH)."""
    import torch
    M, V = 512, 2048
    g = torch.Generator(device="cuda").manual_seed(62)
    H = (2.0 * torch.randn(M, V, generator=g, device="cuda")).bfloat16()
    W = torch.eye(V, device="cuda").bfloat16()
    t = torch.randint(0, V, (M,), generator=g, device="cuda")
    z = H.double()
    r_lse = torch.logsumexp(z, 1)
    lse, tl, loss = _nan(M), _nan(M), _nan(M)
    C.compass_xent_forward(H, W, t, lse, tl, loss, _scratch(C.compass_xent_workspace(M, V, V)))
    # chains of at most 64 + 16 + 2 roundings, 2 for each exponential; lse's own
    tol = U23 * (84 + float(r_lse.max()))
    assert float((lse.double() - r_lse).abs().max()) <= tol
    assert float((lse.double() - r_lse).mean().abs()) <= tol / 4

    lse = r_lse.float()
    grad = 0.01 + 0.001 * torch.arange(M, device="cuda")
    dH, _ = _backward(H, W, t, lse, grad)
    ref = grad.double()[:, None] * (z - lse.double()[:, None]).exp()
    other = torch.ones(M, V, dtype=torch.bool, device="cuda")
    other[torch.arange(M, device="cuda"), t] = False
    assert float((dH.double() / ref - 1)[other].abs().max()) <= 2 * U8 + U8 ** 2
