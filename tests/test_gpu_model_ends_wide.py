"""More of the operators at a model's ends on the GPU: operands whose elements
lie more than 2^31 elements (2^32 bytes) from the first (a long vocabulary, a
long batch, rows far apart), and few rows of the cross entropy. Cross entropy
against fp64 with the bounds of test_gpu_model_ends.py; the others bit for bit
(exact sums, or the same rows packed)."""
from __future__ import annotations

import pytest

from paper_2609_10549_amd import compass as C

pytestmark = pytest.mark.gpu

U8, U24 = 2.0 ** -8, 2.0 ** -24


def _torch():
    import torch
    return torch


def _gen(seed):
    return _torch().Generator(device="cuda").manual_seed(seed)


def _scratch(n):
    torch = _torch()
    return torch.full((max(n, 16),), 0xFF, dtype=torch.uint8, device="cuda")   # NaN patterns


def _nan(*shape, dtype=None):
    torch = _torch()
    return torch.full(shape, float("nan"), dtype=dtype or torch.float32, device="cuda")


def _within(name, got, ref, tol):
    torch = _torch()
    assert torch.isfinite(got).all(), name
    over = (got.double() - ref).abs() - tol
    assert not (over > 0).any(), f"{name}: {int((over > 0).sum())} of {got.numel()} out of bound, by up to {float(over.max()):.3g}"


def _blocks(n, step):
    return [slice(i, min(n, i + step)) for i in range(0, n, step)]


@pytest.mark.parametrize("M,V,K", [(5, 270001, 8192), (600001, 70, 4096)])
def test_xent_operands_beyond_32_bits(M, V, K):
    print(f"xent wide {M} {V} {K}", flush=True)
    torch = _torch()
    bf = torch.bfloat16
    g = _gen(51)
    W = torch.empty(V, K, dtype=bf, device="cuda").normal_(generator=g).mul_(1.5 / K ** 0.5)
    H = torch.empty(M, K, dtype=bf, device="cuda").normal_(generator=g)
    assert max(W.numel(), H.numel()) > 2 ** 31
    t = torch.randint(0, V, (M,), generator=g, device="cuda")
    t[0], t[M - 1] = V - 1, V - 2
    t[1::7] = -100
    # of a long batch the ends alone carry a loss: rows of zeros add no rounding,
    # and the weight gradient's bound stays below what a misplaced row would change
    t[1000:-1000] = -100
    ms, vs = _blocks(M, 32768), _blocks(V, 32768)

    def product(f):
        return torch.cat([torch.cat([f(H[m].double()) @ f(W[v].double()).T for v in vs], 1) for m in ms], 0)

    mag = product(torch.abs).amax(1)
    z = product(lambda x: x)
    kept = t >= 0
    at = t.clamp(min=0)[:, None]
    r_lse = torch.logsumexp(z, 1)
    r_tl = torch.where(kept, z.gather(1, at)[:, 0], 0.0)
    z_tol = 2 * K * U24 * mag
    tol = z_tol + 2 * U24 * (V + 64 + 4 * mag)
    lse, tl, loss = _nan(M), _nan(M), _nan(M)
    C.compass_xent_forward(H, W, t, lse, tl, loss, _scratch(C.compass_xent_workspace(M, V, K)))
    _within("lse", lse, r_lse, tol)
    _within("tlogit", tl, r_tl, z_tol + 2 * U24 * r_tl.abs())
    r_loss = torch.where(kept, r_lse - r_tl, 0.0)
    _within("loss", loss, r_loss, z_tol + tol + 2 * U24 * r_loss.abs())

    lse = r_lse.float()
    grad = (torch.randn(M, generator=g, device="cuda") * 0.3 + 1.0) / M
    dH, dW = _nan(M, K, dtype=bf), _nan(V, K, dtype=bf)
    C.compass_xent_backward(H, W, t, lse, grad, dH, dW, _scratch(C.compass_xent_workspace(M, V, K, backward=True)))
    gd = grad.double()[:, None]
    p = (z - lse.double()[:, None]).exp_()
    delta = (z_tol + tol + 128 * U24)[:, None] * 1.01
    err = (1 + U8) * gd.abs() * (p * delta + 4 * U24)
    p.scatter_add_(1, at, -kept.double()[:, None])
    dz = torch.where(kept[:, None], gd, 0.0) * p
    err += dz.abs() * (U8 + 4 * U24 * (1 + U8))
    err[~kept] = 0.0
    del p, z

    def check(name, got, left, left_err, right, blocks, terms):
        """got = left right, both summed over `blocks`; left's error is given."""
        ref = bound = 0.0
        for b in blocks:
            r = right[b].double()
            ref = ref + left[:, b].contiguous() @ r
            bound = bound + (left_err[:, b] + 2 * terms * U24 * left[:, b].abs()).contiguous() @ r.abs()
        _within(name, got, ref, bound + U8 * (ref.abs() + bound))

    for m in ms:
        check("dH", dH[m], dz[m], err[m], W, vs, V)
    for v in vs:
        check("dW", dW[v], dz[:, v].T, err[:, v].T, H, ms, int(kept.sum()))


@pytest.mark.parametrize("dtype,N", [("bfloat16", 1032), ("float32", 1031)])
def test_norm_rows_beyond_32_bits(dtype, N):
    print(f"norm wide {dtype} {N}", flush=True)
    torch = _torch()
    dt = getattr(torch, dtype)
    M, ld = 301, 8_000_000
    assert (M - 1) * ld > 2 ** 31
    g = _gen(52)
    x, dy = (torch.randn(M, N, generator=g, device="cuda").to(dt) for _ in range(2))
    gamma, beta = (torch.randn(N, generator=g, device="cuda").to(dt) for _ in range(2))
    ws = _scratch(C.compass_norm_workspace(M, N))

    def run(x, dy, y, dx):
        mean, rstd, dg, db = _nan(M), _nan(M), _nan(N), _nan(N)
        C.compass_norm_forward(x, gamma, beta, y, mean, rstd)
        C.compass_norm_backward(dy, x, gamma, mean, rstd, dx, dg, db, ws)
        return y, dx, mean, rstd, dg, db

    want = run(x, dy, _nan(M, N, dtype=dt), _nan(M, N, dtype=dt))

    def apart():
        return torch.empty(M, ld, dtype=dt, device="cuda")[:, :N]

    got = run(apart().copy_(x), apart().copy_(dy), apart(), apart())
    for a, b in zip(got, want):
        assert torch.isfinite(b).all() and torch.equal(a, b)


@pytest.mark.parametrize("K", [33000, 32999])
def test_embed_operands_beyond_32_bits(K):
    print(f"embed wide {K}", flush=True)
    torch = _torch()
    bf = torch.bfloat16
    T = V = 66000
    assert T * K > 2 ** 31
    g = _gen(53)
    ids = torch.randint(-2, V + 2, (T,), generator=g, device="cuda")
    ids[::11] = V - 1                       # a long run, at the table's end
    inside = (ids >= 0) & (ids < V)
    row = torch.where(inside, ids, 0)
    table = torch.empty(V, K, dtype=bf, device="cuda").normal_(generator=g)
    y = _nan(T, K, dtype=bf)
    C.compass_embed_forward(ids, table, y, scale=4.0)
    for b in _blocks(T, 8192):
        assert torch.equal(y[b], torch.where(inside[b, None], table[row[b]] * 4.0, 0.0))
    # integers, whose fp32 sums are exact
    dy = y.copy_(torch.randint(-4, 5, (T, K), generator=g, device="cuda", dtype=torch.int8))
    d = table.fill_(float("nan"))
    C.compass_embed_backward(ids, dy, d, _scratch(C.compass_embed_workspace(T, V, K)), scale=0.5)
    for b in _blocks(K, 4096):
        ref = torch.zeros(V, dy[:, b].shape[1], device="cuda")
        ref.index_add_(0, row, torch.where(inside[:, None], dy[:, b].float() * 0.5, 0.0))
        assert torch.equal(d[:, b], ref.to(bf))


# few rows whose weight gradient does not lie on 128-byte lines, in every tile
# that such a gradient takes (64 x 64, 256 x 192, 192 x 192, 128 x 128), and both
# sides of the sizes where that ends (64 rows) and where the largest weight takes
# a launch of its own (256)
@pytest.mark.parametrize("M,V,K", [(1, 1, 8), (33, 1161, 8200), (16, 4099, 2056), (3, 130, 12296), (64, 20011, 72),
                                   (65, 20011, 72), (256, 1000, 264), (257, 1000, 264)])
def test_xent_few_rows(M, V, K):
    from tests.test_gpu_model_ends import test_xent_every_tile
    test_xent_every_tile(M, V, K)


def test_xent_rows_of_very_different_weight():
    """The largest weight in the last of 256 rows (of the rows that dz's own
    workgroups look through): those of the others, 2^20 times smaller, stay
    whole numbers of bf16 steps of their own."""
    torch = _torch()
    M, V, K = 256, 8, 64
    H = torch.zeros(M, K, dtype=torch.bfloat16, device="cuda")
    H[:, 0] = 1.0
    W = torch.zeros(V, K, dtype=torch.bfloat16, device="cuda")
    W[:, 1] = torch.tensor([1.0, 2.0, 4.0, 8.0, 16.0, 32.0, 64.0, 128.0], device="cuda")
    t = torch.arange(M, device="cuda") % V
    lse = torch.full((M,), 3 * 0.6931471805599453, device="cuda")    # 8 equal logits
    grad = torch.full((M,), 2.0 ** -20, device="cuda")
    grad[M - 1] = 1.0
    dH, dW = _nan(M, K, dtype=torch.bfloat16), _nan(V, K, dtype=torch.bfloat16)
    C.compass_xent_backward(H, W, t, lse, grad, dH, dW, _scratch(C.compass_xent_workspace(M, V, K, backward=True)))
    g = grad.double()[:, None]
    p = (0.0 - lse.double()[:, None]).exp().expand(M, V).clone()
    p[torch.arange(M, device="cuda"), t] -= 1.0
    dz = g * p
    err = dz.abs() * U8 + g * 128 * U24
    w, h = W.double(), H.double()
    for name, got, ref, e in (("dH", dH, dz @ w, err @ w.abs() + 2 * V * U24 * (dz.abs() @ w.abs())),
                              ("dW", dW, dz.T @ h, err.T @ h.abs() + 2 * M * U24 * (dz.abs().T @ h.abs()))):
        _within(name, got, ref, e + U8 * (ref.abs() + e))
