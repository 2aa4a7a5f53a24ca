"""The 8-bit product and the weight gradient at sizes that take every tile, as the
only launch, cut into slices, and as the rest behind whole rounds of another tile
along either axis; operands and results beyond 2^31 elements. References in fp64 on
the GPU; bounds as in test_gpu_eight_bits.py."""
from __future__ import annotations

import pytest

from paper_2609_10549_amd import compass as C

pytestmark = pytest.mark.gpu

U8, U24 = 2.0 ** -8, 2.0 ** -24

PRODUCT = [(643, 12241, 272), (386, 16325, 3568), (257, 10963, 128), (130, 13419, 912), (129, 11682, 128), (18, 67, 128),
           (73, 8348, 7776), (68, 5426, 4976), (66, 4180, 4672), (18, 64, 2688), (1175, 13168, 288), (1441, 5933, 6656),
           (4128, 7761, 1184), (559, 13930, 4208), (3760, 4370, 2720), (660, 11004, 3472), (589, 13175, 2640),
           (2878, 2836, 272), (5282, 1444, 3616), (4996, 782, 128), (8132, 463, 688), (7111, 259, 128), (66, 65, 128),
           (5734, 65, 4800), (4400, 65, 4768), (66, 65, 2656), (4610, 3551, 272), (4630, 1854, 4768), (7753, 4201, 1776),
           (5935, 2755, 3344), (3341, 2321, 3616), (4384, 1901, 2960), (16, 5003, 32768), (16, 77, 32784), (5, 40, 131072),
           (300, 300, 131056), (5400, 385, 22560), (2751, 3862, 32960), (12478, 1825, 3728), (656, 3515, 12208),
           (1950, 5055, 20352), (5097, 1876, 10752), (1813, 10232, 784), (3357, 2632, 7296), (19771, 1164, 144),
           (1686, 5044, 7248), (17, 4096, 4096), (32, 515, 8208), (33, 2048, 1552), (48, 4096, 4096), (47, 100, 32768)]
GRAD = [(129, 3744, 4304), (917, 928, 8144), (1, 528, 6560), (1, 392, 7136), (1, 64, 128), (7723, 664, 5520),
        (8141, 136, 4080), (2506, 136, 4624), (1982, 72, 2592), (720, 64, 128), (259, 2112, 7744), (1319, 4560, 5376),
        (760, 3728, 4368), (1010, 2256, 3616), (924, 1328, 6000), (197, 8296, 1728), (969, 5280, 1424), (1, 2328, 1712),
        (7526, 12200, 144), (4347, 8136, 144), (2650, 1312, 976), (3147, 592, 336), (707, 128, 128), (259, 5400, 3008),
        (1024, 10928, 2176), (302, 12008, 1328), (202, 14648, 1072), (913, 9352, 1680), (898, 5416, 1504),
        (918, 2984, 2704), (70000, 72, 144), (10396, 2200, 4752), (903, 1944, 12176), (5847, 3840, 2576),
        (3197, 4112, 2224), (1556, 3800, 2208)]


def _torch():
    import torch
    return torch


def _rows(rows, n, seed):
    """8-bit rows of values of one size, and what they stand for (fp64)."""
    torch = _torch()
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.randn(rows, n, generator=g, device="cuda")
    q = torch.full((rows, n), 0x7F, dtype=torch.uint8, device="cuda")
    s = torch.full((rows, C.compass_fp8_scale_cols(n)), 255, dtype=torch.uint8, device="cuda")
    C.compass_fp8_quant(x, q, s)
    return q, s


def _values(q, s):
    torch = _torch()
    step = torch.exp2(s.double() - 127).repeat_interleave(128, dim=1)[:, :q.shape[1]]
    return q.view(torch.float8_e4m3fn).double() * step


def _within(got, ref, tol):
    torch = _torch()
    over = (got.double() - ref).abs() - tol
    assert torch.isfinite(got).all() and float(over.max()) <= 0, f"{int((over > 0).sum())} out of bound by up to {float(over.max()):.3g}"


def _scratch(n):
    torch = _torch()
    return torch.full((max(n, 16),), 0xFF, dtype=torch.uint8, device="cuda")


def _cut(a, w):
    """Sum over 8 consecutive k of the largest product: what the matrix core aligns to."""
    torch = _torch()
    a, w = a.abs().float(), w.abs().float()
    out = torch.zeros(len(a), len(w), device="cuda")
    for k in range(0, a.shape[1], 8):
        top = a[:, k, None] * w[None, :, k]
        for i in range(1, 8):
            torch.maximum(top, a[:, k + i, None] * w[None, :, k + i], out=top)
        out += top
    return out.double() * (1 + 1e-3)


@pytest.mark.parametrize("M,N,K", PRODUCT)
def test_product(M, N, K):
    torch = _torch()
    (qa, sa), (qw, sw) = _rows(M, K, 1), _rows(N, K, 2)
    c = torch.full((M * N + 64,), 3.0, dtype=torch.bfloat16, device="cuda")
    need = C.compass_fp8_gemm_workspace(M, N, K)
    ws = torch.full((need + 64,), 0xA5, dtype=torch.uint8, device="cuda")
    C.compass_fp8_gemm(qa, sa, qw, sw, c[:M * N].view(M, N), ws[:need] if need else None)
    assert (c[M * N:] == 3.0).all() and (ws[need:] == 0xA5).all()
    va, vw = _values(qa, sa), _values(qw, sw)
    ref = va @ vw.T
    some = slice(None) if M * N * K < 4e9 else torch.arange(0, M, max(1, M // 40), device="cuda")   # rows that are bounded
    mag = va[some].abs() @ vw.abs().T
    # (every value against a bound that no row's is above, the sampled rows against their own)
    r = ref[some]
    _within(c[:M * N].view(M, N)[some], r, r.abs() * U8 + (K * U24 * mag + 7 * 2.0 ** -13 * _cut(va[some], vw)) * (1 + U8))
    most = 7 * 2.0 ** -13 * float(va.abs().max()) * float(vw.abs().max()) * K / 8
    _within(c[:M * N].view(M, N), ref, ref.abs() * U8 + (K * U24 * float(va.abs().max()) * vw.abs().sum(1)[None] + most) * (1 + U8))


@pytest.mark.parametrize("gtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,N,K", GRAD)
def test_weight_gradient(M, N, K, gtype):
    torch = _torch()
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    dy = (1e-3 * torch.randn(M, N, generator=g, device="cuda")).bfloat16()
    q, s = _rows(M, K, 4)
    dt = torch.bfloat16 if gtype == "bf16" else torch.float32
    out = torch.full((N * K + 64,), 3.0, dtype=dt, device="cuda")
    dw = out[:N * K].view(N, K)
    need = C.compass_fp8_wgrad_workspace(M, N, K)
    ws = torch.full((need + 64,), 0xA5, dtype=torch.uint8, device="cuda")
    C.compass_fp8_wgrad(dy, q, s, dw, ws[:need] if need else None)
    v = _values(q, s)
    ref, mag = dy.double().T @ v, dy.double().abs().T @ v.abs()
    u = U8 if gtype == "bf16" else U24
    _within(dw, ref, ref.abs() * u + M * U24 * mag * (1 + u))
    base = dw.clone()
    C.compass_fp8_wgrad(dy, q, s, dw, ws[:need] if need else None, accumulate=True)
    ref = ref + base.double()
    _within(dw, ref, ref.abs() * u + (M * U24 * mag + U24 * base.double().abs() + U24 * ref.abs()) * (1 + u))
    assert (out[N * K:] == 3.0).all() and (ws[need:] == 0xA5).all()


# ------------------------------------------------ beyond 2^31 elements, by samples
def _picked(rows, n=40):
    torch = _torch()
    at = torch.linspace(0, rows - 1, n).long()
    return torch.cat([at, torch.tensor([rows - 2])]).cuda()


@pytest.mark.parametrize("across", [False, True])
def test_wide_rows(across):
    torch = _torch()
    M, K = 70001, 32768
    x = torch.randn(M, K, device="cuda", dtype=torch.bfloat16)
    rows, n = (K, M) if across else (M, K)
    q = torch.empty(rows, n, dtype=torch.uint8, device="cuda")
    s = torch.empty(rows, C.compass_fp8_scale_cols(n), dtype=torch.uint8, device="cuda")
    C.compass_fp8_quant(x, q, s, across=across)
    at = _picked(rows)
    ref = (x[:, at].T if across else x[at]).contiguous()
    q2, s2 = torch.empty(len(at), n, dtype=torch.uint8, device="cuda"), torch.empty(len(at), s.shape[1], dtype=torch.uint8, device="cuda")
    C.compass_fp8_quant(ref, q2, s2)      # (checked element by element at small sizes)
    assert torch.equal(q[at], q2) and torch.equal(s[at], s2)
    del x
    y = torch.empty(rows, n, dtype=torch.bfloat16, device="cuda")
    C.compass_fp8_dequant(q, s, y)
    assert torch.equal(y[at].double(), _values(q2, s2))


def test_wide_norm():
    torch = _torch()
    M, N = 180001, 12288
    x, r = torch.randn(M, N, device="cuda", dtype=torch.bfloat16), torch.randn(M, N, device="cuda", dtype=torch.bfloat16)
    gamma, at = torch.rand(N, device="cuda") + 0.5, _picked(M)
    args = [t[at].contiguous() for t in (x, r)]
    rstd, y = torch.empty(M, device="cuda"), torch.empty_like(x)
    q, s = torch.empty(M, N, dtype=torch.uint8, device="cuda"), torch.empty(M, 96, dtype=torch.uint8, device="cuda")
    C.compass_rms_forward(x, gamma, y, rstd, residual=r, h=r, y8=q, scale=s)     # the stream in place
    small = [torch.empty(len(at), N, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    rs, q2, s2 = torch.empty(len(at), device="cuda"), torch.empty(len(at), N, dtype=torch.uint8, device="cuda"), torch.empty(len(at), 96, dtype=torch.uint8, device="cuda")
    C.compass_rms_forward(args[0], gamma, small[1], rs, residual=args[1], h=small[0], y8=q2, scale=s2)
    for a, b in ((r[at], small[0]), (y[at], small[1]), (rstd[at], rs), (q[at], q2), (s[at], s2)):
        assert torch.equal(a, b)
    dx = x
    C.compass_rms_backward(y, r, gamma, rstd, dx, None, None, dh=r)
    want = torch.empty_like(small[0])
    C.compass_rms_backward(small[1], small[0], gamma, rs, want, None, None, dh=small[0])
    assert torch.equal(dx[at], want)


@pytest.mark.parametrize("M,N,K", [(262149, 72, 8208), (40000, 54001, 32), (8, 262149, 8208), (300, 262149, 8208)])
def test_wide_product(M, N, K):
    torch = _torch()
    (qa, sa), (qw, sw) = _rows(M, K, 5), _rows(N, K, 6)
    c = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
    C.compass_fp8_gemm(qa, sa, qw, sw, c, _scratch(C.compass_fp8_gemm_workspace(M, N, K)))
    am, an = _picked(M, 60 if M > 100 else M - 1) % M, _picked(N, 60)
    va, vw = _values(qa[am], sa[am]), _values(qw[an], sw[an])
    ref, mag = va @ vw.T, va.abs() @ vw.abs().T
    _within(c[am][:, an], ref, ref.abs() * U8 + (K * U24 * mag + 7 * 2.0 ** -13 * _cut(va, vw)) * (1 + U8))


@pytest.mark.parametrize("M,N,K", [(262149, 8, 8208), (262149, 8200, 16), (3, 131080, 16400)])
def test_wide_weight_gradient(M, N, K):
    torch = _torch()
    dy = (1e-3 * torch.randn(M, N, device="cuda", dtype=torch.bfloat16))
    q, s = _rows(M, K, 7)
    dw = torch.empty(N, K, device="cuda")
    C.compass_fp8_wgrad(dy, q, s, dw, _scratch(C.compass_fp8_wgrad_workspace(M, N, K)))
    an, ak = _picked(N, 60) % N, _picked(K, 60) % K
    step = torch.exp2(s.double() - 127)[:, (ak // 128)]
    v = q[:, ak].view(torch.float8_e4m3fn).double() * step
    d = dy[:, an].double()
    ref, mag = d.T @ v, d.abs().T @ v.abs()
    _within(dw[an][:, ak], ref, ref.abs() * U24 + M * U24 * mag)
