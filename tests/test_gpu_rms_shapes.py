"""The root-mean-square norm in every shape of its kernels (threads per row, vectors per
thread, aligned and loose rows), at the longest and the shortest row of each, over
several rows per group of the backward pass and a last one that only some groups have,
against fp64 on the GPU. Bounds as in test_gpu_eight_bits.py."""
from __future__ import annotations

import pytest

from paper_2609_10549_amd import compass as C

pytestmark = pytest.mark.gpu

U = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
U24 = 2.0 ** -24
EPS = 1e-5
VECTOR = {"bf16": 8, "f32": 4}
# threads per row and vectors each, in the order in which a row takes the first that holds it
FORWARD = [(64, 1), (64, 2), (256, 1), (256, 2), (512, 2), (1024, 2), (1024, 4)]
BACKWARD = [(64, 1), (64, 2), (128, 2), (192, 2), (256, 2), (384, 2), (512, 2), (768, 2), (1024, 2), (1024, 3), (1024, 4)]
LONGEST = 16384


def _cases(shapes):
    for dtype, v in VECTOR.items():
        below = 0
        for threads, vectors in shapes:
            most = threads * vectors * v
            if most > LONGEST:
                continue
            yield dtype, threads, vectors, False, most
            yield dtype, threads, vectors, True, below + 1
            below = most


def _torch():
    import torch
    return torch


def _gen(seed):
    torch = _torch()
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return lambda *s: torch.randn(*s, generator=g, device="cuda")


def _weights(n, N, dtype):
    """A weight of the rows' type, one of the other type, none."""
    torch = _torch()
    one = 1.0 + 0.2 * n(N)
    types = (torch.bfloat16, torch.float32) if dtype == "bf16" else (torch.float32, torch.bfloat16)
    return [one.to(t) for t in types] + [None]


def _within(name, got, ref, tol):
    over = (got.double() - ref).abs() - tol
    assert _torch().isfinite(got).all() and float(over.max()) <= 0, f"{name}: {int((over > 0).sum())} out of bound by up to {float(over.max()):.3g}"


@pytest.mark.parametrize("dtype,threads,vectors,loose,N", _cases(FORWARD))
def test_forward(dtype, threads, vectors, loose, N):
    torch = _torch()
    M, n = 2 * max(256, threads) // threads + 1, _gen(N)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    x, r = n(M, N).to(dt), (2 * n(M, N)).to(dt)
    for gamma in _weights(n, N, dtype):
        h, y, y2 = (torch.full((M, N), float("nan"), dtype=dt, device="cuda") for _ in range(3))
        rstd = torch.full((M,), float("nan"), device="cuda")
        q = torch.full((M, N), 0x7F, dtype=torch.uint8, device="cuda")
        s = torch.full((M, C.compass_fp8_scale_cols(N)), 255, dtype=torch.uint8, device="cuda")
        C.compass_rms_forward(x, gamma, y, rstd, residual=r, h=h, eps=EPS)
        assert torch.equal(h, (x.float() + r.float()).to(dt))
        d = h.double()
        want = 1.0 / torch.sqrt(d.square().mean(1) + EPS)
        rel = (N + 8) * U24
        _within("rstd", rstd, want, want * rel)
        ref = d * want[:, None] * (1.0 if gamma is None else gamma.double())
        _within("y", y, ref, ref.abs() * (U[dtype] + rel + 4 * U24))
        # the same with the 8 bits, which are those of the fp32 values: of y where y holds them whole
        C.compass_rms_forward(x, gamma, y2, rstd, residual=r, h=h, y8=q, scale=s, eps=EPS)
        assert torch.equal(y, y2)
        if dtype == "f32":
            q2, s2 = torch.empty_like(q), torch.empty_like(s)
            C.compass_fp8_quant(y, q2, s2)
            assert torch.equal(q, q2) and torch.equal(s, s2)
        else:
            step = torch.exp2(s.double() - 127).repeat_interleave(128, dim=1)[:, :N]
            v = q.view(torch.float8_e4m3fn).double() * step
            _within("y8", v, ref, torch.maximum(ref.abs() * 2.0 ** -4, step * 2.0 ** -10) + 1.1 * ref.abs() * (rel + 4 * U24))


def test_forward_at_the_ends_of_what_an_fp32_sum_holds():
    torch = _torch()
    N = 1024
    x = _gen(5)(6, N)
    x[0] *= 2.0 ** 55                  # inside: |h| up to 2^58, the sum below 2^126
    x[1] = 2.0 ** 70                   # its square is beyond
    x[2] = -2.0 ** 63 + 2.0 ** 40      # only the sum is
    x[3] *= 2.0 ** -55                 # inside: squares from 2^-125
    x[3][x[3].abs() < 2.0 ** -60] = 2.0 ** -58
    x[4] = 0.0
    y, rstd = torch.full((6, N), float("nan"), device="cuda"), torch.full((6,), float("nan"), device="cuda")
    q = torch.full((6, N), 0x7F, dtype=torch.uint8, device="cuda")
    s = torch.full((6, C.compass_fp8_scale_cols(N)), 255, dtype=torch.uint8, device="cuda")
    C.compass_rms_forward(x, None, y, rstd, y8=q, scale=s, eps=0.0)
    for m in (0, 3, 5):
        want = 1.0 / torch.sqrt(x[m].double().square().mean())
        _within("rstd", rstd[m], want, want * (N + 8) * U24)
        _within("y", y[m], x[m].double() * want, (x[m].double() * want).abs() * (N + 13) * U24)
    assert (rstd[1:3] == 0).all() and (y[1:3] == 0).all() and (q[1:3] & 127 == 0).all()
    assert torch.isinf(rstd[4]) and torch.isnan(y[4]).all() and (q[4] & 127 == 127).all()
    C.compass_rms_forward(x, None, y, rstd, y8=q, scale=s, eps=EPS)
    assert (y[4] == 0).all() and (q[4] == 0).all() and torch.isfinite(rstd[3:]).all()


def _check_backward(dy, h, gamma, rstd, dh, dtype):
    torch = _torch()
    M, N = h.shape
    dx = torch.full((M, N), float("nan"), dtype=h.dtype, device="cuda")
    dgamma = torch.full((N,), float("nan"), device="cuda")
    ws = torch.full((C.compass_rms_workspace(M, N),), 0xFF, dtype=torch.uint8, device="cuda")
    C.compass_rms_backward(dy, h, gamma, rstd, dx, dgamma, ws, dh=dh)
    d, r = dy.double(), rstd.double()[:, None]
    hh = h.double() * r
    a = d if gamma is None else d * gamma.double()
    extra = 0.0 if dh is None else dh.double()
    ref = extra + r * (a - hh * (a * hh).mean(1, keepdim=True))
    inner = (a.abs() * hh.abs()).mean(1, keepdim=True)
    off = U24 * (abs(extra) + r * (6 * a.abs() + hh.abs() * (N + 8) * inner))
    _within("dx", dx, ref, ref.abs() * (U[dtype] + U24) + off * (1 + U[dtype]))
    _within("dgamma", dgamma, (d * hh).sum(0), (M + 8) * U24 * (d * hh).abs().sum(0))


@pytest.mark.parametrize("dtype,threads,vectors,loose,N", _cases(BACKWARD))
def test_backward_over_several_rows_of_a_group(dtype, threads, vectors, loose, N):
    torch = _torch()
    rows = max(1, 1024 // threads)               # groups of a workgroup, at most
    M, n = 2 * 256 * rows + 256 * rows // 2 + 1, _gen(N + 1)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    h, dy, dh = (2 * n(M, N)).to(dt), n(M, N).to(dt), n(M, N).to(dt)
    rstd = (h.float().square().mean(1) + EPS).rsqrt()
    for gamma in _weights(n, N, dtype):
        _check_backward(dy, h, gamma, rstd, dh if gamma is not None else None, dtype)


@pytest.mark.parametrize("dtype,M,N", [("bf16", 8192, 12288), ("f32", 1000, 4097), ("bf16", 1000, 4096), ("f32", 9001, 256)])
def test_backward_of_batches(dtype, M, N):
    torch = _torch()
    n, dt = _gen(M), torch.bfloat16 if dtype == "bf16" else torch.float32
    h, dy, dh = (2 * n(M, N)).to(dt), (1e-3 * n(M, N)).to(dt), (1e-3 * n(M, N)).to(dt)
    rstd = (h.float().square().mean(1) + EPS).rsqrt()
    _check_backward(dy, h, (1.0 + 0.2 * n(N)).to(dt), rstd, dh, dtype)


def test_weight_gradient_beyond_2_to_31_elements():
    torch = _torch()
    M, N = 180001, 12288
    n = _gen(1)
    h, dy = (torch.empty(M, N, dtype=torch.bfloat16, device="cuda").normal_() for _ in range(2))
    rstd, dgamma = 0.5 + n(M).abs(), torch.full((N,), float("nan"), device="cuda")
    ws = torch.full((C.compass_rms_workspace(M, N),), 0xFF, dtype=torch.uint8, device="cuda")
    C.compass_rms_backward(dy, h, None, rstd, torch.empty_like(dy), dgamma, ws)
    at = torch.cat([torch.arange(0, N, 331), torch.tensor([1, N - 2, N - 1])]).cuda()
    terms = dy[:, at].double() * h[:, at].double() * rstd.double()[:, None]
    _within("dgamma", dgamma[at], terms.sum(0), (M + 8) * U24 * terms.abs().sum(0))
