"""The operators at a model's ends without a GPU: the oracle's gradients against
differences of its forward pass, the cross entropy's plans over a grid of sizes
(tests/xent_plan_check.cpp), and what the entry points refuse before they
enqueue anything."""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest

from oracle import model_ends as E
from paper_2609_10549_amd import compass as C

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "..", "paper_2609_10549_amd", "csrc")


# -------------------------------------------------------------------- the oracle
def test_xent_gradient_is_the_loss_derivative():
    rng = np.random.default_rng(1)
    H, W = rng.standard_normal((6, 5)), rng.standard_normal((11, 5))
    t = np.array([0, 3, -100, 10, 3, 7])
    g = rng.standard_normal(6)
    lse = E.xent_forward(H, W, t)[0]
    dH, dW = E.xent_backward(H, W, t, lse, g)
    f = lambda h, w: (E.xent_forward(h, w, t)[2] * g).sum()  # noqa: E731
    for _ in range(5):
        D, G, e = rng.standard_normal(H.shape), rng.standard_normal(W.shape), 1e-6
        assert abs((dH * D).sum() - (f(H + e * D, W) - f(H - e * D, W)) / (2 * e)) < 1e-7
        assert abs((dW * G).sum() - (f(H, W + e * G) - f(H, W - e * G)) / (2 * e)) < 1e-7
    assert not dH[2].any()


def test_xent_shards_join_to_the_whole():
    rng = np.random.default_rng(2)
    H, W = rng.standard_normal((7, 4)), rng.standard_normal((12, 4))
    t = np.array([0, 5, 11, -1, 6, 3, 8])
    lse, _, loss = E.xent_forward(H, W, t)
    parts = [E.xent_forward(H, W[q * 3:q * 3 + 3], t, q * 3) for q in range(4)]
    joined = np.log(sum(np.exp(p[0]) for p in parts))
    assert np.allclose(joined, lse, atol=1e-13)
    assert np.allclose(np.where(t < 0, 0, joined - sum(p[1] for p in parts)), loss, atol=1e-13)
    g = rng.standard_normal(7)
    dH, dW = E.xent_backward(H, W, t, lse, g)
    shards = [E.xent_backward(H, W[q * 3:q * 3 + 3], t, lse, g, q * 3) for q in range(4)]
    assert np.allclose(sum(s[0] for s in shards), dH, atol=1e-13)
    assert np.allclose(np.vstack([s[1] for s in shards]), dW, atol=1e-13)


def test_norm_gradient_is_the_derivative():
    rng = np.random.default_rng(3)
    x, g, b, D = rng.standard_normal((4, 9)), rng.standard_normal(9), rng.standard_normal(9), rng.standard_normal((4, 9))
    _, mean, rstd = E.norm_forward(x, g, b, 1e-3)
    dx, dg, db = E.norm_backward(D, x, g, mean, rstd)
    f = lambda a, p, q: (E.norm_forward(a, p, q, 1e-3)[0] * D).sum()  # noqa: E731
    for _ in range(5):
        V, P, e = rng.standard_normal(x.shape), rng.standard_normal(9), 1e-6
        assert abs((dx * V).sum() - (f(x + e * V, g, b) - f(x - e * V, g, b)) / (2 * e)) < 1e-7
        assert abs((dg * P).sum() - (f(x, g + e * P, b) - f(x, g - e * P, b)) / (2 * e)) < 1e-7
        assert abs((db * P).sum() - (f(x, g, b + e * P) - f(x, g, b - e * P)) / (2 * e)) < 1e-7


def test_embed_gradient_is_the_transpose_of_the_lookup():
    rng = np.random.default_rng(4)
    ids = np.array([3, 7, 3, 1, -1, 9, 4])
    table, dy = rng.standard_normal((6, 5)), rng.standard_normal((7, 5))
    y = E.embed_forward(ids, table, 1.5, 2)
    assert not y[[3, 4, 5]].any()
    assert abs((y * dy).sum() - (E.embed_backward(ids, dy, 6, 1.5, 2) * table).sum()) < 1e-12


# --------------------------------------------------------------------- the plans
@pytest.mark.skipif(shutil.which("g++") is None, reason="needs a host C++ compiler")
def test_xent_plans_cover_their_products_and_the_gpu_tests_reach_every_tile(tmp_path):
    from tests.test_gpu_model_ends import XENT, XENT_TILES
    exe = tmp_path / "xent_plan_check"
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", f"-I{CSRC}", "-o", str(exe),
                    os.path.join(HERE, "xent_plan_check.cpp")], check=True)
    sizes = [f"{M},{V},{K},0" for M, V, K in XENT + XENT_TILES]
    out = subprocess.run([str(exe)] + sizes, capture_output=True, text=True, timeout=120)
    assert out.returncode == 0, out.stdout + out.stderr
    lines = out.stdout.split("\n")
    assert lines[0].startswith("ok ") and int(lines[0].split()[1]) > 5000
    reached = {ln for ln in lines[1:] if ln and not ln.startswith("any ")}
    used = {ln[4:] for ln in lines if ln.startswith("any ")}
    assert used - reached == set()


def test_workspaces_grow_with_what_they_hold():
    assert C.compass_xent_workspace(1, 1, 8) == 16     # two parts of one row
    whole = C.compass_xent_workspace(4096, 30000, 1024, backward=True)
    pieces = C.compass_xent_workspace(4096, 30000, 1024, backward=True, piece=4096)
    assert whole >= 4096 * 30000 * 2 and pieces < 4096 * 4096 * 2 + 4096 * 1024 * 4 * 33 + 1024 and pieces < whole
    assert C.compass_xent_workspace(1 << 20, 1 << 20, 512, backward=True) < (8 << 30)    # a piece, not the vocabulary
    assert C.compass_norm_workspace(1, 100) == 800 and C.compass_norm_workspace(10 ** 6, 100) == 256 * 800
    assert C.compass_embed_workspace(31, 10, 8) < C.compass_embed_workspace(32 * 32, 10, 8)


# ------------------------------------------------------------------ the refusals
P, Q = 4096, 4098     # an aligned address and one that is not aligned to 16 bytes


def test_xent_refusals_before_enqueue():
    lib = C.lib()
    fwd = lambda M=4, V=8, K=8, H=P, W=P, t=P, v0=0, lse=P, tl=P, ws=P, n=1 << 20: lib.compass_xent_forward(  # noqa: E731
        M, V, K, H, W, t, v0, lse, tl, None, ws, n, None)
    bwd = lambda M=4, V=8, K=8, H=P, W=P, t=P, v0=0, lse=P, g=P, dH=P, dW=P, piece=0, ws=P, n=1 << 20: (  # noqa: E731
        lib.compass_xent_backward(M, V, K, H, W, t, v0, lse, g, dH, dW, piece, ws, n, None))
    for call in (fwd, bwd):
        for kw in (dict(M=0), dict(V=0), dict(K=0), dict(K=12), dict(M=-1), dict(H=None), dict(W=None), dict(t=None),
                   dict(lse=None), dict(ws=None), dict(H=Q), dict(W=Q), dict(ws=Q), dict(v0=-1), dict(n=15)):
            assert call(**kw) == C.ERR_INVALID, kw
        for kw in (dict(M=(1 << 20) + 1), dict(V=(1 << 24) + 1), dict(K=(1 << 17) + 8)):
            assert call(**kw) == C.ERR_UNSUPPORTED, kw
    assert fwd(tl=None) == C.ERR_INVALID
    for kw in (dict(g=None), dict(dH=None), dict(dW=None), dict(dH=Q), dict(dW=Q), dict(piece=-1)):
        assert bwd(**kw) == C.ERR_INVALID, kw
    assert "need" in C.compass_last_error() or "piece" in C.compass_last_error()
    for args in ((0, 4), (2, 0)):
        assert lib.compass_xent_join(*args, P, P, P, P, P, None) == C.ERR_INVALID
    assert lib.compass_xent_join(2, 4, P, P, None, P, P, None) == C.ERR_INVALID
    out = ctypes.c_size_t()
    assert lib.compass_xent_workspace(4, 8, 8, 1, -1, ctypes.byref(out)) == C.ERR_INVALID
    assert lib.compass_xent_workspace(4, 8, 8, 0, 0, None) == C.ERR_INVALID
    # 256 rows of a piece over 1 GiB of dz (as the library's own choice is not)
    assert lib.compass_xent_workspace(256, 1 << 24, 8, 1, (1 << 21) + 64, ctypes.byref(out)) == C.ERR_UNSUPPORTED
    assert bwd(M=256, V=1 << 24, piece=(1 << 21) + 64, n=1 << 40) == C.ERR_UNSUPPORTED
    for M in (1, 16, 255, 256, 4096, 1 << 20):
        assert lib.compass_xent_workspace(M, 1 << 24, 8, 1, 0, ctypes.byref(out)) == C.OK
    with pytest.raises(C.CompassError):
        C.compass_xent_workspace(4, 8, 9)


def test_norm_refusals_before_enqueue():
    lib = C.lib()
    fwd = lambda M=4, N=8, d=C.F32, p=C.F32, x=P, ldx=8, g=P, b=P, eps=1e-5, y=P, ldy=8, mean=P, rstd=P: (  # noqa: E731
        lib.compass_norm_forward(M, N, d, p, x, ldx, g, b, eps, y, ldy, mean, rstd, None))
    bwd = lambda M=4, N=8, d=C.F32, p=C.F32, dy=P, lddy=8, x=P, ldx=8, g=P, mean=P, rstd=P, dx=P, lddx=8, dg=P, db=P, ws=P, n=1 << 20: (  # noqa: E731,E501
        lib.compass_norm_backward(M, N, d, p, dy, lddy, x, ldx, g, mean, rstd, dx, lddx, dg, db, ws, n, None))
    for call in (fwd, bwd):
        for kw in (dict(M=0), dict(N=0), dict(d=2), dict(p=-1), dict(x=None), dict(mean=None), dict(rstd=None),
                   dict(ldx=7), dict(x=Q), dict(g=Q)):
            assert call(**kw) == C.ERR_INVALID, kw
        assert call(M=(1 << 21) + 1) == C.ERR_UNSUPPORTED
        assert call(N=16385, **({"ldx": 16385, "ldy": 16385} if call is fwd else {"ldx": 16385})) == C.ERR_UNSUPPORTED
    for kw in (dict(y=None), dict(ldy=7), dict(eps=-1.0), dict(eps=float("nan")), dict(y=Q), dict(b=Q)):
        assert fwd(**kw) == C.ERR_INVALID, kw
    for kw in (dict(dy=None), dict(dx=None), dict(lddy=7), dict(lddx=7), dict(dy=Q), dict(dx=Q), dict(ws=None),
               dict(ws=Q), dict(n=63), dict(dg=None, n=63), dict(db=None, ws=None)):
        assert bwd(**kw) == C.ERR_INVALID, kw


def test_embed_refusals_before_enqueue():
    lib = C.lib()
    fwd = lambda T=4, V=8, K=8, d=C.F32, ids=P, v0=0, table=P, ldt=8, y=P, ldy=8: lib.compass_embed_forward(  # noqa: E731
        T, V, K, d, ids, v0, table, ldt, 1.0, y, ldy, None)
    bwd = lambda T=4, V=8, K=8, d=C.F32, g=C.F32, ids=P, v0=0, dy=P, ldy=8, dt=P, ldt=8, ws=P, n=1 << 20: (  # noqa: E731
        lib.compass_embed_backward(T, V, K, d, g, ids, v0, dy, ldy, 1.0, dt, ldt, 0, ws, n, None))
    for call in (fwd, bwd):
        for kw in (dict(T=0), dict(V=0), dict(K=0), dict(d=3), dict(ids=None), dict(v0=-1), dict(ldt=7), dict(ldy=7)):
            assert call(**kw) == C.ERR_INVALID, kw
        for kw in (dict(T=(1 << 20) + 1), dict(V=(1 << 24) + 1), dict(K=(1 << 20) + 1)):
            assert call(**kw) == C.ERR_UNSUPPORTED, kw
    for kw in (dict(table=None), dict(y=None), dict(table=Q), dict(y=Q)):
        assert fwd(**kw) == C.ERR_INVALID, kw
    for kw in (dict(g=-1), dict(dy=None), dict(dt=None), dict(ws=None), dict(ws=Q), dict(dy=Q), dict(dt=Q), dict(n=100)):
        assert bwd(**kw) == C.ERR_INVALID, kw


def test_binding_refuses_wrong_operands():
    import torch
    f32, bf = torch.float32, torch.bfloat16
    H, W, t = torch.zeros(4, 8, dtype=bf), torch.zeros(6, 8, dtype=bf), torch.zeros(4, dtype=torch.int64)
    row, ws = torch.zeros(4), torch.zeros(1 << 16, dtype=torch.uint8)
    for bad, what in (((H.float(), W, t, row, row, row), "H: torch.float32"), ((H, W[:, :4], t, row, row, row), "W: shape"),
                      ((H.half(), W, t, row, row, row), "H: torch.float16"), ((H, W, t.int(), row, row, row), "target"),
                      ((H, W, t, row[:3], row, row), "lse"), ((H, W, t, row, row, row.double()), "loss")):
        with pytest.raises(ValueError, match=what):
            C.compass_xent_forward(*(meta(x) for x in bad), ws)
    with pytest.raises(ValueError, match="H: must be on the GPU"):
        C.compass_xent_forward(H, W, t, row, row, row, ws)
    with pytest.raises(ValueError, match="workspace"):
        C.compass_xent_forward(*(meta(x) for x in (H, W, t, row, row, row)), ws)
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError, match="y: torch.bfloat16"):
        C.compass_norm_forward(meta(x), None, None, meta(x.to(bf)), meta(row), meta(row))
    with pytest.raises(ValueError, match="one type"):
        C.compass_norm_forward(meta(x), meta(x[0]), meta(x[0].to(bf)), meta(x), meta(row), meta(row))
    with pytest.raises(ValueError, match="contiguous within rows"):
        C.compass_norm_forward(meta(x.T), None, None, meta(torch.zeros(8, 4)), meta(row), meta(row))
    with pytest.raises(ValueError, match="workspace"):
        C.compass_embed_backward(meta(t), meta(x), meta(torch.zeros(6, 8, dtype=f32)), None)
    with pytest.raises(ValueError, match="ids: torch.int32"):
        C.compass_embed_forward(meta(t.int()), meta(torch.zeros(6, 8)), meta(x))


class meta:
    """A tensor that says it is on the GPU: its checks run, its address is never
    used (every call here is refused first)."""

    def __init__(self, x):
        self._x = x
        self.is_cuda = True

    def __getattr__(self, name):
        return getattr(self._x, name)
