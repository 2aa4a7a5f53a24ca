"""What the entry points of the MLP in 8 bits refuse before they enqueue anything,
and the sizes they give (no GPU)."""
import ctypes
import os
import shutil
import subprocess

import pytest

from paper_2609_10549_amd import compass as C

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2609_10549_amd", "csrc")
P = 4096     # an aligned address
BIG = 1 << 40


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs a host C++ compiler")
def test_plans_cover_their_outputs_and_the_gpu_tests_reach_every_launch(tmp_path):
    from tests import test_gpu_eight_bits as small
    from tests import test_gpu_eight_bits_plans as plans
    exe = tmp_path / "fp8_plan_check"
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", f"-I{CSRC}", "-o", str(exe),
                    os.path.join(HERE, "fp8_plan_check.cpp")], check=True)
    sizes = [f"0,{M},{N},{K}" for M, N, K in small.PRODUCT + plans.PRODUCT]
    sizes += [f"1,{M},{N},{K}" for M, N, K in small.GRAD + plans.GRAD]
    out = subprocess.run([str(exe)] + sizes, capture_output=True, text=True, timeout=120)
    assert out.returncode == 0, out.stdout + out.stderr
    lines = out.stdout.split("\n")
    assert lines[0].startswith("ok ") and int(lines[0].split()[1]) > 8000
    reached = {ln for ln in lines[1:] if ln and not ln.startswith("any ")}
    used = {ln[4:] for ln in lines if ln.startswith("any ")}
    assert used - reached == set()


def test_scale_columns_are_whole_words():
    assert [C.compass_fp8_scale_cols(n) for n in (1, 128, 512, 513, 12288)] == [4, 4, 4, 8, 96]
    for n in (0, -5):
        with pytest.raises(C.CompassError, match="positive"):
            C.compass_fp8_scale_cols(n)
    with pytest.raises(C.CompassError, match="at most"):
        C.compass_fp8_scale_cols((1 << 21) + 1)
    assert C.lib().compass_fp8_scale_cols(8, None) == C.ERR_INVALID


def test_workspaces():
    assert C.compass_rms_workspace(1, 100) == 400 and C.compass_rms_workspace(10 ** 6, 100) == 256 * 400
    lib, out = C.lib(), ctypes.c_size_t()
    for f in (lib.compass_fp8_gemm_workspace, lib.compass_fp8_wgrad_workspace):
        assert f(8, 8, 16, ctypes.byref(out)) == C.OK
        assert f(8, 8, 16, None) == C.ERR_INVALID
        for sizes in ((0, 8, 16), (8, 0, 16), (8, 8, 0), (8, 8, 8), (-1, 8, 16)):
            assert f(*sizes, ctypes.byref(out)) == C.ERR_INVALID
        for sizes in (((1 << 20) + 1, 8, 16), (8, (1 << 20) + 8, 16), (8, 8, (1 << 17) + 16)):
            assert f(*sizes, ctypes.byref(out)) == C.ERR_UNSUPPORTED
    assert lib.compass_fp8_wgrad_workspace(8, 9, 16, ctypes.byref(out)) == C.ERR_INVALID
    assert lib.compass_fp8_gemm_workspace(8, 9, 16, ctypes.byref(out)) == C.OK


# entry point: operands that fit, by name; (change, words of the message)
def _rms_forward(**o):
    a = dict(M=4, N=8, d=C.F32, p=C.F32, x=P, ldx=8, r=P, ldr=8, g=P, eps=1e-5, h=P, ldh=8, y=P, ldy=8, y8=P, s=P,
             rstd=P) | o
    return C.lib().compass_rms_forward(a["M"], a["N"], a["d"], a["p"], a["x"], a["ldx"], a["r"], a["ldr"], a["g"], a["eps"],
                                       a["h"], a["ldh"], a["y"], a["ldy"], a["y8"], a["s"], a["rstd"], None)


def _rms_backward(**o):
    a = dict(M=4, N=8, d=C.F32, p=C.F32, dy=P, lddy=8, h=P, ldh=8, dh=P, lddh=8, g=P, rstd=P, dx=P, lddx=8, dg=P, ws=P,
             n=BIG) | o
    return C.lib().compass_rms_backward(a["M"], a["N"], a["d"], a["p"], a["dy"], a["lddy"], a["h"], a["ldh"], a["dh"],
                                        a["lddh"], a["g"], a["rstd"], a["dx"], a["lddx"], a["dg"], a["ws"], a["n"], None)


def _quant(**o):
    a = dict(M=4, K=8, d=C.F32, x=P, ld=8, across=0, q=P, s=P) | o
    return C.lib().compass_fp8_quant(a["M"], a["K"], a["d"], a["x"], a["ld"], a["across"], a["q"], a["s"], None)


def _dequant(**o):
    a = dict(M=4, K=8, d=C.F32, q=P, s=P, x=P, ld=8) | o
    return C.lib().compass_fp8_dequant(a["M"], a["K"], a["d"], a["q"], a["s"], a["x"], a["ld"], None)


def _gemm(**o):
    a = dict(M=4, N=8, K=16, A=P, sA=P, W=P, sW=P, c=P, ws=P, n=BIG) | o
    return C.lib().compass_fp8_gemm(a["M"], a["N"], a["K"], a["A"], a["sA"], a["W"], a["sW"], a["c"], a["ws"], a["n"], None)


def _wgrad(**o):
    a = dict(M=4, N=8, K=16, g=C.F32, dY=P, X=P, sX=P, dW=P, acc=0, ws=P, n=BIG) | o
    return C.lib().compass_fp8_wgrad(a["M"], a["N"], a["K"], a["g"], a["dY"], a["X"], a["sX"], a["dW"], a["acc"], a["ws"],
                                     a["n"], None)


INVALID = [
    (_rms_forward, [dict(M=0), dict(N=0), dict(M=-3)], "positive"),
    (_rms_forward, [dict(d=2), dict(p=-1)], "element type"),
    (_rms_forward, [dict(x=None), dict(rstd=None)], "required"),
    (_rms_forward, [dict(r=None), dict(h=None)], "residual and h come together"),
    (_rms_forward, [dict(y8=None), dict(s=None)], "y8 and scale come together"),
    (_rms_forward, [dict(y=None, y8=None, s=None)], "required"),
    (_rms_forward, [dict(ldx=7), dict(ldr=7), dict(ldh=7), dict(ldy=7), dict(ldx=-8)], "overlap"),
    (_rms_forward, [dict(eps=-1e-9), dict(eps=float("nan"))], "eps"),
    (_rms_forward, [dict(x=P + 2), dict(r=P + 1), dict(h=P + 2), dict(y=P + 3), dict(g=P + 2), dict(rstd=P + 2)], "aligned"),
    (_rms_forward, [dict(y8=P + 8), dict(s=P + 2)], "aligned"),
    (_rms_backward, [dict(M=0), dict(N=0)], "positive"),
    (_rms_backward, [dict(d=5), dict(p=5)], "element type"),
    (_rms_backward, [dict(dy=None), dict(h=None), dict(rstd=None), dict(dx=None)], "required"),
    (_rms_backward, [dict(lddy=7), dict(ldh=7), dict(lddh=7), dict(lddx=7)], "overlap"),
    (_rms_backward, [dict(dy=P + 2), dict(h=P + 2), dict(dh=P + 2), dict(dx=P + 2), dict(g=P + 2), dict(dg=P + 2)], "aligned"),
    (_rms_backward, [dict(ws=None), dict(ws=P + 8), dict(n=4 * 8 * 4 - 1)], "workspace"),
    (_quant, [dict(M=0), dict(K=0)], "positive"),
    (_quant, [dict(d=3)], "element type"),
    (_quant, [dict(across=2), dict(across=-1)], "across"),
    (_quant, [dict(x=None), dict(q=None), dict(s=None)], "required"),
    (_quant, [dict(ld=7), dict(ld=7, across=1)], "overlap"),
    (_quant, [dict(x=P + 2), dict(q=P + 8), dict(s=P + 1)], "aligned"),
    (_dequant, [dict(M=0), dict(K=-1)], "positive"),
    (_dequant, [dict(d=3)], "element type"),
    (_dequant, [dict(x=None), dict(q=None), dict(s=None)], "required"),
    (_dequant, [dict(ld=7)], "overlap"),
    (_dequant, [dict(x=P + 2), dict(q=P + 8), dict(s=P + 1)], "aligned"),
    (_gemm, [dict(M=0), dict(N=0), dict(K=0), dict(K=24)], "positive M, N and K"),
    (_gemm, [dict(A=None), dict(sA=None), dict(W=None), dict(sW=None), dict(c=None)], "required"),
    (_gemm, [dict(A=P + 8), dict(sA=P + 2), dict(W=P + 8), dict(sW=P + 1), dict(c=P + 8)], "aligned"),
    (_wgrad, [dict(M=0), dict(N=0), dict(K=0), dict(K=24), dict(N=12)], "positive M, N and K"),
    (_wgrad, [dict(g=2)], "element type"),
    (_wgrad, [dict(acc=2), dict(acc=-1)], "accumulate"),
    (_wgrad, [dict(dY=None), dict(X=None), dict(sX=None), dict(dW=None)], "required"),
    (_wgrad, [dict(dY=P + 8), dict(X=P + 8), dict(sX=P + 2), dict(dW=P + 8)], "aligned"),
]


@pytest.mark.parametrize("call,changes,words", INVALID, ids=lambda v: getattr(v, "__name__", None))
def test_invalid_arguments(call, changes, words):
    for change in changes:
        assert call(**change) == C.ERR_INVALID, change
        assert words in C.compass_last_error(), change


def test_sizes_beyond_the_limits():
    for rc in (_rms_forward(N=16385, ldx=16385, ldr=16385, ldh=16385, ldy=16385), _rms_forward(M=(1 << 21) + 1),
               _rms_backward(M=(1 << 21) + 1), _quant(K=(1 << 17) + 1, ld=BIG), _quant(M=(1 << 21) + 1),
               _dequant(M=(1 << 21) + 1), _gemm(M=(1 << 20) + 1), _gemm(N=(1 << 20) + 1), _gemm(K=(1 << 17) + 16),
               _wgrad(M=(1 << 20) + 1), _wgrad(N=(1 << 20) + 8), _wgrad(K=(1 << 17) + 16)):
        assert rc == C.ERR_UNSUPPORTED
        assert "most" in C.compass_last_error() or "beyond" in C.compass_last_error()


class OnGpu:
    """A tensor that says it is on the GPU: its checks run, its address is never
    used (every call here is refused first)."""

    def __init__(self, *shape, dtype=None):
        import torch
        self._x = torch.zeros(*shape, dtype=dtype or torch.bfloat16)
        self.is_cuda = True

    def __getattr__(self, name):
        return getattr(self._x, name)


def _calls():
    import torch
    u8, f32 = torch.uint8, torch.float32
    H, row, par = OnGpu(4, 16), OnGpu(4, dtype=f32), OnGpu(16, dtype=f32)
    q, s, w, sw = OnGpu(4, 16, dtype=u8), OnGpu(4, 4, dtype=u8), OnGpu(8, 16, dtype=u8), OnGpu(8, 4, dtype=u8)
    ws = OnGpu(16, dtype=u8)
    return {C.compass_fp8_quant: dict(x=H, x8=q, scale=s),
            C.compass_fp8_dequant: dict(x8=q, scale=s, x=H),
            C.compass_rms_forward: dict(x=H, gamma=par, y=H, rstd=row, residual=H, h=H, y8=q, scale=s),
            C.compass_rms_backward: dict(dy=H, h=H, gamma=par, rstd=row, dx=H, dgamma=par, workspace=ws, dh=H),
            C.compass_fp8_gemm: dict(A=q, A_scale=s, W=w, W_scale=sw, C=OnGpu(4, 8), workspace=ws),
            C.compass_fp8_wgrad: dict(dY=OnGpu(4, 8), X8=q, X_scale=s, dW=OnGpu(8, 16), workspace=ws)}


@pytest.mark.parametrize("name", ["quant", "dequant", "forward", "backward", "gemm", "wgrad"])
def test_the_binding_checks_shapes_types_and_places(name):
    import torch
    f, operands = next((f, o) for f, o in _calls().items() if f.__name__.endswith(name))
    for what, x in operands.items():
        if what == "workspace":
            bad = [torch.zeros(16, dtype=torch.uint8), 4096]
        elif what in ("gamma", "dgamma", "rstd"):
            bad = [OnGpu(5, dtype=torch.float32), torch.zeros(*x.shape), OnGpu(*x.shape, dtype=torch.float64)]
        else:
            bad = [OnGpu(x.shape[0], x.shape[1] + 1, dtype=x.dtype), OnGpu(*x.shape, dtype=torch.float64),
                   torch.zeros(*x.shape, dtype=x.dtype)]
            if what in ("x", "h") and name not in ("quant", "dequant"):
                bad = bad[1:]     # (its sizes are the call's)
            if x.dtype == torch.bfloat16:
                bad.append(OnGpu(*x.shape, dtype=torch.float16))
            if name in ("gemm", "wgrad") and x.dtype == torch.uint8:
                bad.append(OnGpu(*x.shape, dtype=torch.int8))
        for b in bad:
            with pytest.raises(ValueError):
                f(**{**operands, what: b}, stream=0)


def test_rows_of_8_bits_are_packed():
    import torch
    o = _calls()
    apart = OnGpu(4, 16, dtype=torch.uint8)
    apart._x = torch.zeros(4, 32, dtype=torch.uint8)[:, :16]
    for f, what in ((C.compass_fp8_quant, "x8"), (C.compass_fp8_gemm, "A"), (C.compass_fp8_wgrad, "X8")):
        with pytest.raises(ValueError, match="contiguous"):
            f(**{**o[f], what: apart}, stream=0)


def test_operands_whose_sizes_are_read_are_tensors():
    o = _calls()
    for f, names in ((C.compass_fp8_quant, "x"), (C.compass_fp8_dequant, "x"), (C.compass_rms_forward, "x"),
                     (C.compass_rms_backward, "h"), (C.compass_fp8_gemm, "A W"), (C.compass_fp8_wgrad, "dY X8 dW")):
        for n in names.split():
            for other in (None, P):
                with pytest.raises(ValueError, match="must be a tensor"):
                    f(**{**o[f], n: other}, stream=0)


def test_operands_on_another_gpu_are_refused(monkeypatch):
    class Away(OnGpu):
        def get_device(self):
            return 1
    monkeypatch.setattr(C, "_current_device", lambda: 0)
    for f, operands in _calls().items():
        away = {n: Away(*x.shape, dtype=x.dtype) for n, x in operands.items()}
        with pytest.raises(ValueError, match="on GPU 1, the current one is 0"):
            f(**away, stream=0)


def test_the_current_gpu_is_found_at_the_first_call(monkeypatch):
    import torch
    monkeypatch.setattr(C, "_current_device", None)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 3, raising=False)

    class Here(OnGpu):
        def get_device(self):
            return 3
    for _ in range(2):
        assert C._stream_by(Here(2, 2), 7) == 7
        with pytest.raises(ValueError, match="the current one is 3"):
            C._stream_by(OnGpu(2, 2), 7)
