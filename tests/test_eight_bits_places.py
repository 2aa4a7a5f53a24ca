"""Where the operands of the MLP in 8 bits lie: each of them, and the stream, on the
current GPU. Without one, every call here is refused before the library is reached, or
reaches a library that only counts."""
import pytest

from paper_2609_10549_amd import compass as C
from tests import test_eight_bits_host as host


class Somewhere(host.OnGpu):
    """A tensor that says it is on GPU `at`."""
    at = 0

    def get_device(self):
        return self.at


class Stream:
    cuda_stream = 1 << 20

    def __init__(self, device_index):
        self.device_index = device_index


def _calls(monkeypatch):
    """Entry points with operands on GPU 0, the current one, and the calls that got
    through."""
    class Library:
        reached = []

        def __getattr__(self, name):
            return lambda *a: self.reached.append(name) or 0
    library = Library()
    library.reached.clear()
    monkeypatch.setattr(C, "_current_device", lambda: 0)
    monkeypatch.setattr(C, "_lib", library)
    monkeypatch.setattr(host, "OnGpu", Somewhere)
    calls = host._calls()
    return calls, library.reached


def test_each_operand_on_another_gpu_is_refused(monkeypatch):
    calls, reached = _calls(monkeypatch)
    for f, operands in calls.items():
        f(**operands, stream=0)
        assert reached.pop() == f.__name__ and not reached
        for what, x in operands.items():
            away = Somewhere(*x.shape, dtype=x.dtype)
            away.at = 2
            others = "2, the current one is 0|0, the current one is 2"
            with pytest.raises(ValueError, match=f"on GPU ({others})"):
                f(**{**operands, what: away}, stream=0)
            assert not reached, what


def test_a_stream_of_another_gpu_is_refused(monkeypatch):
    calls, reached = _calls(monkeypatch)
    for f, operands in calls.items():
        with pytest.raises(ValueError, match="stream on GPU 1, the current one is 0"):
            f(**operands, stream=Stream(1))
        assert not reached
        f(**operands, stream=Stream(0))
        f(**operands, stream=1 << 20)      # a plain address is the caller's
        assert len(reached) == 2
        reached.clear()


def test_operands_that_are_absent_or_addresses_have_no_place(monkeypatch):
    calls, reached = _calls(monkeypatch)
    norm, back = calls[C.compass_rms_forward], calls[C.compass_rms_backward]
    C.compass_rms_forward(norm["x"], None, norm["y"], norm["rstd"], stream=0)
    C.compass_rms_backward(back["dy"], back["h"], None, 4096, back["dx"], None, None, stream=0)
    gemm = calls[C.compass_fp8_gemm]
    C.compass_fp8_gemm(**{**gemm, "A_scale": 4096, "C": 8192, "workspace": None}, stream=0)
    assert len(reached) == 3


@pytest.mark.gpu
def test_streams_of_the_current_gpu_are_taken():
    import torch
    x = torch.arange(1, 601, device="cuda").view(2, 300).float()
    q, s = torch.empty(2, 300, dtype=torch.uint8, device="cuda"), torch.empty(2, 4, dtype=torch.uint8, device="cuda")
    C.compass_fp8_quant(x, q, s)
    want = q.clone(), s.clone()
    own = torch.cuda.Stream()
    streams = [own, own.cuda_stream, torch.cuda.ExternalStream(own.cuda_stream), torch.cuda.default_stream(), torch.cuda.current_stream()]
    for stream in streams:
        q.zero_(), s.zero_()
        torch.cuda.synchronize()
        C.compass_fp8_quant(x, q, s, stream=stream)
        torch.cuda.synchronize()
        assert torch.equal(q, want[0]) and torch.equal(s, want[1])
