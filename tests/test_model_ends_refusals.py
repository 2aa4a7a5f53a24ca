"""More of what the entry points at a model's ends refuse before they enqueue
anything: vocabulary ids beyond 64 bits."""
import pytest

from paper_2609_10549_amd import compass as C

P = 4096     # an aligned address
LAST = 2 ** 63 - 1


@pytest.mark.parametrize("v0", [LAST, LAST - 7, -1, -LAST - 1])
def test_ids_beyond_64_bits_are_refused(v0):
    lib = C.lib()
    V = 8
    for rc in (lib.compass_xent_forward(4, V, 8, P, P, P, v0, P, P, None, P, 1 << 20, None),
               lib.compass_xent_backward(4, V, 8, P, P, P, v0, P, P, P, P, 0, P, 1 << 20, None),
               lib.compass_xent_backward(4, V, 8, P, P, P, v0, P, P, P, P, 1, P, 1 << 20, None),
               lib.compass_embed_forward(4, V, 8, C.F32, P, v0, P, 8, 1.0, P, 8, None),
               lib.compass_embed_backward(4, V, 8, C.F32, C.F32, P, v0, P, 8, 1.0, P, 8, 0, P, 1 << 20, None)):
        assert rc == C.ERR_INVALID
        assert "v0" in C.compass_last_error()


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
    """Every entry point with operands that fit: (function, operands by name, the
    names of those whose sizes or rows it reads)."""
    import torch
    f32, i64 = torch.float32, torch.int64
    H, W, t, row = OnGpu(4, 8), OnGpu(6, 8), OnGpu(4, dtype=i64), OnGpu(4, dtype=f32)
    ws = OnGpu(8, dtype=torch.uint8)      # too small for any of them: refused by the library
    par = OnGpu(8, dtype=f32)
    return [(C.compass_xent_forward, dict(H=H, W=W, target=t, lse=row, tlogit=row, loss=row, workspace=ws), "H W"),
            (C.compass_xent_backward, dict(H=H, W=W, target=t, lse=row, grad=row, dH=H, dW=W, workspace=ws), "H W"),
            (C.compass_norm_backward, dict(dy=H, x=H, gamma=par, mean=row, rstd=row, dx=H, dgamma=par, dbeta=par,
                                           workspace=ws), "dy x dx"),
            (C.compass_embed_backward, dict(ids=t, dy=H, dtable=W, workspace=ws), "dy dtable")]


def test_the_binding_asks_for_tensors_where_it_reads_their_sizes():
    import torch
    row, par = OnGpu(4, dtype=torch.float32), OnGpu(8, dtype=torch.float32)
    calls = _calls() + [
        (C.compass_norm_forward, dict(x=OnGpu(4, 8), gamma=par, beta=par, y=OnGpu(4, 8), mean=row, rstd=row), "x y"),
        (C.compass_embed_forward, dict(ids=OnGpu(4, dtype=torch.int64), table=OnGpu(6, 8), y=OnGpu(4, 8)), "ids table y"),
        (C.compass_xent_join, dict(lse_parts=OnGpu(2, 4), tlogit_parts=OnGpu(2, 4), target=OnGpu(4), lse=row, loss=row),
         "lse_parts")]
    for f, operands, sized in calls:
        for name in sized.split():
            for other in (None, P):
                with pytest.raises(ValueError, match=f"^{name}: must be a tensor"):
                    f(**{**operands, name: other}, stream=0)
            if name not in ("y", "dx", "ids"):
                with pytest.raises(ValueError, match=f"^{name}: shape .*, expected"):
                    f(**{**operands, name: OnGpu(8)}, stream=0)
    f, operands, _ = calls[4]
    for other in (dict(gamma=P), dict(beta=P), dict(gamma=None, beta=P), dict(gamma=P, beta=P)):
        with pytest.raises(ValueError, match="^gamma, beta: must be tensors"):
            f(**{**operands, **other}, stream=0)


def test_the_binding_takes_plain_addresses_elsewhere():
    """They reach the library, which here refuses the workspace."""
    for f, operands, sized in _calls():
        plain = {k: v if k in sized.split() or k in ("workspace", "gamma") else P for k, v in operands.items()}
        with pytest.raises(C.CompassError, match="workspace of 8 bytes"):
            f(**plain, stream=0)
    with pytest.raises(ValueError, match="workspace"):
        f(**{**plain, "workspace": P}, stream=0)
