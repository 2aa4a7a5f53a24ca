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
