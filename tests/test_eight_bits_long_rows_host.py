"""The rows that quantising across writes are rows that reading back takes (no GPU: what
is refused for its size is refused before an operand is looked at)."""
import pytest

from paper_2609_10549_amd import compass as C
from tests.test_eight_bits_host import BIG, P, _dequant, _quant


@pytest.mark.parametrize("M,K", [(1 << 21, 1), (1 << 21, 1 << 17), ((1 << 17) + 1, 4), (1 << 17, 1 << 17)])
def test_what_is_written_across_can_be_read_back(M, K):
    for call, o in ((_quant, dict(M=M, K=K, ld=BIG, across=1, q=None)), (_dequant, dict(M=K, K=M, ld=BIG, q=None)),
                    (_quant, dict(M=M, K=K, ld=BIG, q=None)), (_dequant, dict(M=M, K=K, ld=BIG, q=None))):
        assert call(**o) == C.ERR_INVALID
        assert "required" in C.compass_last_error()


@pytest.mark.parametrize("M,K", [(1, (1 << 21) + 1), ((1 << 17) + 1, (1 << 17) + 1), ((1 << 21) + 1, 1), (1 << 18, 1 << 20)])
def test_longer_rows_and_more_of_them_are_refused(M, K):
    assert _dequant(M=M, K=K, ld=BIG, q=P) == C.ERR_UNSUPPORTED
    assert "at most" in C.compass_last_error()
