"""The binding where torch has no 8-bit types (no GPU): operators without 8-bit
operands are as before, 8-bit operands are their raw patterns."""
import pytest

from paper_2609_10549_amd import compass as C


@pytest.mark.parametrize("missing", [("float8_e8m0fnu",), ("float8_e8m0fnu", "float8_e4m3fn")])
def test_the_kinds_of_operands_without_8_bit_types(monkeypatch, missing):
    import torch
    whole = C._Kinds()
    for name in missing:
        monkeypatch.delattr(torch, name)
    k = C._Kinds()
    assert (k.bits, k.elements, k.float, k.index) == (whole.bits, whole.elements, whole.float, whole.index)
    assert k.scale == (torch.uint8,) and torch.uint8 in k.eight
    assert set(k.eight) < set(whole.eight) or "float8_e4m3fn" not in missing
