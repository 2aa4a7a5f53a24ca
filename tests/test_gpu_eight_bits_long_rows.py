"""Rows of more than 2^17 values: written across, read back, against the fp64 oracle. The
codes and the values that they stand for are exact."""
from __future__ import annotations

import numpy as np
import pytest

from oracle import eight_bits as E
from paper_2609_10549_amd import compass as C
from tests.test_gpu_eight_bits import Rows, _nan, _np, _same_codes, _spread_values, _type

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,K", [((1 << 17) + 1, 3), ((1 << 17) + 520, 65), (1 << 21, 2)])
def test_across_and_back(M, K, dtype):
    x = _spread_values(M, K, 11, dtype)
    out = Rows(K, M)
    C.compass_fp8_quant(x, out.q, out.scale, across=True)
    got, scale = out.numpy()
    want, want_scale = E.quant(_np(x).T)
    _same_codes(got, want, scale, want_scale)
    pad = K % 2     # rows of the values apart, and not on 16 bytes
    whole = _nan(K, M + pad, dtype=_type(dtype))
    C.compass_fp8_dequant(out.q, out.scale, whole[:, :M])
    import torch
    assert torch.equal(whole[:, :M].cpu(), torch.from_numpy(E.values(want, want_scale)).to(_type(dtype)))
    assert torch.isnan(whole[:, M:]).all()
    assert np.isfinite(_np(whole[:, :M])).all()
