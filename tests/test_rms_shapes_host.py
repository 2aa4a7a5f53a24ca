"""The shapes that the GPU tests of the root-mean-square norm take are all that the
built library has (no GPU)."""
import re

import pytest

from tests import test_gpu_rms_shapes as shapes
from tests.test_kernel_resources import kernels  # noqa: F401  (a fixture)

NAME = re.compile(r"rms_(forward|backward)_kernelI(.+?)Li(\d+)ELb([01])ELi(\d+)ELi(\d+)E")


@pytest.mark.parametrize("direction", ["forward", "backward"])
def test_every_shape_is_tested(kernels, direction):  # noqa: F811
    built = set()
    for k in kernels:
        found = NAME.search(k[".name"])
        if found and found[1] == direction:
            dtype = "f32" if found[2] == "f" else "bf16"
            assert int(found[3]) == shapes.VECTOR[dtype]
            built.add((dtype, int(found[5]), int(found[6]), found[4] == "1"))
    cases = list(shapes._cases(getattr(shapes, direction.upper())))
    assert {c[:4] for c in cases} == built and len(cases) == len(built)
    for dtype, threads, vectors, loose, N in cases:
        v = shapes.VECTOR[dtype]
        assert (N % v != 0) == loose and N <= threads * vectors * v
