"""What the built library's kernels ask of the runtime, from the code object's
metadata: none may use private memory (spilled registers), for which the runtime
would have to provide scratch behind a call that allocates nothing."""
import struct

import pytest

from paper_2609_10549_amd import compass as C

msgpack = pytest.importorskip("msgpack")

MAGIC = b"__CLANG_OFFLOAD_BUNDLE__"


def _code_objects(blob):
    """The device ELF images of the library's fat binaries."""
    at = blob.find(MAGIC)
    while at >= 0:
        n, = struct.unpack_from("<Q", blob, at + 24)
        p = at + 32
        for _ in range(n):
            off, size, length = struct.unpack_from("<QQQ", blob, p)
            target = blob[p + 24:p + 24 + length].decode()
            p += 24 + length
            if "gfx950" in target and size:
                yield blob[at + off:at + off + size]
        at = blob.find(MAGIC, at + 24)


def _kernels(elf):
    """The kernels of a code object: its AMDGPU metadata note (type 32)."""
    shoff, = struct.unpack_from("<Q", elf, 40)
    entsize, count = struct.unpack_from("<HH", elf, 58)
    for i in range(count):
        kind, = struct.unpack_from("<I", elf, shoff + i * entsize + 4)
        off, size = struct.unpack_from("<QQ", elf, shoff + i * entsize + 24)
        if kind != 7:   # SHT_NOTE
            continue
        p = off
        while p < off + size:
            name, desc, typ = struct.unpack_from("<III", elf, p)
            d = p + 12 + (name + 3) // 4 * 4
            if typ == 32:
                yield from msgpack.unpackb(elf[d:d + desc])["amdhsa.kernels"]
            p = d + (desc + 3) // 4 * 4


@pytest.fixture(scope="module")
def kernels():
    with open(C.LIB_PATH, "rb") as f:
        blob = f.read()
    found = [k for elf in _code_objects(blob) for k in _kernels(elf)]
    assert len(found) > 100
    return found


@pytest.mark.parametrize("family", ["tile_kernel", "norm_", ""])
def test_no_kernel_uses_private_memory(kernels, family):
    mine = [k for k in kernels if family in k[".name"]]
    assert mine
    bad = {k[".name"]: k[".private_segment_fixed_size"] for k in mine
           if k[".private_segment_fixed_size"] or k.get(".vgpr_spill_count") or k.get(".uses_dynamic_stack")}
    assert not bad, bad
