"""What the built library's kernels keep outside of their registers, from the code objects' own metadata (CPU only)."""
import os
import re
import struct

import pytest

from paper_2605_02262_amd import build

msgpack = pytest.importorskip("msgpack")
MAGIC = b"__CLANG_OFFLOAD_BUNDLE__"


def _code_objects(data):
    at = data.find(MAGIC)
    while at >= 0:
        count, = struct.unpack_from("<Q", data, at + 24)
        entry = at + 32
        for _ in range(count):
            offset, size, n = struct.unpack_from("<QQQ", data, entry)
            if b"gfx950" in data[entry + 24:entry + 24 + n]:
                yield data[at + offset:at + offset + size]
            entry += 24 + n
        at = data.find(MAGIC, at + 24)


def _kernels(elf):
    """The metadata note of an ELF file (its owner's name, then MessagePack)."""
    sections, = struct.unpack_from("<Q", elf, 0x28)
    size, count = struct.unpack_from("<HH", elf, 0x3A)
    for i in range(count):
        kind, = struct.unpack_from("<I", elf, sections + i * size + 4)
        offset, length = struct.unpack_from("<QQ", elf, sections + i * size + 0x18)
        if kind != 7:                                                    # SHT_NOTE
            continue
        end = offset + length
        while offset < end:
            name, desc, note = struct.unpack_from("<III", elf, offset)
            body = offset + 12 + (name + 3) // 4 * 4
            if note == 32:                                               # NT_AMDGPU_METADATA
                return msgpack.unpackb(elf[body:body + desc], strict_map_key=False)["amdhsa.kernels"]
            offset = body + (desc + 3) // 4 * 4
    return []


def test_kernels_of_shared_caches():
    """k_shared waits for its vector instructions: scalars that it keeps in vector registers, and registers in scratch, are more of them.  (Scalars by the
    thirties took 1 to 2 % of its calls.)"""
    if not os.path.exists(build.LIB):
        build.build(verbose=False)
    with open(build.LIB, "rb") as f:
        kernels = [k for elf in _code_objects(f.read()) for k in _kernels(elf)]
    found = 0
    for k in kernels:
        m = re.search(r"k_sharedINS_\d+(\w+?)ELi(\d+)ELi(\d)", k[".name"])
        if not m:
            continue
        found += 1
        spilled = {("F32", "128"): 28, ("F16", "128"): 6 if m[3] == "4" else 0}.get((m[1], m[2]), 0)
        assert k[".sgpr_spill_count"] <= 7 and k[".vgpr_spill_count"] <= spilled, (m[0], k[".sgpr_spill_count"], k[".vgpr_spill_count"])
    assert found == 9
