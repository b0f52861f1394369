"""LDS of the distillation kernels as they were compiled: behind what a kernel declares itself lie the teacher's tables and kept pieces, which it clears, writes and reads by 16 bytes."""
import os
import re
import struct

import msgpack

import paper_2503_01840_amd as E


def _kernels():
    """name -> metadata of the library's gfx950 kernels: the notes of the code objects in it (type 32, MessagePack)."""
    if not os.path.exists(E.LIB_PATH):
        from paper_2503_01840_amd.build import build_library
        build_library()
    data = open(E.LIB_PATH, "rb").read()
    found = {}
    for m in re.finditer(rb"AMDGPU\0\0", data):
        name, size, kind = struct.unpack_from("<III", data, max(0, m.start() - 12))
        if name == 7 and kind == 32:
            for k in msgpack.unpackb(data[m.end():m.end() + size])["amdhsa.kernels"]:
                found[k[".name"]] = k
    return found


def test_memory_behind_a_kernels_own_starts_at_16_bytes():
    kernels = {n: k for n, k in _kernels().items() if re.search("distill_(loss|grad|step)_kernel", n)}
    assert sum("step_kernel" in n for n in kernels) == 18 and sum("grad_kernel" in n for n in kernels) == 24
    for n, k in kernels.items():
        assert k[".group_segment_fixed_size"] % 16 == 0, n
        # 1024 entries: 16 bytes each and 2048 places of 4; 8 pieces of 16 bytes to each of 1024 threads where rows are kept there
        kept = 8 * 1024 * 16 if re.search("step_kernelI[tf]Li1024ELi16ELi8E", n) else 0
        assert k[".group_segment_fixed_size"] + 1024 * 16 + 2048 * 4 + kept <= 160 * 1024, n
