"""Scratch memory of the built attention kernels on caches, from the code objects' metadata (no GPU needed)."""
import os
import re
import struct
import subprocess

import pytest

from paper_2605_08123_amd.build import LIB

from .test_kernel_registers import BUNDLE, READELF

# storage, queries, head dimension, blocks of rows, both walks: bytes a lane.  32 rows' results, two operands of P, and keys that wait for LDS while the
# next are in flight do not fit 256 registers; what is spilled are 24
SPILLS = {("DF16b", "DF16b", 128, 2, 0): 100}


def scratch(tmp_path):
    """{(storage, queries, D, NQ, both): bytes of scratch a lane} of ca_attn_kernel's instances, from every gfx950 code object in the library."""
    blob, found, at = open(LIB, "rb").read(), {}, -1
    while (at := blob.find(BUNDLE, at + 1)) >= 0:
        pos, n = at + len(BUNDLE) + 8, struct.unpack_from("<Q", blob, at + len(BUNDLE))[0]
        for _ in range(n):
            off, size, idlen = struct.unpack_from("<QQQ", blob, pos)
            ident = blob[pos + 24:pos + 24 + idlen].decode()
            pos += 24 + idlen
            if "gfx950" not in ident:
                continue
            obj = tmp_path / "device.o"
            obj.write_bytes(blob[at + off:at + off + size])
            notes = subprocess.run([READELF, "--notes", str(obj)], capture_output=True, text=True, check=True).stdout
            for m in re.finditer(r"\.name: +_Z\S*ca_attn_kernelI(\S+?)Li(\d+)ELi(\d+)ELb(\d)E\S*.*?\.private_segment_fixed_size: +(\d+)", notes, re.S):
                types = re.findall(r"E4M3|INT8|DF16b|f", m.group(1))
                types += types[:1] * (2 - len(types))   # (S_ or T_ for one that was there)
                found[(*types, *(int(m.group(i)) for i in (2, 3, 4)))] = int(m.group(5))
    return found


@pytest.mark.skipif(not os.path.exists(LIB) or not os.path.exists(READELF), reason="library not built, or no llvm-readelf")
def test_scratch_of_attention_on_caches(tmp_path):
    found = scratch(tmp_path)
    assert len(found) == 46, sorted(found)   # 18 of one block that take both walks, 18 of two, 10 of four
    assert all(v <= SPILLS.get(k, 0) for k, v in found.items()), {k: v for k, v in found.items() if v}
