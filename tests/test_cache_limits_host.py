"""The largest launches of the attention on caches: refused where the threads would pass 32 bits, before anything is launched (no GPU)."""
import pytest

import paper_2605_08123_amd as ska
from paper_2605_08123_amd import binding, cache

from .test_cache_host import BF16, E4M3, F32, INT8, _attn


# Lq (Hq / Hk) query rows of B Hk problems, 64 to a workgroup of 512 threads (32 for d = 128): 2^32 threads are 2^23 workgroups
@pytest.mark.parametrize("dt,d,rows", [(BF16, 64, 64), (BF16, 32, 64), (BF16, 128, 32), (F32, 32, 64), (F32, 128, 32)])
@pytest.mark.parametrize("store", [E4M3, INT8])
def test_threads_within_32_bits(dt, d, rows, store):
    lib = cache._lib()
    most = (1 << 23) // 16 * rows   # rows of each of 16 problems at which 2^23 workgroups are reached
    for prefix in (False, True):
        for Hq, Lq in ((2, most), (4, most // 2), (32, (most + 15) // 16)):
            if Lq <= 1 << 24:
                assert _attn(lib, prefix, B=8, Hq=Hq, Hk=2, Lq=Lq, d=d, dt=dt, store=store) == binding.SKA_EUNSUPPORTED
    # the size before is taken (no workspace: it would be launched with one)
    assert ska.ska_prefix_attn_workspace_bytes(1, 32, 2, rows * 256, 64, 64, d, 8, dtype=dt, store=store) > 0
    assert _attn(lib, True, B=1, Hq=32, Hk=2, Lq=rows * 256, Lk=64, d=d, dt=dt, store=store, ws=None) == binding.SKA_EWORKSPACE
