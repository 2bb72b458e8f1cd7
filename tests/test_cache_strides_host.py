"""Strides of a shared prefix: those between heads and tokens count, those between items say nothing (no GPU)."""
import pytest

from paper_2605_08123_amd import binding, cache

from .test_cache_host import BF16, E4M3, P, by


@pytest.mark.parametrize("store", [BF16, E4M3])
@pytest.mark.parametrize("b", [-64, -1, 0, 7, 1 << 40])
def test_strides_between_items_of_a_prefix_do_not_count(b, store):
    """Taken as far as the workspace that is not there."""
    lib = cache._lib()

    def call(h, l, hs):
        s, ss = by((b, h, l)), by((b, hs)) if store == E4M3 else None
        scale = P if store == E4M3 else None
        return lib.ska_prefix_attn_fwd(P, None, P, s, scale, ss, P, s, scale, ss, P, None, scale, None, P, None, scale, None, P, None, P, None, None, None,
                                       None, None, None, None, 1, 4, 2, 40, 5000, 64, 64, 8, 0, 1.0, BF16, store, None, 0, None)
    assert call(1 << 20, 64, 1 << 20) == binding.SKA_EWORKSPACE
    assert call(-64, 64, 1 << 20) == call(1 << 20, -64, 1 << 20) == binding.SKA_EINVAL
    assert call(1 << 20, 72 if store == E4M3 else 68, 1 << 20) == binding.SKA_EUNSUPPORTED
