"""Caches that pass 32 bits of bytes, and the longest ones."""
import math

import pytest
import torch

import paper_2605_08123_amd as ska

from . import cache_ref as ref
from .layer_ref import check, pairs
from .test_gpu_cache import ALL, BF16, F32, ints, rnd, say

pytestmark = pytest.mark.gpu
MOST = 1 << 24


@pytest.fixture(autouse=True)
def memory():
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("store", ["e4m3", "int8"])
def test_the_end_of_a_long_cache(store):
    """Two items of two heads of 2^24 tokens of 128 bytes: written and read near the ends, by queries whose band begins there."""
    say("long cache", store)
    g = torch.Generator().manual_seed(1)
    B, Hk, d, L, n = 2, 2, 128, MOST, 300
    cache = ska.KVCache(*(x.zero_() if x.dtype == F32 else x.view(torch.uint8).zero_().view(x.dtype) for x in ska.ska_cache_empty(B, Hk, L, d, store)))
    k, v = (rnd(g, B, Hk, n, d, dtype=BF16) for _ in range(2))
    at = ints(L - n, L - n - 40)
    ska.ska_cache_write(cache, k.cuda(), v.cuda(), start=at.cuda())
    small = ska.KVCache(*(x[:, :, L - 512:].contiguous() for x in cache))
    plain = ska.ska_cache_write(ska.KVCache(*(x.clone().zero_() if x.dtype == F32 else x.view(torch.uint8).clone().zero_().view(x.dtype) for x in small)), k.cuda(), v.cuda(),
                                start=(at - (L - 512)).cuda())
    for a, b in zip(small, plain):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    for a, b in zip(ska.ska_cache_read(cache, 350, start=at.cuda()), ska.ska_cache_read(small, 350, start=(at - (L - 512)).cuda())):
        assert torch.equal(a, b) and a.any()
    for Lq in (1, 20):
        q = rnd(g, B, 4, Lq, d, dtype=BF16)
        start = ints(L - Lq, L - Lq - 40)
        O, LSE = ska.ska_cache_attn_fwd(q.cuda(), cache, 200, True, start_q=start.cuda(), len_k=(start + Lq).int().cuda())
        kv = [ref.values(c.cpu().float(), s.cpu()) for c, s in ((small.K, small.K_scale), (small.V, small.V_scale))]
        want = ref.attn(q, *kv, pairs(B, Lq, 512, 200, True, start=start - (L - 512)), 1.0)
        check("O", O, want["O"])
        check("LSE", LSE, want["LSE"])


def test_the_end_of_a_long_prefix():
    """bf16: two heads of 2^24 tokens of 256 bytes, 4 GiB each."""
    say("long prefix")
    g = torch.Generator().manual_seed(2)
    B, Hq, Hk, d, n, Lk, W = 3, 4, 2, 128, 300, 20, 250
    pk, pv = (torch.zeros((Hk, MOST, d), dtype=BF16, device="cuda") for _ in range(2))
    tk, tv = (rnd(g, Hk, n, d, dtype=BF16) for _ in range(2))
    pk[:, MOST - n:], pv[:, MOST - n:] = tk.cuda(), tv.cuda()
    q, k, v = rnd(g, B, Hq, 2, d, dtype=BF16), rnd(g, B, Hk, Lk, d, dtype=BF16), rnd(g, B, Hk, Lk, d, dtype=BF16)
    start = ints(18, 0, 7)
    O, LSE = ska.ska_prefix_attn_fwd(q.cuda(), (pk, pv), (k.cuda(), v.cuda()), W, start_q=start.cuda())
    want = ref.prefix_attn(q, tk.double(), tv.double(), k.double(), v.double(), W, True, 1.0, start=start, codes=False)
    check("O", O, want["O"])
    check("LSE", LSE, want["LSE"])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_weights_over_the_longest_cache(dtype):
    """2^24 keys of the same weight: LSE is the logarithm of their number, O the mean of values that are 1 in the first half and 3 behind it.
    Weights are powers of two in every partial sum's own units; sums of n terms in parts and wavefronts: (n / 2^13 + 64) half-steps (a
    wavefront's share of 2048 at least, 32 tokens at a time, and the joins)."""
    say("longest", dtype)
    d, Hk = 64, 1
    cache = ska.KVCache(*(x.zero_() if x.dtype == F32 else x.view(torch.uint8).zero_().view(x.dtype) for x in ska.ska_cache_empty(1, Hk, MOST, d, "int8")))
    cache.V.fill_(1)
    cache.K_scale.fill_(1.0)
    cache.V_scale.fill_(1.0)
    cache.V_scale[:, :, MOST // 2:] = 3.0
    O, LSE = ska.ska_cache_attn_fwd(torch.ones((1, 2, 1, d), device="cuda", dtype=dtype), cache, MOST, False)
    tol = (MOST / 2 ** 13 + 64) * 2.0 ** -24
    assert (O.double() - 2).abs().max().item() <= 2 * (tol + (2.0 ** -8 if dtype == BF16 else 0))
    assert (LSE.double() - math.log(MOST)).abs().max().item() <= tol + 4 * 2.0 ** -24 * 17


def test_writing_the_most_tokens():
    """2^24 tokens of one row by strides of 0, heads next to each other in a token and apart."""
    say("most tokens")
    d = 128
    row = torch.randn(1, 2, 1, d, generator=torch.Generator().manual_seed(3)).to(BF16).cuda()
    one = ska.ska_cache_write(ska.ska_cache_empty(1, 2, 1, d), row, row)
    apart = torch.empty((1, 2, 2, d), dtype=BF16, device="cuda")[:, :, :1].copy_(row)
    for x in (row, apart):
        cache = ska.ska_cache_empty(1, 2, MOST, d)
        ska.ska_cache_write(cache, x.expand(1, 2, MOST, d), x.expand(1, 2, MOST, d))
        for a, b in zip(cache, one):
            a, b = a.view(torch.uint8) if a.dtype != F32 else a, b.view(torch.uint8) if b.dtype != F32 else b
            for i in range(0, MOST, 1 << 20):
                assert (a[:, :, i:i + (1 << 20)] == b).all(), i
        del cache
