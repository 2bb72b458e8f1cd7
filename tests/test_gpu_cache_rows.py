"""Attention on caches in workgroups of 64 query rows, which larger problems take (test_cache_plan_host.py holds that these do): masks, bands, rows left
empty, memory that holds anything, scales far apart, d = 32 and 64, parts of a walk."""
import pytest
import torch

import paper_2605_08123_amd as ska

from . import cache_ref as ref
from .layer_ref import check, pairs
from .test_gpu_cache import ALL, BF16, F32, cache_of, case, clamped, cuda, ints, kept, limits, rnd, say
from .test_gpu_cache_nonfinite import KINDS
from .test_gpu_cache_nonfinite import test_garbage_beside_a_prefix as garbage_beside_a_prefix
from .test_gpu_cache_nonfinite import test_garbage_in_a_cache as garbage_in_a_cache
from .test_gpu_cache_precision import scales

pytestmark = pytest.mark.gpu
CODES = KINDS[2:]
# B, Hq, Hk, Lq, Lk, d, W, causal
ROWS = [(40, 3, 3, 66, 70, 32, 5, True), (6, 5, 5, 300, 333, 32, 31, True), (12, 6, 2, 150, 210, 32, ALL, False), (5, 4, 1, 700, 260, 64, ALL, True),
        (33, 4, 2, 65, 25, 64, 5, True)]
# ... in parts, and the kinds that take 64 rows there
PARTS = [((3, 3, 1, 299, 2680, 64, ALL, True), ("e4m3", F32)), ((33, 6, 2, 12, 2479, 64, ALL, False), ("int8", F32)), ((33, 8, 2, 10, 4033, 32, ALL, True), ("e4m3", BF16))]
# B, Hq, Hk, Lq, Lp, Lk, d, W, causal: all kinds but fp32 caches, whose workgroups have 32 rows
PREFIX = [(33, 6, 3, 19, 300, 45, 64, ALL, True), (20, 4, 2, 74, 23, 19, 32, 5, True), (6, 6, 2, 150, 100, 100, 32, ALL, True), (33, 6, 3, 19, 45, 18, 64, 100, False)]
PREFIX_PARTS = [((9, 4, 1, 33, 12000, 20, 64, ALL, True), ("same", BF16)), ((9, 4, 1, 33, 12000, 20, 64, 11000, True), ("e4m3", F32)),
                ((16, 4, 2, 17, 20000, 40, 64, ALL, True), ("int8", BF16)), ((16, 4, 2, 17, 20000, 40, 32, ALL, True), ("e4m3", BF16)),
                ((16, 4, 2, 17, 20000, 40, 32, ALL, True), ("same", BF16))]


def cache_call(shape, store, dtype, which):
    """Limits `which` (of limits()) of a problem against the reference, twice the same bits."""
    B, Hq, Hk, Lq, Lk, d, W, causal = shape
    say("64 rows", shape, store, dtype)
    g = torch.Generator().manual_seed(Lq * 31 + Lk)
    q, k, v = case(g, B, Hq, Hk, Lq, Lk, d, dtype)
    cache = cache_of(k, v, store)
    kv = [ref.values(c, s) for c, s in (kept(k, store), kept(v, store))]
    for n, kw in enumerate(limits(g, B, Lq, Lk)):
        if n not in which:
            continue
        call = lambda: ska.ska_cache_attn_fwd(q.cuda(), cache, W, causal, **{n: x.cuda() for n, x in kw.items()})   # noqa: E731
        O, LSE = call()
        want = ref.attn(q, *kv, pairs(B, Lq, Lk, W, causal, **clamped(kw, Lq, Lk)), 1.0)
        check("O", O, want["O"])
        check("LSE", LSE, want["LSE"])
        again = call()
        assert torch.equal(O, again[0]) and torch.equal(LSE, again[1])


@pytest.mark.parametrize("store,dtype", CODES)
@pytest.mark.parametrize("shape", ROWS)
def test_cache(shape, store, dtype):
    cache_call(shape, store, dtype, range(5))


@pytest.mark.parametrize("shape,kind", PARTS)
def test_cache_in_parts(shape, kind):
    cache_call(shape, *kind, (1, 3))


def prefix_call(shape, store, dtype, which):
    B, Hq, Hk, Lq, Lp, Lk, d, W, causal = shape
    say("64 rows behind a prefix", shape, store, dtype)
    g = torch.Generator().manual_seed(Lp * 31 + Lk)
    q, k, v = case(g, B, Hq, Hk, Lq, Lk, d, dtype)
    _, pk, pv = case(g, 1, Hq, Hk, Lq, Lp, d, dtype)
    if store == "same":
        own, prefix, kv, pkv = (k.cuda(), v.cuda()), (pk[0].cuda(), pv[0].cuda()), (k.double(), v.double()), (pk[0].double(), pv[0].double())
    else:
        own, prefix = cache_of(k, v, store), ska.KVCache(*(x[0] for x in cache_of(pk, pv, store)))
        kv, pkv = ([ref.values(*kept(x, store)) for x in two] for two in ((k, v), (pk[0], pv[0])))
    for n, kw in enumerate(limits(g, B, Lq, Lk)):
        if n not in which:
            continue
        P = Lp - Lp // 7 if n in (1, 2) else None
        mask_p = (torch.rand(Lp, generator=g) > 0.3).to(torch.uint8) if n == 3 else torch.zeros(Lp, dtype=torch.uint8) if n == 4 else None
        call = lambda: ska.ska_prefix_attn_fwd(q.cuda(), prefix, own, W, causal, len_p=None if P is None else ints(P).cuda(), mask_p=cuda(mask_p),   # noqa: E731
                                               **{n: x.cuda() for n, x in kw.items()})
        O, LSE = call()
        want = ref.prefix_attn(q, *pkv, *kv, W, causal, 1.0, P=P, mask_p=mask_p, codes=store != "same", **clamped(kw, Lq, Lk))
        check("O", O, want["O"])
        check("LSE", LSE, want["LSE"])
        again = call()
        assert torch.equal(O, again[0]) and torch.equal(LSE, again[1])


@pytest.mark.parametrize("store,dtype", KINDS[1:])
@pytest.mark.parametrize("shape", PREFIX)
def test_prefix(shape, store, dtype):
    prefix_call(shape, store, dtype, range(5))


@pytest.mark.parametrize("shape,kind", PREFIX_PARTS)
def test_prefix_in_parts(shape, kind):
    prefix_call(shape, *kind, (3,))


@pytest.mark.parametrize("store,dtype", CODES)
@pytest.mark.parametrize("shape", ROWS)
def test_garbage_in_a_cache_of_many_rows(shape, store, dtype):
    garbage_in_a_cache(*shape, store, dtype)


@pytest.mark.parametrize("store,dtype", KINDS[1:])
@pytest.mark.parametrize("shape", PREFIX)
def test_garbage_beside_a_prefix_of_many_rows(shape, store, dtype):
    garbage_beside_a_prefix(*shape, store, dtype)


@pytest.mark.parametrize("kind", ["near", "far", "growing", "shrinking", "zeros", "one"])
@pytest.mark.parametrize("store,dtype", CODES)
@pytest.mark.parametrize("B,Hq,Hk,Lq,Lk,d,W,causal", [ROWS[1], ROWS[3]])
def test_values_far_apart_under_many_rows(B, Hq, Hk, Lq, Lk, d, W, causal, store, dtype, kind):
    say("values far apart, 64 rows", B, Hq, Hk, Lq, Lk, d, W, store, dtype, kind)
    g = torch.Generator().manual_seed(Lq)
    q, k, v = rnd(g, B, Hq, Lq, d, dtype=dtype), rnd(g, B, Hk, Lk, d, dtype=dtype), torch.randn(B, Hk, Lk, d, generator=g)
    v = (v * scales(g, kind, Lk)[None, None, :, None]).to(dtype)
    O, LSE = ska.ska_cache_attn_fwd(q.cuda(), cache_of(k, v, store), W, causal)
    want = ref.attn(q, *(ref.values(*kept(x, store)) for x in (k, v)), pairs(B, Lq, Lk, W, causal), 1.0)
    check("O", O, want["O"])
    check("LSE", LSE, want["LSE"])
