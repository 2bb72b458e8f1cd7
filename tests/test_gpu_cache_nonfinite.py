"""Attention on caches where memory that does not count holds anything, and where what counts is not finite."""
import math

import pytest
import torch

import paper_2605_08123_amd as ska

from .layer_ref import pairs
from .cache_ref import prefix_pairs
from .test_gpu_cache import ALL, BF16, F32, cache_of, case, cuda, ints, rnd, say

pytestmark = pytest.mark.gpu
KINDS = [("same", F32), ("same", BF16), ("e4m3", F32), ("e4m3", BF16), ("int8", F32), ("int8", BF16)]


def spoilt(x, keep, what):
    """x with `what` in the rows that `keep` (of x's first dimensions without the heads) does not have."""
    y = x.clone()
    on = (keep[:, None] if x.dim() >= 3 else keep[None]).expand(x.shape[:keep.dim() + 1])
    if x.dtype in (torch.int8, torch.float8_e4m3fn):
        y.view(torch.uint8)[~on] = what
    else:
        y[~on] = what
    return y


def garbage(kept, keep, n):
    """The n-th way to spoil keys and values (and scales) that do not count."""
    out = []
    for i, x in enumerate(kept):
        if x.dtype in (torch.int8, torch.float8_e4m3fn):
            out.append(spoilt(x, keep, (0x7f, 0xff, 0x80)[(n + i) % 3]))      # e4m3: NaN, -NaN, -0; int8: 127, -1, -128
        else:
            out.append(spoilt(x, keep, (math.nan, math.inf, -math.inf)[(n + i) % 3]))
    return out


SHAPES = [(2, 4, 2, 1, 37, 64, ALL, True), (2, 8, 1, 1, 9000, 128, ALL, True), (3, 6, 2, 5, 333, 32, 40, True), (1, 4, 4, 33, 290, 64, 9, False),
          (2, 4, 1, 70, 700, 128, 100, True), (1, 4, 1, 130, 500, 64, 60, False)]


@pytest.mark.parametrize("store,dtype", KINDS[2:])
@pytest.mark.parametrize("B,Hq,Hk,Lq,Lk,d,W,causal", SHAPES)
def test_garbage_in_a_cache(B, Hq, Hk, Lq, Lk, d, W, causal, store, dtype):
    """Beyond the lengths, inactive, out of reach, and queries that do not take part: the same bits whatever is there."""
    say("garbage", B, Hq, Hk, Lq, Lk, d, W, causal, store, dtype)
    g = torch.Generator().manual_seed(Lk)
    q, k, v = case(g, B, Hq, Hk, Lq, Lk, d, dtype)
    cache = cache_of(k, v, store, "cpu")
    start = ints(*[max(Lk - Lq - 7 - 3 * b, 0) for b in range(B)])
    len_k, len_q = ints(*[Lk - 3 - b for b in range(B)]), ints(*[max(Lq - b, 1) for b in range(B)])
    mask_k, mask_q = (torch.rand(B, Lk, generator=g) > 0.3).to(torch.uint8), (torch.rand(B, Lq, generator=g) > 0.2).to(torch.uint8)
    mask_q[:, 0] = 1
    reached = pairs(B, Lq, Lk, W, causal, start=start, len_q=len_q, len_k=len_k).any(1)
    row = (torch.arange(Lq)[None] < len_q[:, None]) & mask_q.bool()
    kw = dict(start_q=start.cuda(), len_q=len_q.cuda(), len_k=len_k.cuda(), mask_q=mask_q.cuda(), mask_k=mask_k.cuda())
    want = ska.ska_cache_attn_fwd(spoilt(q, row, 0.0).cuda(), ska.KVCache(*(spoilt(x, reached & mask_k.bool(), 0).cuda() for x in cache)), W, causal, **kw)
    assert torch.isfinite(want[0]).all()
    for n in range(3):
        got = ska.ska_cache_attn_fwd(spoilt(q, row, (math.nan, math.inf, -math.inf)[n]).cuda(),
                                     ska.KVCache(*(x.cuda() for x in garbage(cache, reached & mask_k.bool(), n))), W, causal, **kw)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


PSHAPES = [(3, 4, 2, 1, 400, 37, 64, ALL, True), (5, 8, 1, 1, 9000, 70, 128, ALL, True), (3, 6, 2, 5, 333, 100, 32, 90, True), (2, 4, 4, 33, 290, 80, 64, 130, False)]


@pytest.mark.parametrize("store,dtype", KINDS)
@pytest.mark.parametrize("B,Hq,Hk,Lq,Lp,Lk,d,W,causal", PSHAPES)
def test_garbage_beside_a_prefix(B, Hq, Hk, Lq, Lp, Lk, d, W, causal, store, dtype):
    say("garbage prefix", B, Hq, Hk, Lq, Lp, Lk, d, W, causal, store, dtype)
    g = torch.Generator().manual_seed(Lk + Lp)
    q, k, v = case(g, B, Hq, Hk, Lq, Lk, d, dtype)
    _, pk, pv = case(g, 1, Hq, Hk, Lq, Lp, d, dtype)
    own, pre = ((k, v), (pk, pv)) if store == "same" else (cache_of(k, v, store, "cpu"), cache_of(pk, pv, store, "cpu"))
    P = Lp - 13
    start = ints(*[max(Lk - Lq - 7 - 3 * b, 0) for b in range(B)])
    len_k, len_q = ints(*[Lk - 3 - b for b in range(B)]), ints(*[max(Lq - b, 1) for b in range(B)])
    mask_k, mask_q, mask_p = ((torch.rand(*s, generator=g) > 0.3).to(torch.uint8) for s in ((B, Lk), (B, Lq), (Lp,)))
    mask_q[:, 0] = 1
    reached = pairs(B, Lq, Lk, W, causal, start=start, len_q=len_q, len_k=len_k).any(1) & mask_k.bool()
    preached = (prefix_pairs(B, Lq, P, Lp, W, start, len_q, None, None).any(1).any(0) & mask_p.bool())[None]
    row = (torch.arange(Lq)[None] < len_q[:, None]) & mask_q.bool()
    kw = dict(len_p=ints(P).cuda(), start_q=start.cuda(), len_q=len_q.cuda(), len_k=len_k.cuda(), mask_q=mask_q.cuda(), mask_k=mask_k.cuda(), mask_p=mask_p.cuda())
    want = ska.ska_prefix_attn_fwd(spoilt(q, row, 0.0).cuda(), [spoilt(x, preached, 0)[0].cuda() for x in pre], [spoilt(x, reached, 0).cuda() for x in own], W, causal, **kw)
    assert torch.isfinite(want[0]).all()
    for n in range(3):
        got = ska.ska_prefix_attn_fwd(spoilt(q, row, (math.nan, math.inf, -math.inf)[n]).cuda(), [x[0].cuda() for x in garbage(pre, preached, n)],
                                      [x.cuda() for x in garbage(own, reached, n)], W, causal, **kw)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("store,dtype", KINDS)
@pytest.mark.parametrize("Lk,d", [(9, 32), (700, 128), (9000, 64)])   # one tile, a few, parts of a walk
def test_what_is_not_finite_goes_on(Lk, d, store, dtype):
    """Scores: minus infinity weighs nothing, alone it is NaN, NaN and infinity are NaN, in the rows that meet them alone.  A NaN query row is
    its own, a NaN value is in the rows that reach it."""
    say("not finite", Lk, d, store, dtype)
    g = torch.Generator().manual_seed(Lk + d)
    B, Hq, Hk, Lq = 1, 2, 1, 6
    q, k, v = case(g, B, Hq, Hk, Lq, Lk, d, dtype)
    q = q.abs() + 0.5
    at, start, W = Lk - 3, Lk - 6, 2          # queries at Lk - 6 ... Lk - 1 reach themselves and two before: those at Lk - 3 ... Lk - 1 reach `at`
    q, k = q.to(dtype), k.abs().to(dtype)

    def run(qq, kk, vv, W=W, masked=None, poison=None):
        kw = dict(start_q=ints(start).cuda(), mask_k=None if masked is None else masked.cuda())
        if store == "same":
            pk, pv = (x[0, :, :8].cuda() for x in (k, v))
            m = torch.zeros(8, dtype=torch.uint8).cuda()
            kk = kk.clone()
            if poison is not None:
                kk[:, :, at] = poison[0] if poison[1] == "k" else kk[:, :, at]
                vv = vv.clone()
                if poison[1] == "v":
                    vv[:, :, at] = poison[0]
            return [x.cpu() for x in ska.ska_prefix_attn_fwd(qq.cuda(), (pk, pv), (kk.cuda(), vv.cuda()), W, True, mask_p=m, **kw)]
        c = ska.KVCache(*(x.clone() for x in cache_of(kk, vv, store, "cpu")))
        if poison is not None:
            (c.K_scale if poison[1] == "k" else c.V_scale)[:, :, at] = poison[0]
            if poison[1] == "k":
                c.K.view(torch.uint8)[:, :, at] = 0x38 if store == "e4m3" else 1      # 1: the product with a positive query has the scale's sign
        return [x.cpu() for x in ska.ska_cache_attn_fwd(qq.cuda(), ska.KVCache(*(x.cuda() for x in c)), W, True, **kw)]

    O, LSE = run(q, k, v)
    before, meet = slice(0, 3), slice(3, 6)
    for bad in (math.nan, math.inf):
        o, lse = run(q, k, v, poison=(bad, "k"))
        assert torch.equal(o[:, :, before], O[:, :, before]) and torch.equal(lse[:, :, before], LSE[:, :, before])
        assert torch.isnan(o[:, :, meet]).all() and torch.isnan(lse[:, :, meet]).all()
    o, lse = run(q, k, v, poison=(-math.inf, "k"))
    m = torch.ones(1, Lk, dtype=torch.uint8)
    m[0, at] = 0
    o1, lse1 = run(q, k, v, masked=m)
    assert torch.equal(o, o1) and torch.equal(lse, lse1)
    # alone: row 3 with a band of itself
    o, lse = run(q, k, v, W=0, poison=(-math.inf, "k"))
    o1, lse1 = run(q, k, v, W=0)
    for i in range(6):
        if i == 3:
            assert torch.isnan(o[:, :, i]).all() and torch.isnan(lse[:, :, i]).all()
        else:
            assert torch.equal(o[:, :, i], o1[:, :, i]) and torch.equal(lse[:, :, i], lse1[:, :, i])
    # a NaN row of queries
    qn = q.clone()
    qn[:, 1, 4, 5] = math.nan
    o, lse = run(qn, k, v)
    assert torch.isnan(o[:, 1, 4]).all() and torch.isnan(lse[:, 1, 4]).all()
    keep = torch.ones(1, 2, 6, dtype=torch.bool)
    keep[:, 1, 4] = False
    assert torch.equal(o[keep], O[keep]) and torch.equal(lse[keep], LSE[keep])
    # a NaN value
    o, lse = run(q, k, v, poison=(math.nan, "v"))
    assert torch.isnan(o[:, :, meet]).all() and torch.equal(lse, LSE)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("store", ["e4m3", "int8"])
def test_a_row_that_is_not_finite_is_written_and_met(store, dtype):
    """Through the cache: a token with an infinity stands for NaN, and the queries that reach it are NaN."""
    g = torch.Generator().manual_seed(5)
    k, v = rnd(g, 1, 2, 50, 64, dtype=dtype), rnd(g, 1, 2, 50, 64, dtype=dtype)
    k[0, 1, 20, 7] = math.inf
    cache = ska.ska_cache_write(ska.ska_cache_empty(1, 2, 64, 64, store), k.cuda(), v.cuda())
    O, LSE = ska.ska_cache_attn_fwd(rnd(g, 1, 2, 50, 64, dtype=dtype).cuda(), cache, 10, True, len_k=cuda(ints(50)))
    hit = torch.zeros(2, 50, dtype=torch.bool)
    hit[1, 20:31] = True
    assert torch.equal(torch.isnan(LSE[0]).cpu(), hit) and torch.equal(torch.isnan(O[0]).all(-1).cpu(), hit)
    assert torch.isfinite(O[0].cpu()[~hit]).all()
