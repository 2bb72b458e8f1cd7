"""The operators on caches (include/sinkhorn_attn_cache.h) on the GPU against their 64-bit definitions: what is written and read back
exactly, attention entry by entry within the bounds of tests/cache_ref.py, at the sizes, masks, strides and streams where they can go
wrong."""
import math

import pytest
import torch

import paper_2605_08123_amd as ska

from . import cache_ref as ref
from .layer_ref import check, pairs

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
ALL = 1 << 20


def rnd(g, *shape, dtype=F32, scale=1.0):
    """Activations: tokens of different sizes."""
    x = torch.randn(*shape, generator=g) * torch.exp(0.5 * torch.randn(*shape[:-1], 1, generator=g))
    return (x * scale).to(dtype)


def say(*what):
    print("\n[case]", *what, flush=True)


def cuda(x):
    return None if x is None else x.cuda()


def kept(x, store):
    """(codes, scales) on the CPU in the types of a cache."""
    c, s = ref.quantise(x, store)
    return c.float().to(ska.cache.CACHE_STORES[store]), s.float()


def cache_of(k, v, store, device="cuda"):
    (kc, ks), (vc, vs) = kept(k, store), kept(v, store)
    return ska.KVCache(*(x.to(device) for x in (kc, vc, ks, vs)))


def ints(*x):
    return torch.tensor(x, dtype=torch.int32)


# ------------------------------------------------------------------ writing and reading
@pytest.mark.parametrize("store", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,Hk,d,L,Lc", [(1, 1, 32, 1, 1), (8, 2, 64, 1, 37), (3, 2, 128, 5, 9), (2, 4, 64, 130, 150), (1, 3, 32, 515, 515), (2, 1, 128, 1000, 2001)])
def test_write_and_read(B, Hk, d, L, Lc, dtype, store):
    """Every code and scale is the definition's, other places stay as they were, and what comes back is rounded once."""
    say("cache", B, Hk, d, L, Lc, dtype, store)
    g = torch.Generator().manual_seed(L * 17 + d)
    k, v = rnd(g, B, Hk, L, d, dtype=dtype), rnd(g, B, Hk, L, d, dtype=dtype, scale=100.0)
    old = [rnd(g, B, Hk, Lc, d, dtype=dtype) for _ in range(2)]
    # all of it from 0; ragged; places before the cache and behind it; nothing at all
    for start, new in ((None, None), (torch.randint(0, Lc, (B,), generator=g, dtype=torch.int32), torch.randint(0, L + 1, (B,), generator=g, dtype=torch.int32)),
                       (ints(*[-2] * B), None), (ints(*[Lc - 1] * B), None), (ints(*[2 ** 31 - 1] * B), None), (ints(*[-2 ** 31] * B), None), (None, ints(*[0] * B)),
                       (None, ints(*[-5] * B)), (None, ints(*[2 ** 31 - 1] * B))):
        cache, want = cache_of(*old, store), cache_of(*old, store, "cpu")
        got = ska.ska_cache_write(cache, k.cuda(), v.cuda(), start=cuda(start), len_new=cuda(new))
        assert got is cache
        fresh = [kept(x, store) for x in (k, v)]
        for b in range(B):
            i, n = 0 if start is None else int(start[b]), L if new is None else min(max(int(new[b]), 0), L)
            l0, l1 = max(0, -i), max(0, min(n, Lc - i))
            if l0 < l1:
                for w in range(2):
                    want[w][b, :, i + l0:i + l1] = fresh[w][0][b, :, l0:l1]
                    want[2 + w][b, :, i + l0:i + l1] = fresh[w][1][b, :, l0:l1]
        for a, b in zip(cache, want):
            assert torch.equal(a.cpu().float(), b.float())
        for out in (F32, BF16):
            vals = [(c.float() * s[..., None]).to(out) for c, s in ((want.K, want.K_scale), (want.V, want.V_scale))]   # fp32 product, rounded once
            for a, b in zip(ska.ska_cache_read(cache, dtype=out), vals):
                assert torch.equal(a.cpu(), b)
    # windows that begin before the cache and end behind it, lengths
    first, end = torch.randint(-3, Lc, (B,), generator=g, dtype=torch.int32), torch.randint(-1, Lc + 3, (B,), generator=g, dtype=torch.int32)
    n = L // 2 + 3
    K, V = ska.ska_cache_read(cache, n, start=first.cuda(), len_k=end.cuda(), dtype=F32)
    for got, val in ((K, want.K.float() * want.K_scale[..., None]), (V, want.V.float() * want.V_scale[..., None])):
        for b in range(B):
            expect = torch.zeros(Hk, n, d)
            for l in range(n):
                at = int(first[b]) + l
                if 0 <= at < min(max(int(end[b]), 0), Lc):
                    expect[:, l] = val[b, :, at]
            assert torch.equal(got[b].cpu(), expect)


@pytest.mark.parametrize("store", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_write_at_borders(dtype, store):
    """Ties, zeros, the smallest and the largest numbers, rows that are not finite."""
    d = 32
    rows = []
    for e in (0, 5, -20, 100, -100):
        top = 2.0 ** e
        if store == "int8":
            t = torch.arange(32).float() + 0.5
            rows += [torch.cat([torch.tensor([127.0]), t[1:]]) * top, -torch.cat([torch.tensor([127.0]), t[:31] + 95]) * top]
        else:
            n = ref.e4m3_numbers().float()
            mid = (n[1:] + n[:-1]) / 2
            rows += [torch.cat([torch.tensor([448.0]), s * mid[i:i + 31]]) * top for i in range(0, 126, 31) for s in (1, -1) if i + 31 <= 126]
    zero = torch.zeros(d)
    tiny = torch.full((d,), 1e-45)
    rows += [zero, -zero, tiny, tiny * 3e4, torch.linspace(-1, 1, d) * 2.0 ** -120, torch.linspace(-1, 1, d) * 3.3e38,
             torch.linspace(-1, 1, d) * torch.finfo(F32).max if dtype == F32 else zero, torch.linspace(-1, 1, d) * 1e-38]
    # scales that round, quotients near borders: random bits in fp32
    g = torch.Generator().manual_seed(0)
    rows += list(torch.randn(4000, d, generator=g) * torch.exp(3 * torch.randn(4000, 1, generator=g)))
    for bad in (math.nan, math.inf, -math.inf):
        r = torch.randn(d, generator=g)
        r[7] = bad
        rows.append(r)
    x = torch.stack(rows).to(dtype)[None, None]
    c, s = ref.quantise(x, store)
    cache = ska.ska_cache_write(ska.ska_cache_empty(1, 1, x.shape[2], d, store), x.cuda(), x.cuda())
    for codes, scale in ((cache.K, cache.K_scale), (cache.V, cache.V_scale)):
        assert torch.equal(codes.cpu().double(), c)
        assert torch.equal(scale.cpu().double().nan_to_num(nan=-1.0), s.nan_to_num(nan=-1.0))
    K, _ = ska.ska_cache_read(cache, dtype=F32)
    assert torch.isnan(K[0, 0, -3:]).all() and torch.isfinite(K[0, 0, :-3]).all()


def test_write_ties_of_int8_in_fp32():
    """Products (n + 1/2) s rounded to fp32 lie a little beside a border or on it: the code goes by the numbers and not by a rounded quotient."""
    g = torch.Generator().manual_seed(2)
    d, n = 128, 3000
    a = torch.rand(n, 1, generator=g) + 0.5
    s = a / 127
    x = (torch.randint(0, 126, (n, d), generator=g) + 0.5) * s      # rounded to fp32
    x = torch.where(torch.rand(n, d, generator=g) < 0.3, torch.nextafter(x, torch.zeros(())), x)
    x[:, :1] = a
    c, scale = ref.quantise(x, "int8")
    cache = ska.ska_cache_write(ska.ska_cache_empty(1, 1, n, d, "int8"), x[None, None].cuda(), x[None, None].cuda())
    assert torch.equal(cache.K_scale[0, 0].cpu().double(), scale) and torch.equal(cache.K[0, 0].cpu().double(), c)


@pytest.mark.parametrize("store", ["e4m3", "int8"])
def test_views(store):
    """New tokens in a projection's layout and broadcast over heads, caches that are views of items, heads and places, outputs in views."""
    say("cache views", store)
    g = torch.Generator().manual_seed(4)
    B, Hk, L, Lc, d = 2, 3, 11, 29, 64
    wide = rnd(g, B, L, 2 * Hk, d, dtype=BF16).cuda().transpose(1, 2)
    k, v = wide[:, :Hk], wide[:, Hk:]
    big = ska.ska_cache_empty(2 * B, 2 * Hk, Lc + 8, d, store)
    for x in big:
        x.view(torch.uint8 if x.dtype != F32 else F32).fill_(3)
    part = ska.KVCache(*(x[1::2, 2:2 + Hk, 5:5 + Lc] for x in big))
    ska.ska_cache_write(part, k, v, start=ints(4, 7).cuda())
    plain = ska.ska_cache_empty(B, Hk, Lc, d, store)
    for x in plain:
        x.view(torch.uint8 if x.dtype != F32 else F32).fill_(3)
    ska.ska_cache_write(plain, k.contiguous(), v.contiguous(), start=ints(4, 7).cuda())
    for a, b in zip(part, plain):
        assert torch.equal(a.float(), b.float())
    for x in big:   # nothing around the view
        y = x.view(torch.uint8).clone() if x.dtype != F32 else x.clone()
        y[1::2, 2:2 + Hk, 5:5 + Lc] = 3
        assert (y == 3).all()
    out = torch.full((B, L, 2 * Hk, d), 9.0, device="cuda", dtype=BF16)
    K, V = (out.transpose(1, 2)[:, i:i + Hk] for i in (0, Hk))
    ska.ska_cache_read(part, start=ints(4, 7).cuda(), K=K, V=V)
    for a, b in zip((K, V), ska.ska_cache_read(plain, L, start=ints(4, 7).cuda())):
        assert torch.equal(a, b)
    # one key head for all items and heads
    one = k[:1, :1].expand(B, Hk, L, d)
    a, b = (ska.ska_cache_write(ska.ska_cache_empty(B, Hk, L, d, store), x, x) for x in (one, one.contiguous()))
    assert all(torch.equal(x.float(), y.float()) for x, y in zip(a, b))
    # attention on the view, and without any copy of it
    q = rnd(g, B, 2 * Hk, 3, d, dtype=BF16).cuda()
    O, LSE = ska.ska_cache_attn_fwd(q, part, ALL, True, start_q=ints(12, 15).cuda(), len_k=ints(15, 18).cuda())
    O1, LSE1 = ska.ska_cache_attn_fwd(q, plain, ALL, True, start_q=ints(12, 15).cuda(), len_k=ints(15, 18).cuda())
    assert torch.equal(O, O1) and torch.equal(LSE, LSE1)


def test_nothing_to_write():
    c = ska.ska_cache_empty(2, 2, 8, 64)
    x = torch.zeros((2, 2, 0, 64), device="cuda")
    ska.ska_cache_write(c, x, x)
    K, V = ska.ska_cache_read(c, 0)
    assert K.shape == V.shape == (2, 2, 0, 64)


# ------------------------------------------------------------------ attention on a cache
# B, Hq, Hk, Lq, Lk, d, W, causal, eps: from one token on one key to several blocks of rows and parts of a walk
ATTN = [(1, 1, 1, 1, 1, 32, 0, True, 1.0), (2, 4, 2, 1, 37, 64, ALL, True, 1.0), (3, 8, 1, 1, 500, 128, ALL, True, 0.5), (1, 8, 2, 1, 9000, 64, ALL, False, 1.0),
        (2, 6, 2, 5, 333, 32, 64, True, 1.0), (2, 16, 2, 3, 1000, 64, 100, False, 1.0), (1, 3, 3, 17, 64, 128, 9, True, 1.0), (1, 4, 4, 33, 33, 32, ALL, True, 1.0),
        (1, 8, 2, 40, 700, 64, ALL, True, 1.0), (1, 4, 1, 130, 1500, 64, 300, False, 0.5), (2, 2, 1, 300, 300, 128, 31, True, 1.0), (1, 2, 2, 600, 600, 32, 5, False, 1.0),
        (1, 32, 1, 1, 100, 64, 7, False, 1.0), (1, 5, 1, 7, 5000, 128, ALL, True, 1.0)]


def case(g, B, Hq, Hk, Lq, Lk, d, dtype):
    return rnd(g, B, Hq, Lq, d, dtype=dtype), rnd(g, B, Hk, Lk, d, dtype=dtype), rnd(g, B, Hk, Lk, d, dtype=dtype, scale=3.0)


def limits(g, B, Lq, Lk):
    """A few ways to say who takes part; arguments of the call."""
    lens = torch.randint(0, Lk + 1, (B,), generator=g, dtype=torch.int32)
    yield dict(start_q=ints(*[max(Lk - Lq, 0)] * B))
    yield dict(start_q=torch.clamp(lens - Lq, min=0).int(), len_k=lens)
    yield dict(start_q=torch.randint(-3, Lk + 5, (B,), generator=g, dtype=torch.int32), len_q=torch.randint(0, Lq + 1, (B,), generator=g, dtype=torch.int32),
               len_k=torch.randint(-1, Lk + 3, (B,), generator=g, dtype=torch.int32))
    on = lambda n: (torch.rand(B, (n + 7) // 8, generator=g) > 0.4).repeat_interleave(8, 1)[:, :n].to(torch.uint8).contiguous()   # noqa: E731
    yield dict(start_q=ints(*[max(Lk - Lq, 0)] * B), mask_q=on(Lq), mask_k=on(Lk))
    yield dict(mask_k=torch.zeros(B, Lk, dtype=torch.uint8))


def clamped(kw, Lq, Lk):
    """The same as the header's limits make of it, for the reference."""
    kw = dict(kw)
    if "start_q" in kw:
        kw["start"] = kw.pop("start_q").clamp(0, 1 << 24)
    return kw


@pytest.mark.parametrize("store", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,Hq,Hk,Lq,Lk,d,W,causal,eps", ATTN)
def test_attention(B, Hq, Hk, Lq, Lk, d, W, causal, eps, dtype, store):
    say("cache attention", B, Hq, Hk, Lq, Lk, d, W, causal, eps, dtype, store)
    g = torch.Generator().manual_seed(Lq * 31 + Lk)
    q, k, v = case(g, B, Hq, Hk, Lq, Lk, d, dtype)
    cache = cache_of(k, v, store)
    kv = [ref.values(c, s) for c, s in (kept(k, store), kept(v, store))]
    for kw in limits(g, B, Lq, Lk):
        O, LSE = ska.ska_cache_attn_fwd(q.cuda(), cache, W, causal, eps, **{n: x.cuda() for n, x in kw.items()})
        want = ref.attn(q, *kv, pairs(B, Lq, Lk, W, causal, **clamped(kw, Lq, Lk)), eps)
        check("O", O, want["O"])
        check("LSE", LSE, want["LSE"])
        again = ska.ska_cache_attn_fwd(q.cuda(), cache, W, causal, eps, **{n: x.cuda() for n, x in kw.items()})
        assert torch.equal(O, again[0]) and torch.equal(LSE, again[1])


# ------------------------------------------------------------------ attention behind a shared prefix
# B, Hq, Hk, Lq, Lp, Lk, d, W, causal, eps
PREFIX = [(1, 1, 1, 1, 1, 1, 32, 0, True, 1.0), (2, 4, 2, 1, 40, 7, 64, ALL, True, 1.0), (3, 6, 2, 3, 1003, 77, 32, 300, True, 0.5), (20, 8, 2, 1, 3000, 40, 64, ALL, True, 1.0),
          (5, 4, 4, 7, 33, 500, 128, ALL, False, 1.0), (40, 4, 1, 2, 700, 30, 64, 100, False, 1.0), (2, 16, 4, 9, 2500, 20, 128, ALL, True, 1.0),
          (70, 2, 1, 1, 129, 64, 32, 90, True, 1.0), (1, 8, 2, 1, 5000, 33, 64, ALL, True, 1.0), (3, 2, 1, 100, 256, 130, 64, ALL, True, 1.0)]


@pytest.mark.parametrize("store,dtype", [("same", F32), ("same", BF16), ("e4m3", F32), ("e4m3", BF16), ("int8", F32), ("int8", BF16)])
@pytest.mark.parametrize("B,Hq,Hk,Lq,Lp,Lk,d,W,causal,eps", PREFIX)
def test_prefix(B, Hq, Hk, Lq, Lp, Lk, d, W, causal, eps, store, dtype):
    say("prefix attention", B, Hq, Hk, Lq, Lp, Lk, d, W, causal, eps, store, dtype)
    g = torch.Generator().manual_seed(Lp * 31 + Lk)
    q, k, v = case(g, B, Hq, Hk, Lq, Lk, d, dtype)
    _, pk, pv = case(g, 1, Hq, Hk, Lq, Lp, d, dtype)
    if store == "same":
        own, prefix, kv, pkv = (k.cuda(), v.cuda()), (pk[0].cuda(), pv[0].cuda()), (k.double(), v.double()), (pk[0].double(), pv[0].double())
    else:
        own, prefix = cache_of(k, v, store), ska.KVCache(*(x[0] for x in cache_of(pk, pv, store)))
        kv, pkv = ([ref.values(*kept(x, store)) for x in two] for two in ((k, v), (pk[0], pv[0])))
    for n, kw in enumerate(limits(g, B, Lq, Lk)):
        P = mask_p = None
        if n == 2:
            P = int(torch.randint(0, Lp + 1, (1,), generator=g))
        if n >= 3:
            mask_p = (torch.rand(Lp, generator=g) > 0.3).to(torch.uint8) if n == 3 else torch.zeros(Lp, dtype=torch.uint8)
        call = lambda: ska.ska_prefix_attn_fwd(q.cuda(), prefix, own, W, causal, eps, len_p=None if P is None else ints(P).cuda(), mask_p=cuda(mask_p),   # noqa: E731
                                               **{n: x.cuda() for n, x in kw.items()})
        O, LSE = call()
        want = ref.prefix_attn(q, *pkv, *kv, W, causal, eps, P=P, mask_p=mask_p, codes=store != "same", **clamped(kw, Lq, Lk))
        check("O", O, want["O"])
        check("LSE", LSE, want["LSE"])
        again = call()
        assert torch.equal(O, again[0]) and torch.equal(LSE, again[1])


def test_prefix_lengths_at_their_ends():
    """Lengths of the prefix below 0 and beyond Lp, items without a token of their own."""
    g = torch.Generator().manual_seed(8)
    q, k, v = case(g, 3, 4, 2, 1, 9, 64, BF16)
    _, pk, pv = case(g, 1, 4, 2, 1, 50, 64, BF16)
    call = lambda **kw: ska.ska_prefix_attn_fwd(q.cuda(), (pk[0].cuda(), pv[0].cuda()), (k.cuda(), v.cuda()), ALL, **kw)   # noqa: E731
    n = ints(0, 4, 9)
    for given, P in ((-7, 0), (0, 0), (50, 50), (2 ** 31 - 1, 50)):
        O, LSE = call(len_p=ints(given).cuda(), len_k=n.cuda(), start_q=(n - 1).cuda())
        want = ref.prefix_attn(q, pk[0].double(), pv[0].double(), k.double(), v.double(), ALL, True, 1.0, P=P, len_k=n, start=(n - 1).clamp(min=0), codes=False)
        check("O", O, want["O"])
        check("LSE", LSE, want["LSE"])
        if P == 0:
            assert not O[0].any() and (LSE[0] == -math.inf).all()


@pytest.mark.parametrize("store,dtype", [("same", F32), ("same", BF16), ("e4m3", F32), ("e4m3", BF16), ("int8", BF16)])
@pytest.mark.parametrize("B,Hq,Hk,Lq,Lp,Lk,d,W", [(120, 4, 2, 1, 300, 900, 32, ALL), (250, 1, 1, 3, 700, 1500, 32, 1800), (64, 8, 4, 2, 900, 60, 64, ALL)])
def test_prefix_of_many_items(B, Hq, Hk, Lq, Lp, Lk, d, W, store, dtype):
    """As many workgroups as there are CUs, or nearly: these walk over the prefix and their own keys of ragged lengths."""
    say("prefix of many", B, Hq, Hk, Lq, Lp, Lk, d, W, store, dtype)
    g = torch.Generator().manual_seed(Lp + Lk)
    q, k, v = case(g, B, Hq, Hk, Lq, Lk, d, dtype)
    _, pk, pv = case(g, 1, Hq, Hk, Lq, Lp, d, dtype)
    if store == "same":
        own, prefix, kv, pkv = (k.cuda(), v.cuda()), (pk[0].cuda(), pv[0].cuda()), (k.double(), v.double()), (pk[0].double(), pv[0].double())
    else:
        own, prefix = cache_of(k, v, store), ska.KVCache(*(x[0] for x in cache_of(pk, pv, store)))
        kv, pkv = ([ref.values(*kept(x, store)) for x in two] for two in ((k, v), (pk[0], pv[0])))
    lens = torch.randint(0, Lk + 1, (B,), generator=g, dtype=torch.int32)
    start, P = torch.clamp(lens - Lq, min=0).int(), Lp - 5
    mask_p = (torch.rand(Lp, generator=g) > 0.1).to(torch.uint8)
    call = lambda: ska.ska_prefix_attn_fwd(q.cuda(), prefix, own, W, start_q=start.cuda(), len_k=lens.cuda(), len_p=ints(P).cuda(), mask_p=mask_p.cuda())   # noqa: E731
    O, LSE = call()
    want = ref.prefix_attn(q, *pkv, *kv, W, True, 1.0, P=P, mask_p=mask_p, codes=store != "same", start=start, len_k=lens)
    check("O", O, want["O"])
    check("LSE", LSE, want["LSE"])
    again = call()
    assert torch.equal(O, again[0]) and torch.equal(LSE, again[1])


@pytest.mark.parametrize("B,Hq,Hk,Lq,Lk,d", [(66, 4, 2, 1, 4000, 32), (3, 4, 2, 700, 2100, 64), (150, 2, 2, 2, 1300, 128)])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("store", ["e4m3", "int8"])
def test_parts_of_many_problems(B, Hq, Hk, Lq, Lk, d, store, dtype):
    """More problems than fill whole rounds of workgroups: walks in parts, ragged lengths, some of which leave parts without a key."""
    say("parts", B, Hq, Hk, Lq, Lk, d, store, dtype)
    g = torch.Generator().manual_seed(Lk)
    q, k, v = case(g, B, Hq, Hk, Lq, Lk, d, dtype)
    lens = torch.randint(0, Lk + 1, (B,), generator=g, dtype=torch.int32)
    start = torch.clamp(lens - Lq, min=0).int()
    call = lambda: ska.ska_cache_attn_fwd(q.cuda(), cache_of(k, v, store), ALL, True, start_q=start.cuda(), len_k=lens.cuda())   # noqa: E731
    O, LSE = call()
    want = ref.attn(q, *(ref.values(*kept(x, store)) for x in (k, v)), pairs(B, Lq, Lk, ALL, True, start=start, len_k=lens), 1.0)
    check("O", O, want["O"])
    check("LSE", LSE, want["LSE"])
    again = call()
    assert torch.equal(O, again[0]) and torch.equal(LSE, again[1])
