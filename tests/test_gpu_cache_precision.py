"""Attention on caches: accuracy in the 2-norm, and values whose scales lie far apart."""
import math

import pytest
import torch

import paper_2605_08123_amd as ska

from . import cache_ref as ref
from .layer_ref import check, half, pairs
from .test_gpu_cache import ALL, BF16, F32, cache_of, ints, kept, rnd, say

pytestmark = pytest.mark.gpu
ROUND = 2.0 ** -8 / math.sqrt(3)   # bf16: uniform in half a step, which is 2^-8 of the value at most
SHAPES = [(1, 8, 2, 1, 9000, 64, ALL), (4, 4, 4, 5, 700, 32, ALL), (1, 8, 8, 300, 300, 128, 200), (2, 8, 1, 40, 900, 64, ALL), (1, 4, 2, 90, 400, 128, 50)]


@pytest.mark.parametrize("store", ["e4m3", "int8", "same"])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,Hq,Hk,Lq,Lk,d,W", SHAPES)
def test_two_norms(B, Hq, Hk, Lq, Lk, d, W, dtype, store):
    """bf16: the result's rounding, and of codes three of 2^-11 (P, the scale, their product) that sums over keys average as they do the
    values; of bf16 values 2^-16.  fp32: scores of size 1 from d products (three times as many for a query in three parts, whose second part
    is 2^-8 and adds nothing), sums over the keys, and a dozen for scaling, exponential and LSE."""
    g = torch.Generator().manual_seed(Lq + d)
    q, k, v = (torch.randn(B, h, n, d, generator=g).to(dtype) for h, n in ((Hq, Lq), (Hk, Lk), (Hk, Lk)))
    start = ints(*[Lk - Lq] * B)
    ok = pairs(B, Lq, Lk, W, True, start=start)
    if store == "same":
        none = torch.zeros((Hk, 1, d), dtype=dtype).cuda()
        O, LSE = ska.ska_prefix_attn_fwd(q.cuda(), (none, none), (k.cuda(), v.cuda()), W, True, len_p=ints(0).cuda(), start_q=start.cuda())
        want = ref.attn(q, k.double(), v.double(), ok, 1.0, codes=False)
    else:
        O, LSE = ska.ska_cache_attn_fwd(q.cuda(), cache_of(k, v, store), W, True, start_q=start.cuda())
        want = ref.attn(q, *(ref.values(*kept(x, store)) for x in (k, v)), ok, 1.0)
    off = ((O.double().cpu() - want["O"][0]).norm() / want["O"][0].norm()).item()
    say("2-norm", B, Hq, Hk, Lq, Lk, d, W, dtype, store, f"{off:.2e}")
    n = ok.sum().item() / (B * Lq)
    limit = ROUND * math.sqrt(1 + (0 if store == "same" else 3 / 64)) if dtype == BF16 else (2 * math.sqrt(d) + math.sqrt(n) + 12) * 2.0 ** -24
    assert off <= limit, (off, limit)


def scales(g, kind, n):
    """Sizes of n values' rows, a few powers of two to the whole range apart."""
    i = torch.arange(n)
    if kind == "near":
        return torch.exp2(-torch.randint(0, 8, (n,), generator=g).float())
    if kind == "far":                                    # within a tile
        return torch.exp2(-torch.randint(0, 40, (n,), generator=g).float())
    if kind == "growing":                                # every few tiles
        return torch.exp2(torch.div(i, 70, rounding_mode="floor").float() * 7 - 50)
    if kind == "shrinking":
        return torch.exp2(40 - torch.div(i, 70, rounding_mode="floor").float() * 7)
    if kind == "zeros":                                  # rows of zeros between others
        return (torch.rand(n, generator=g) > 0.3).float()
    return torch.where(i == n // 2, 2.0 ** 30, 1.0)      # "one"


@pytest.mark.parametrize("kind", ["near", "far", "growing", "shrinking", "zeros", "one"])
@pytest.mark.parametrize("store,dtype", [("e4m3", BF16), ("int8", BF16), ("e4m3", F32), ("int8", F32)])
@pytest.mark.parametrize("B,Hq,Hk,Lq,Lk,d,W", [(1, 4, 2, 1, 1000, 64, ALL), (1, 4, 2, 9, 1000, 128, ALL), (1, 8, 1, 100, 1000, 32, 300)])
def test_values_far_apart(B, Hq, Hk, Lq, Lk, d, W, store, dtype, kind):
    say("values far apart", B, Hq, Hk, Lq, Lk, d, W, store, dtype, kind)
    g = torch.Generator().manual_seed(Lq)
    q, k, v = rnd(g, B, Hq, Lq, d, dtype=dtype), rnd(g, B, Hk, Lk, d, dtype=dtype), torch.randn(B, Hk, Lk, d, generator=g)
    v = (v * scales(g, kind, Lk)[None, None, :, None]).to(dtype)
    start = ints(Lk - Lq)
    O, LSE = ska.ska_cache_attn_fwd(q.cuda(), cache_of(k, v, store), W, True, start_q=start.cuda())
    want = ref.attn(q, *(ref.values(*kept(x, store)) for x in (k, v)), pairs(B, Lq, Lk, W, True, start=start), 1.0)
    check("O", O, want["O"])
    check("LSE", LSE, want["LSE"])


@pytest.mark.parametrize("store", ["e4m3", "int8"])
@pytest.mark.parametrize("apart", [2.0 ** 5, 2.0 ** 9, 2.0 ** 12, 2.0 ** 20, 2.0 ** 60])
def test_rows_that_do_not_reach_a_large_value(apart, store):
    """Queries whose own values are `apart` times smaller than one that only their neighbours in the tile reach, and whose keys but one have
    the same small weights, so that roundings of products do not average.  bf16, codes: a value's product is off by 2^-20 of the value at
    most (half of fp16's smallest number, with P in 2^-4 and the value at least 2^-9 of the unit; below that 2^-16 relative), P by 2^-29."""
    say("unreached", apart, store)
    g = torch.Generator().manual_seed(3)
    Hq, Lq, Lk, d = 1, 16, 200, 64
    q = torch.ones(1, Hq, Lq, d)
    k = torch.full((1, 1, Lk, d), -0.75)
    k[:, :, 100] = 0.0                           # the largest score, 8 0.75 above the others: weights of exp(-6), and one of 1
    v = torch.rand(1, 1, Lk, d, generator=g) + 0.5
    v[:, :, Lk - 1] *= apart                     # the last query's own token, which causality keeps from the others
    q, k, v = (x.to(BF16) for x in (q, k, v))
    start = ints(Lk - Lq)
    O, LSE = ska.ska_cache_attn_fwd(q.cuda(), cache_of(k, v, store), ALL, True, start_q=start.cuda())
    kv = [ref.values(*kept(x, store)) for x in (k, v)]
    ok = pairs(1, Lq, Lk, ALL, True, start=start)
    ok[:, -1] = False                            # (the bound by the largest value that a row reaches: without the one that does)
    want, bound = ref.attn(q, *kv, ok, 1.0)["O"]
    n = ok.sum(2).double()[:, None, :, None]
    vmax = kv[1][:, :, :Lk - 1].abs().amax()
    p = torch.softmax((q.double() @ kv[0].transpose(-1, -2) / 8).masked_fill(~ok[:, None], -math.inf)[:, :, :-1], -1)
    top = p.amax(-1, keepdim=True)               # (a weight of 1 in P is `top` after the division by the row's sum)
    floor = (2.0 ** -20 + 2.0 ** -29) * n[:, :, :-1] * vmax * top
    check("O", O[:, :, :-1], (want[:, :, :-1], bound[:, :, :-1] + floor))
    assert (floor < 4 * half(BF16) * want[:, :, :-1].abs().amax()).all()   # (the bound says something)


@pytest.mark.parametrize("store", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("W", [0, 3])
def test_values_at_the_ends_of_fp32(W, dtype, store):
    """Each item with values of a size of its own, from the largest (alone: sums of several pass fp32) to the smallest that a scale has."""
    say("ends of fp32", W, dtype, store)
    g = torch.Generator().manual_seed(9)
    sizes = [2.9e38 if W == 0 else 5e37, 1e30, 1.0, 1e-20, 1e-30, 1e-36]
    B, Hq, Hk, L, d = len(sizes), 2, 1, 40, 64
    q, k = rnd(g, B, Hq, L, d, dtype=dtype), rnd(g, B, Hk, L, d, dtype=dtype)
    v = (torch.rand(B, Hk, L, d, generator=g) * 2 - 1).to(dtype) * torch.tensor(sizes).view(-1, 1, 1, 1).to(dtype)
    v = v.to(dtype)
    cache = ska.ska_cache_write(ska.ska_cache_empty(B, Hk, L, d, store), k.cuda(), v.cuda())
    O, LSE = ska.ska_cache_attn_fwd(q.cuda(), cache, W, True)
    kv = [ref.values(*kept(x, store)) for x in (k, v)]
    for b in range(B):   # (the bound takes the largest value of all: one item at a time)
        want = ref.attn(q[b:b + 1], *(x[b:b + 1] for x in kv), pairs(1, L, L, W, True), 1.0)
        # below 2^-126 a number has a rounding of 2^-150 at least, and flushing it is 2^-126 in units of the value's scale
        check("O", O[b:b + 1], (want["O"][0], want["O"][1] + 2.0 ** -126 * (1 + 2.0 ** -8)))
        check("LSE", LSE[b:b + 1], want["LSE"])
