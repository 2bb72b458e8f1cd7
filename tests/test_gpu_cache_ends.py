"""Numbers at the ends of their ranges on caches: scores that climb while a walk goes on, beside large values;
small values; codes of rows whose scale is near the smallest."""
import math

import pytest
import torch

import paper_2605_08123_amd as ska

from . import cache_ref as ref
from .layer_ref import check, pairs
from .test_gpu_cache import ALL, BF16, F32, cache_of, ints, kept, say

pytestmark = pytest.mark.gpu
CLIMB = [(1, 300, 64), (1, 2600, 32), (40, 300, 128), (70, 530, 64), (8000, 300, 64)]   # (the last: workgroups of 64 rows)


@pytest.mark.parametrize("store,dtype", [("same", F32), ("same", BF16), ("e4m3", F32), ("e4m3", BF16), ("int8", F32), ("int8", BF16)])
@pytest.mark.parametrize("Lq,Lk,d", CLIMB)
@pytest.mark.parametrize("climb", [11.5, 15.5])
def test_scores_that_climb_beside_large_values(Lq, Lk, d, climb, store, dtype):
    """Scores of 0 in each wavefront's first tile, and `climb` powers of two above them behind it; values as large as the header says: 2^127
    divided by the tokens and 64 more."""
    say("climb", Lq, Lk, d, climb, store, dtype)
    g = torch.Generator().manual_seed(Lk)
    q = torch.zeros(1, 2, Lq, d)
    q[..., 0] = 8.0
    k = torch.zeros(1, 1, Lk, d)
    k[:, :, 256:, 0] = torch.where(torch.arange(Lk - 256) % 7 == 3, climb * math.log(2) * math.sqrt(d) / 8, 0.0)
    most = 2.0 ** 127 / (Lk + 64)
    v = (torch.rand(1, 1, Lk, d, generator=g) + 1) * (0.49 * most)
    q, k, v = (x.to(dtype) for x in (q, k, v))
    start = ints(Lk)   # (all keys for all queries)
    ok = pairs(1, Lq, Lk, ALL, True, start=start)
    if store == "same":
        none = torch.zeros((1, 1, d), dtype=dtype).cuda()
        O, LSE = ska.ska_prefix_attn_fwd(q.cuda(), (none, none), (k.cuda(), v.cuda()), ALL, True, len_p=ints(0).cuda(), start_q=start.cuda())
        want = ref.attn(q, k.double(), v.double(), ok, 1.0, codes=False)
    else:
        O, LSE = ska.ska_cache_attn_fwd(q.cuda(), cache_of(k, v, store), ALL, True, start_q=start.cuda())
        want = ref.attn(q, *(ref.values(*kept(x, store)) for x in (k, v)), ok, 1.0)
    check("O", O, want["O"])
    check("LSE", LSE, want["LSE"])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("size", [1e-20, 1e-30, 1e-36])
@pytest.mark.parametrize("Lq", [1, 40])
def test_small_values_of_plain_caches(Lq, size, dtype):
    """Values whose products with a weight are below the smallest normal number while they are summed: off by 2^-126 at most."""
    say("small values", Lq, size, dtype)
    g = torch.Generator().manual_seed(5)
    q, k = (torch.randn(2, h, n, 64, generator=g).to(dtype) for h, n in ((4, Lq), (2, 400)))
    v = ((torch.rand(2, 2, 400, 64, generator=g) + 1) * size).to(dtype)
    start = ints(400, 300)
    O, LSE = ska.ska_prefix_attn_fwd(q.cuda(), (k[0].cuda(), v[0].cuda()), (k.cuda(), v.cuda()), ALL, start_q=start.cuda())
    want = ref.prefix_attn(q, k[0].double(), v[0].double(), k.double(), v.double(), ALL, True, 1.0, start=start, codes=False)
    check("O", O, (want["O"][0], want["O"][1] + 2.0 ** -126), floor=0.0)
    check("LSE", LSE, want["LSE"])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("e", [-126, -125, -100, 0, 100])
def test_int8_borders_of_small_scales(e, dtype):
    """Numbers beside (n + 1/2) s, s in [2^e, 2^(e + 1)): half of a scale below 2^-125 need not be an fp32 number."""
    say("int8 borders", e, dtype)
    g = torch.Generator().manual_seed(e + 200)
    n, d = 4000, 128
    a = (127 * (1 + torch.rand(n, 1, generator=g, dtype=torch.float64)) * 2.0 ** e).to(dtype)
    s = ref.quantise(a.float(), "int8")[1][:, None]
    x = ((torch.randint(0, 127, (n, d), generator=g).double() + 0.5) * s).to(dtype)
    step = torch.randint(-1, 2, (n, d), generator=g)
    x = torch.where(step < 0, torch.nextafter(x, torch.zeros_like(x)), torch.where(step > 0, torch.nextafter(x, a.expand(n, d)), x))
    x = x * (torch.randint(0, 2, (n, d), generator=g) * 2 - 1).to(dtype)
    x[:, :1] = a
    c, scale = ref.quantise(x, "int8")
    assert (scale < 2.0 ** (e + 1)).float().mean() > 0.9 and (scale >= 2.0 ** e).float().mean() > 0.9
    cache = ska.ska_cache_write(ska.ska_cache_empty(1, 1, n, d, "int8"), x[None, None].cuda(), x[None, None].cuda())
    for codes, got in ((cache.K, cache.K_scale), (cache.V, cache.V_scale)):
        assert torch.equal(got[0, 0].cpu().double(), scale) and torch.equal(codes[0, 0].cpu().double(), c)
