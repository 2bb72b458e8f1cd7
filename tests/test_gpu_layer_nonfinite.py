"""Softmax attention with NaN and infinities in live tokens: what the definition makes NaN is NaN, in O, LSE and the gradients, whole walks
and walks in parts, and what takes no part in it keeps its bits."""
import math

import pytest
import torch

import paper_2605_08123_amd as ska

from . import layer_ref as ref

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def make(B, Hq, Hk, Lq, Lk, d, dtype, seed=0):
    g = torch.Generator().manual_seed(seed + Lq * 31 + Lk)
    return [torch.randn(B, h, n, d, generator=g).to(dtype).cuda() for h, n in ((Hq, Lq), (Hk, Lk), (Hk, Lk), (Hq, Lq))]


def both(q, k, v, do, W, **kw):
    O, LSE = ska.ska_softmax_attn_fwd(q, k, v, W, **kw)
    out = [O, LSE, *ska.ska_softmax_attn_bwd(q, k, v, O, do, LSE, W, **kw)]
    torch.cuda.synchronize()
    return out


# B, Hq, Hk, Lq, Lk, d, W, causal: one wavefront per workgroup and four, whole walks and parts (the last three)
SHAPES = [(2, 2, 1, 200, 200, 64, 20, False), (1, 2, 2, 333, 333, 32, 40, True), (1, 16, 16, 2100, 2100, 64, 70, False),
          (1, 16, 16, 2100, 2100, 128, 33, True), (2, 4, 2, 1, 4000, 64, 1 << 20, True), (1, 8, 2, 17, 3000, 128, 1 << 20, True),
          (1, 2, 2, 700, 700, 32, 700, False)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("what", ["query", "key"])
@pytest.mark.parametrize("B,Hq,Hk,Lq,Lk,d,W,causal", SHAPES)
def test_a_nan_goes_on(B, Hq, Hk, Lq, Lk, d, W, causal, what, dtype):
    """One feature of one live query, or of one live key, is NaN."""
    print("\n[case]", B, Hq, Hk, Lq, Lk, d, W, causal, what, dtype, flush=True)
    start = torch.tensor([Lk - Lq] * B, dtype=torch.int32)
    kw = dict(causal=causal, start_q=start.cuda())
    ok = ref.pairs(B, Lq, Lk, W, causal, start=start)[0]
    q, k, v, do = make(B, Hq, Hk, Lq, Lk, d, dtype)
    clean = both(q, k, v, do, W, **kw)
    assert all(torch.isfinite(x).all() for x in clean)
    for at in (0, (Lq if what == "query" else Lk) // 2, (Lq if what == "query" else Lk) - 1):
        x, y = q.clone(), k.clone()
        (x if what == "query" else y)[0, 0, at, 3] = math.nan
        O, LSE, dQ, dK, dV = both(x, y, v, do, W, **kw)
        heads = slice(0, 1) if what == "query" else slice(0, Hq // Hk)   # query heads that read it
        hit = torch.zeros(Lq, dtype=torch.bool)
        if what == "query":
            hit[at] = True
        else:
            hit = ok[:, at].clone()
        assert hit.any()
        reached = ok[hit].any(0)                  # keys that take part with a poisoned row
        for name, t, rows, h in (("O", O, hit, heads), ("LSE", LSE, hit, heads), ("dQ", dQ, hit, heads), ("dK", dK, reached, slice(0, 1)),
                                 ("dV", dV, reached, slice(0, 1))):
            assert torch.isnan(t[0, h][:, rows.cuda()]).all(), (name, at)
        # scores of pairs are selected by bits: rows apart keep their values, as do the other heads and items
        for name, t, c in (("O", O, clean[0]), ("LSE", LSE, clean[1])):
            assert torch.equal(t[0, heads][:, ~hit.cuda()], c[0, heads][:, ~hit.cuda()]), (name, at)
        for t, c, n in zip((O, LSE, dQ, dK, dV), clean, (heads.stop, heads.stop, heads.stop, 1, 1)):
            assert torch.equal(t[0, n:], c[0, n:]) and torch.equal(t[1:], c[1:])
        # gradients: a product with a probability of 0 is NaN within a tile, not beyond
        i, j = hit.nonzero()[:, 0], reached.nonzero()[:, 0]
        far_q, far_k = torch.ones(Lq, dtype=torch.bool), torch.ones(Lk, dtype=torch.bool)
        far_q[max(0, int(i[0]) - 128):int(i[-1]) + 129] = False
        far_k[max(0, int(j[0]) - 128):int(j[-1]) + 129] = False
        assert torch.equal(dQ[0, heads][:, far_q.cuda()], clean[2][0, heads][:, far_q.cuda()])
        for t, c in ((dK, clean[3]), (dV, clean[4])):
            assert torch.equal(t[0, :1][:, far_k.cuda()], c[0, :1][:, far_k.cuda()])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,Hq,Hk,Lq,Lk,d,W,causal", SHAPES)
def test_infinite_scores(B, Hq, Hk, Lq, Lk, d, W, causal, dtype):
    """A key with an infinite feature: a score of +inf makes its row NaN (inf - inf), one of -inf is a key of no weight, and a row
    with such scores alone is NaN (0 / 0)."""
    print("\n[case]", B, Hq, Hk, Lq, Lk, d, W, causal, dtype, flush=True)
    start = torch.tensor([Lk - Lq] * B, dtype=torch.int32)
    ok = ref.pairs(B, Lq, Lk, W, causal, start=start)
    q, k, v, do = make(B, Hq, Hk, Lq, Lk, d, dtype, seed=5)
    G = Hq // Hk
    at = Lk // 2 if Lq > 17 else Lk - Lq
    sign = torch.sign(q[0, :G, :, 3].float()).cpu()
    assert (sign != 0).all()
    k[0, 0, at, 3] = math.inf
    O, LSE = ska.ska_softmax_attn_fwd(q, k, v, W, causal=causal, start_q=start.cuda())
    torch.cuda.synchronize()
    plus, minus = ok[0, :, at] & (sign > 0), ok[0, :, at] & (sign < 0)
    for h in range(G):
        assert torch.isnan(O[0, h].cpu()[plus[h]]).all() and torch.isnan(LSE[0, h].cpu()[plus[h]]).all()
    without = ok.clone()
    without[0, :, at] = False
    k0 = k.cpu()
    k0[0, 0, at, 3] = 0
    want = ref.attn(q.cpu(), k0, v.cpu(), without, 1.0)
    for h in range(G):
        rows = minus[h] & without[0].any(1)
        for t, name in ((O, "O"), (LSE, "LSE")):
            ref.check(name, t[0, h].cpu()[rows], tuple(x[0, h][rows] for x in want[name]))
    # every key of the first item's group alike: rows of -inf alone
    k[0, 0, :, :] = 0
    k[0, 0, :, 3] = math.inf
    q = q.abs()
    q[0, :, :, 3] = -1.0
    O, LSE = ska.ska_softmax_attn_fwd(q, k, v, W, causal=causal, start_q=start.cuda())
    assert torch.isnan(O[0, :G]).all() and torch.isnan(LSE[0, :G]).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("Lq,Lk", [(1, 3000), (150, 150)])
def test_minus_infinity_alone_among_masked_keys(Lq, Lk, dtype):
    """Rows whose only active key scores -inf are NaN, rows without an active key zeros and -inf: masks tell them apart, not the sum."""
    print("\n[case]", Lq, Lk, dtype, flush=True)
    q, k, v, _ = make(2, 2, 1, Lq, Lk, 64, dtype)
    q[..., 3] = -1.0
    at = Lk // 3
    k[:, :, at] = 0
    k[:, :, at, 3] = math.inf
    mask = torch.zeros(2, Lk, dtype=torch.uint8)
    mask[0, at] = 1   # item 1: none
    O, LSE = ska.ska_softmax_attn_fwd(q, k, v, 1 << 20, mask_k=mask.cuda())
    assert torch.isnan(O[0]).all() and torch.isnan(LSE[0]).all()
    assert not O[1].any() and (LSE[1] == -math.inf).all()


def test_the_last_shapes_are_in_parts():
    """(what the shapes above rely on)"""
    assert all(ska.ska_softmax_attn_workspace_bytes(False, B, Hq, Hk, Lq, Lk, d, W, c) > 0 for B, Hq, Hk, Lq, Lk, d, W, c in SHAPES[4:6])


# B, Hq, Hk, Lq, Lk, d, W, causal, starts: keys past the causal end, beside the band on either side, queries past all keys
UNREACHED = [(1, 2, 1, 1, 1024, 64, 1 << 20, True, [1000]), (2, 4, 2, 1, 1024, 128, 50, False, [1000, 300]), (2, 2, 2, 17, 900, 32, 40, True, [500, 0]),
             (1, 4, 4, 300, 1500, 64, 25, False, [610]), (1, 2, 2, 400, 130, 32, 33, False, [0]), (1, 16, 16, 1100, 4000, 64, 70, True, [1501]),
             (1, 8, 2, 40, 2600, 64, 1 << 20, True, [2000]), (2, 16, 16, 900, 1024, 128, 300, False, [0, 700])]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("fill", [math.nan, math.inf])
@pytest.mark.parametrize("B,Hq,Hk,Lq,Lk,d,W,causal,start", UNREACHED)
def test_what_nothing_reaches_may_hold_anything(B, Hq, Hk, Lq, Lk, d, W, causal, start, fill, dtype):
    """Active keys that lie within no query's band, and queries within no key's, without lengths or masks: an unfilled cache."""
    print("\n[case]", B, Hq, Hk, Lq, Lk, d, W, causal, start, fill, dtype, flush=True)
    q, k, v, do = (x.cpu() for x in make(B, Hq, Hk, Lq, Lk, d, dtype, seed=9))
    at = torch.tensor(start, dtype=torch.int32)
    ok = ref.pairs(B, Lq, Lk, W, causal, start=at)
    want = ref.attn(q, k, v, ok, 1.0, do)
    assert not ok.any(1).all() or not ok.any(2).all()
    for x, dead in ((q, ~ok.any(2)), (do, ~ok.any(2)), (k, ~ok.any(1)), (v, ~ok.any(1))):
        x[dead[:, None].expand(x.shape[:3])] = fill
    kw = dict(causal=causal, start_q=at.cuda())
    q, k, v, do = (x.cuda() for x in (q, k, v, do))
    O, LSE = ska.ska_softmax_attn_fwd(q, k, v, W, **kw)
    ref.check("O", O, want["O"])
    ref.check("LSE", LSE, want["LSE"])
    grads = ska.ska_softmax_attn_bwd(q, k, v, want["O"][0].to(dtype).cuda(), do, want["LSE"][0].float().cuda(), W, **kw)
    torch.cuda.synchronize()
    for name, x in zip(("dQ", "dK", "dV"), grads):
        ref.check(name, x, want[name])
    dead = ~ok.any(1)[:, None].expand(B, Hk, Lk).cuda()
    assert not grads[1][dead].any() and not grads[2][dead].any()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,Hq,Hk,Lq,Lk,d,W,causal", SHAPES)
def test_a_nan_in_a_value(B, Hq, Hk, Lq, Lk, d, W, causal, dtype):
    """It is in O of the queries that read it and in the dQ and dK of their pairs; LSE and dV do not depend on it."""
    print("\n[case]", B, Hq, Hk, Lq, Lk, d, W, causal, dtype, flush=True)
    start = torch.tensor([Lk - Lq] * B, dtype=torch.int32)
    kw = dict(causal=causal, start_q=start.cuda())
    ok = ref.pairs(B, Lq, Lk, W, causal, start=start)[0]
    q, k, v, do = make(B, Hq, Hk, Lq, Lk, d, dtype, seed=3)
    clean = both(q, k, v, do, W, **kw)
    at = Lk // 2 if Lq > 17 else Lk - Lq
    v[0, 0, at, 5] = math.nan
    O, LSE, dQ, dK, dV = both(q, k, v, do, W, **kw)
    hit = ok[:, at]
    reached = ok[hit].any(0)
    heads = slice(0, Hq // Hk)
    assert torch.isnan(O[0, heads][:, hit.cuda(), 5]).all() and torch.isnan(dQ[0, heads][:, hit.cuda()]).all()
    assert torch.isnan(dK[0, :1][:, reached.cuda()]).all()
    assert torch.equal(LSE, clean[1]) and torch.equal(dV, clean[4])
    assert torch.equal(O[0, heads][..., :5], clean[0][0, heads][..., :5])   # (another feature is another sum)
    for t, c, n in zip((O, dQ, dK), (clean[0], clean[2], clean[3]), (heads.stop, heads.stop, 1)):
        assert torch.equal(t[0, n:], c[0, n:]) and torch.equal(t[1:], c[1:])
