"""Softmax attention's accuracy in the 2-norm, and its gradients against differences of its own forward, within limits that a wrong result
does not meet."""
import math

import pytest
import torch

import paper_2605_08123_amd as ska

from . import layer_ref as ref

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def errors(B, Hq, Hk, Lq, Lk, d, W, causal, dtype, start=None):
    """{name: relative 2-norm of what differs from 64 bits}, and the mean number of keys of a query."""
    g = torch.Generator().manual_seed(Lq + d)
    q, k, v, do = (torch.randn(B, h, n, d, generator=g).to(dtype) for h, n in ((Hq, Lq), (Hk, Lk), (Hk, Lk), (Hq, Lq)))
    at = None if start is None else torch.tensor([start] * B, dtype=torch.int32)
    ok = ref.pairs(B, Lq, Lk, W, causal, start=at)
    want = ref.attn(q, k, v, ok, 1.0, do)
    kw = dict(causal=causal, start_q=None if at is None else at.cuda())
    q, k, v, do = (x.cuda() for x in (q, k, v, do))
    got = {"O": ska.ska_softmax_attn_fwd(q, k, v, W, **kw)[0]}
    o, lse = want["O"][0].to(dtype).cuda(), want["LSE"][0].float().cuda()
    got.update(zip(("dQ", "dK", "dV"), ska.ska_softmax_attn_bwd(q, k, v, o, do, lse, W, **kw)))
    torch.cuda.synchronize()
    off = {n: ((x.double().cpu() - want[n][0]).norm() / want[n][0].norm()).item() for n, x in got.items()}
    print("\n[case]", B, Hq, Hk, Lq, Lk, d, W, causal, dtype, {n: f"{x:.2e}" for n, x in off.items()}, flush=True)
    return off, ok.sum().item() / (B * Lq)


ROUND = 2.0 ** -8 / math.sqrt(3)   # bf16: uniform in half a step, which is 2^-8 of the value at most
FEW = [(1, 4, 4, 256, 256, 64, 256, False, None), (2, 4, 2, 200, 200, 32, 40, True, None), (1, 8, 8, 300, 300, 128, 300, True, None),
       (4, 8, 2, 1, 5000, 64, 1 << 20, True, 4999), (2, 4, 4, 17, 900, 128, 1 << 20, True, 883)]
MANY = [(1, 16, 16, 2100, 2100, 64, 70, False, None), (2, 16, 16, 1030, 1030, 32, 1030, True, None), (1, 16, 4, 2048, 2048, 128, 2048, True, None),
        (1, 16, 16, 2100, 2100, 128, 300, True, None)]


@pytest.mark.parametrize("B,Hq,Hk,Lq,Lk,d,W,causal,start", FEW)
def test_few_rows_round_their_results_alone(B, Hq, Hk, Lq, Lk, d, W, causal, start):
    """bf16, one wavefront per workgroup: P and dS go into their products in two parts, whose rest is 2^-16.  What is left is the rounding
    of the results; in the gradients also that of the O given, which reaches them by delta, a sum over d terms of an average over keys: a
    quarter of a rounding's square."""
    off, _ = errors(B, Hq, Hk, Lq, Lk, d, W, causal, BF16, start)
    assert off["O"] <= ROUND, off
    assert max(off.values()) <= ROUND * math.sqrt(1.25), off


@pytest.mark.parametrize("B,Hq,Hk,Lq,Lk,d,W,causal,start", MANY)
def test_many_rows_round_once_more(B, Hq, Hk, Lq, Lk, d, W, causal, start):
    """bf16, four wavefronts per workgroup: P and dS are rounded before their products, independently for each pair, which sums over keys
    average as they do the values themselves: one more rounding of the results' size."""
    off, _ = errors(B, Hq, Hk, Lq, Lk, d, W, causal, BF16, start)
    assert off["O"] <= ROUND * math.sqrt(2.0), off
    assert max(off.values()) <= ROUND * math.sqrt(2.25), off


@pytest.mark.parametrize("B,Hq,Hk,Lq,Lk,d,W,causal,start", FEW + MANY)
def test_fp32(B, Hq, Hk, Lq, Lk, d, W, causal, start):
    """fp32: scores of size 1 from d products (sqrt(d) half-steps if independent), as many for dP, sums over n pairs (sqrt(n)), and a dozen
    for scaling, exponential and LSE."""
    off, n = errors(B, Hq, Hk, Lq, Lk, d, W, causal, F32, start)
    assert max(off.values()) <= (2 * math.sqrt(d) + math.sqrt(max(n, n * Lq / Lk * Hq / Hk)) + 12) * 2.0 ** -24, off


@pytest.mark.parametrize("B,Hq,Hk,Lq,Lk,W,causal,start,masked", [(1, 2, 2, 90, 90, 20, False, 0, False), (2, 4, 2, 70, 70, 70, True, 0, True),
                                                                (1, 4, 1, 5, 600, 1 << 20, True, 590, True)])
def test_gradients_against_differences(B, Hq, Hk, Lq, Lk, W, causal, start, masked):
    """The kernels' own forward in fp32 along a direction with the gradient's signs, so that its slope is the sum of magnitudes.  Difference of
    fourth order; its truncation is below the change from twice the step (15 times it), its noise at most O's bounds over the step, the
    gradient's at most its own.  All of it is below a twentieth of the slope."""
    print("\n[case]", B, Hq, Hk, Lq, Lk, W, causal, start, masked, flush=True)
    g = torch.Generator().manual_seed(8)
    d, eps = 32, 0.8
    x = [torch.randn(B, h, n, d, generator=g) for h, n in ((Hq, Lq), (Hk, Lk), (Hk, Lk))]
    do = torch.randn(B, Hq, Lq, d, generator=g)
    mask = (torch.rand(B, Lk, generator=g) > 0.3).to(torch.uint8) if masked else None
    at = torch.tensor([start] * B, dtype=torch.int32)
    want = ref.attn(*x, ref.pairs(B, Lq, Lk, W, causal, start=at, mask_k=mask), eps, do)
    kw = dict(causal=causal, eps=eps, start_q=at.cuda(), mask_k=None if mask is None else mask.cuda())
    c = [t.cuda() for t in x]
    O, LSE = ska.ska_softmax_attn_fwd(*c, W, **kw)
    grads = ska.ska_softmax_attn_bwd(*c, O, do.cuda(), LSE, W, **kw)
    for n, name in enumerate(("dQ", "dK", "dV")):
        u = torch.randn(x[n].shape, generator=g).abs() * want[name][0].sign().float()

        def f(h):
            y = list(c)
            y[n] = (x[n] + h * u).cuda()
            return (ska.ska_softmax_attn_fwd(*y, W, **kw)[0].double().cpu() * do.double()).sum().item()

        def slope(h):
            return (8 * (f(h) - f(-h)) - (f(2 * h) - f(-2 * h))) / (12 * h)
        h = 2.0 ** -5
        a, b = slope(h), slope(2 * h)
        got = (grads[n].double().cpu() * u.double()).sum().item()
        noise = 1.5 / h * ((want["O"][1] * do.abs()).sum() + 2.0 ** -23 * (want[name][0] * u).abs().sum()).item() + (want[name][1] * u.abs()).sum().item()
        limit = abs(a - b) + noise
        print(name, got, a, limit)
        assert limit < 0.05 * abs(a), (name, limit, a)
        assert abs(got - a) <= limit, (name, got, a, limit)
