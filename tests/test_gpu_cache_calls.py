"""Calls of the operators on caches as a program makes them: on other streams, captured and replayed, with tensors of its own, one after
another; and with arguments at the ends of their ranges."""
import sys

import pytest
import torch

import paper_2605_08123_amd as ska

from . import cache_ref as ref
from .layer_ref import check, pairs
from .test_gpu_cache import ALL, BF16, F32, cache_of, case, cuda, ints, kept, rnd, say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("W", [2 ** 31, 2 ** 32, sys.maxsize])
def test_a_band_of_everything(W):
    g = torch.Generator().manual_seed(1)
    q, k, v = (x.cuda() for x in case(g, 2, 4, 2, 3, 130, 64, BF16))
    cache = ska.ska_cache_write(ska.ska_cache_empty(2, 2, 130, 64), k, v)
    at = ints(120, 2 ** 31 - 1).cuda()
    for causal in (True, False):
        for call in (lambda w: ska.ska_cache_attn_fwd(q, cache, w, causal, start_q=at), lambda w: ska.ska_prefix_attn_fwd(q, (k[0], v[0]), (k, v), w, causal, start_q=at)):
            for a, b in zip(call(W), call(1 << 26)):
                assert torch.equal(a, b)


def test_refusals_of_the_binding():
    g = torch.Generator().manual_seed(1)
    q, k, v = (x.cuda() for x in case(g, 2, 4, 2, 3, 40, 64, BF16))
    c = ska.ska_cache_empty(2, 2, 40, 64)
    i8 = ska.ska_cache_empty(2, 2, 40, 64, "int8")
    pre, ipre = ska.KVCache(*(x[0] for x in c)), ska.KVCache(*(x[0] for x in i8))
    n, long = ints(1, 2).cuda(), ska.ska_cache_empty(2, 2, 20000, 64)
    for n_th, call in enumerate((
            lambda: ska.ska_cache_write(c, k, v[:, :, :39]),
            lambda: ska.ska_cache_write(c, k, v.float()),
            lambda: ska.ska_cache_write(c, k.half(), v.half()),
            lambda: ska.ska_cache_write(c, k[:1], v[:1]),
            lambda: ska.ska_cache_write(c, k[:, :1], v[:, :1]),
            lambda: ska.ska_cache_write((k, v, c[2], c[3]), k, v),
            lambda: ska.ska_cache_write((c.K, i8.V, c[2], c[3]), k, v),
            lambda: ska.ska_cache_write(c, k, v, start=n.long()),
            lambda: ska.ska_cache_write(c, k, v, start=n[:1]),
            lambda: ska.ska_cache_write(c, k, v, start=n.cpu()),
            lambda: ska.ska_cache_write(ska.KVCache(c.K, c.V, c.K_scale.double(), c.V_scale), k, v),
            lambda: ska.ska_cache_write(ska.KVCache(c.K, c.V, c.K_scale[:, :, :39], c.V_scale), k, v),
            lambda: ska.ska_cache_write(ska.KVCache(c.K, c.V, c.K_scale.transpose(1, 2).contiguous().transpose(1, 2), c.V_scale), k, v),
            lambda: ska.ska_cache_write(ska.KVCache(*(x[:1].expand(2, *x.shape[1:]) for x in c)), k, v),
            lambda: ska.ska_cache_write(ska.KVCache(*(x.cpu() for x in c)), k, v),
            lambda: ska.ska_cache_read(c, dtype=torch.float16),
            lambda: ska.ska_cache_read(c, K=k, V=v[:, :, :39]),
            lambda: ska.ska_cache_attn_fwd(q.float().double(), c, 4),
            lambda: ska.ska_cache_attn_fwd(q[:1], c, 4),
            lambda: ska.ska_cache_attn_fwd(q[:, :3], c, 4),
            lambda: ska.ska_cache_attn_fwd(q, (k, v), 4),
            lambda: ska.ska_cache_attn_fwd(q, c, 4, mask_k=n),
            lambda: ska.ska_cache_attn_fwd(q, c, -1),
            lambda: ska.ska_cache_attn_fwd(q, c, 4, eps=0.0),
            lambda: ska.ska_cache_attn_fwd(q, c, 4, O=q[:, :2]),
            lambda: ska.ska_cache_attn_fwd(q, long, ALL, workspace=torch.empty(8, dtype=torch.uint8, device="cuda")),
            lambda: ska.ska_prefix_attn_fwd(q, pre, i8, 4),
            lambda: ska.ska_prefix_attn_fwd(q, ipre, c, 4),
            lambda: ska.ska_prefix_attn_fwd(q, pre, (k, v), 4),
            lambda: ska.ska_prefix_attn_fwd(q, (k[0], v[0]), c, 4),
            lambda: ska.ska_prefix_attn_fwd(q, (k[0].float(), v[0].float()), (k, v), 4),
            lambda: ska.ska_prefix_attn_fwd(q, (k, v), (k, v), 4),
            lambda: ska.ska_prefix_attn_fwd(q, (k[0, :1], v[0, :1]), (k, v), 4),
            lambda: ska.ska_prefix_attn_fwd(q, (k[0], v[0]), (k, v), 4, len_p=n))):
        with pytest.raises((ValueError, TypeError, ska.SinkhornAttnError)):
            print(n_th, call())
    torch.cuda.synchronize()


def test_tensors_of_the_callers():
    """Queries in a projection's layout and broadcast over heads, results in views, a workspace given: the same bits, nothing around."""
    say("views")
    g = torch.Generator().manual_seed(2)
    B, Hq, Hk, Lq, Lk, d = 2, 4, 2, 3, 3000, 64
    k, v = (rnd(g, B, Hk, Lk, d, dtype=BF16).cuda() for _ in range(2))
    cache = ska.ska_cache_write(ska.ska_cache_empty(B, Hk, Lk, d), k, v)
    pre, (pk, pv) = ska.KVCache(*(x[1] for x in cache)), (k[1], v[1])
    wide = rnd(g, B, Lq, Hq + 2, d, dtype=BF16).cuda().transpose(1, 2)
    for q in (wide[:, 1:Hq + 1], wide[:, :1].expand(B, Hq, Lq, d)):
        for call, need in ((lambda q, **kw: ska.ska_cache_attn_fwd(q, cache, ALL, True, start_q=ints(2990, 5).cuda(), **kw), ska.ska_cache_attn_workspace_bytes(B, Hq, Hk, Lq, Lk, d, ALL, True)),
                           (lambda q, **kw: ska.ska_prefix_attn_fwd(q, pre, cache, ALL, start_q=ints(2990, 5).cuda(), **kw),
                            ska.ska_prefix_attn_workspace_bytes(B, Hq, Hk, Lq, Lk, Lk, d, ALL, True)),
                           (lambda q, **kw: ska.ska_prefix_attn_fwd(q, (pk, pv), (k, v), ALL, start_q=ints(2990, 5).cuda(), **kw),
                            ska.ska_prefix_attn_workspace_bytes(B, Hq, Hk, Lq, Lk, Lk, d, ALL, True, store=1))):
            O, LSE = call(q.contiguous())
            out = torch.full((B, Lq + 2, Hq + 3, d), 7.0, device="cuda", dtype=BF16)
            lse = torch.empty((B, Hq, Lq), device="cuda")
            ws = torch.full((need + 256,), 9, dtype=torch.uint8, device="cuda")
            into = out[:, 1:Lq + 1, 2:Hq + 2].transpose(1, 2)
            o, l = call(q, O=into, LSE=lse, workspace=ws[:need])
            assert o is into and l is lse and torch.equal(o, O) and torch.equal(l, LSE) and (ws[need:] == 9).all()
            into.fill_(7.0)
            assert (out == 7).all()
    # keys and values that all items and heads share, by strides of 0
    one = ska.KVCache(*(x[:1, :1].expand(B, Hk, *x.shape[2:]) for x in cache))
    q = wide[:, :Hq].contiguous()
    for a, b in zip(ska.ska_cache_attn_fwd(q, one, 100, True, start_q=ints(2990, 5).cuda()),
                    ska.ska_cache_attn_fwd(q, ska.KVCache(*(x.contiguous() for x in one)), 100, True, start_q=ints(2990, 5).cuda())):
        assert torch.equal(a, b)


@pytest.mark.parametrize("store", ["e4m3", "int8"])
def test_steps_captured_and_replayed(store):
    """A step of an answer (a token written, attention on the cache and behind a prefix) captured, and again into a second graph with the
    same workspaces, replayed in turn with eager work between: always what the eager calls give for the lengths that are there then."""
    say("graphs", store)
    g = torch.Generator().manual_seed(3)
    B, Hq, Hk, Lk, d, Lp = 3, 8, 2, 4000, 64, 5000
    n = ints(1000, 3000, 17).cuda()
    old = [rnd(g, B, Hk, Lk, d, dtype=BF16).cuda() for _ in range(2)]
    pre = ska.KVCache(*(x[0] for x in cache_of(rnd(g, 1, Hk, Lp, d), rnd(g, 1, Hk, Lp, d), store)))
    cache = ska.ska_cache_write(ska.ska_cache_empty(B, Hk, Lk, d, store), *old)
    q, k, v = (rnd(g, B, h, 1, d, dtype=BF16).cuda() for h in (Hq, Hk, Hk))
    new = [(rnd(g, B, Hq, 1, d, dtype=BF16), rnd(g, B, Hk, 1, d, dtype=BF16), rnd(g, B, Hk, 1, d, dtype=BF16)) for _ in range(6)]
    code = ska.cache._STORES[cache.K.dtype]
    ws = torch.empty(max(ska.ska_cache_attn_workspace_bytes(B, Hq, Hk, 1, Lk, d, ALL, True, store=code),
                         ska.ska_prefix_attn_workspace_bytes(B, Hq, Hk, 1, Lp, Lk, d, ALL, True, store=code)), dtype=torch.uint8, device="cuda")
    end = n + 1
    outs = [[torch.empty((B, Hq, 1, d), device="cuda", dtype=BF16) for _ in range(2)] for _ in range(2)]

    def step(c, o=(None, None), w=None):
        torch.add(n, 1, out=end)
        ska.ska_cache_write(c, k, v, start=n)
        a, _ = ska.ska_cache_attn_fwd(q, c, ALL, True, start_q=n, len_k=end, O=o[0], workspace=w)
        b, _ = ska.ska_prefix_attn_fwd(q, pre, c, ALL, start_q=n, len_k=end, O=o[1], workspace=w)
        return a, b
    twin = ska.KVCache(*(x.clone() for x in cache))
    step(ska.KVCache(*(x.clone() for x in cache)), outs[0], ws)     # (loads the kernels)
    torch.cuda.synchronize()
    graphs = []
    for o in outs:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step(cache, o, ws)
        graphs.append(graph)
    for i, (a, b, c) in enumerate(new):
        q.copy_(a); k.copy_(b); v.copy_(c)
        want = step(twin)
        graphs[i % 2].replay()
        if i % 3 == 0:
            torch.cuda.synchronize()
        for x, y in zip(outs[i % 2], want):
            assert torch.equal(x, y), i
        for x, y in zip(cache, twin):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8)), i
        ws.fill_(0xff)
        n += 1


def test_two_calls_at_once():
    """On streams of their own, each with its own workspace (by default): what they give one after another."""
    say("streams")
    g = torch.Generator().manual_seed(4)
    work = []
    for store, d, Lk in (("e4m3", 64, 9000), ("int8", 128, 7000)):
        k, v = (rnd(g, 2, 2, Lk, d, dtype=BF16).cuda() for _ in range(2))
        work.append((rnd(g, 2, 8, 1, d, dtype=BF16).cuda(), ska.ska_cache_write(ska.ska_cache_empty(2, 2, Lk, d, store), k, v), ints(Lk - 1, Lk // 2).cuda()))
    call = lambda q, c, at: ska.ska_cache_attn_fwd(q, c, ALL, True, start_q=at)   # noqa: E731
    want = [call(*w) for w in work]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in work]
    got = [[], []]
    for _ in range(20):
        for s, w, o in zip(streams, work, got):
            with torch.cuda.stream(s):
                o.append(call(*w))
    torch.cuda.synchronize()
    for o, w in zip(got, want):
        for a in o:
            assert torch.equal(a[0], w[0]) and torch.equal(a[1], w[1])


@pytest.mark.parametrize("store", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_prefix_is_the_same_keys_before(store, dtype):
    """A prompt written once and shared, each item's tokens behind it: what one cache per item that holds both gives, within both bounds."""
    say("prefix and cache", store, dtype)
    g = torch.Generator().manual_seed(5)
    B, Hq, Hk, Lq, Lp, Lk, d, W = 4, 8, 2, 3, 1500, 60, 64, 900
    pk, pv = (rnd(g, 1, Hk, Lp, d, dtype=dtype) for _ in range(2))
    k, v = (rnd(g, B, Hk, Lk, d, dtype=dtype) for _ in range(2))
    q, n = rnd(g, B, Hq, Lq, d, dtype=dtype), ints(60, 3, 31, 32)
    shared = ska.ska_cache_write(ska.ska_cache_empty(1, Hk, Lp, d, store), pk.cuda(), pv.cuda())
    own = ska.ska_cache_write(ska.ska_cache_empty(B, Hk, Lk, d, store), k.cuda(), v.cuda(), len_new=cuda(n))
    O, LSE = ska.ska_prefix_attn_fwd(q.cuda(), ska.KVCache(*(x[0] for x in shared)), own, W, start_q=cuda(n - 3), len_k=cuda(n))
    whole = ska.ska_cache_empty(B, Hk, Lp + Lk, d, store)
    ska.ska_cache_write(whole, pk.cuda().expand(B, -1, -1, -1), pv.cuda().expand(B, -1, -1, -1))
    ska.ska_cache_write(whole, k.cuda(), v.cuda(), start=ints(*[Lp] * B).cuda(), len_new=cuda(n))
    O1, LSE1 = ska.ska_cache_attn_fwd(q.cuda(), whole, W, True, start_q=cuda(n - 3 + Lp), len_k=cuda(n + Lp))
    kv = [torch.cat([ref.values(*kept(a, store)).expand(B, -1, -1, -1), ref.values(*kept(b, store))], 2) for a, b in ((pk, k), (pv, v))]
    want = ref.attn(q, *kv, pairs(B, Lq, Lp + Lk, W, True, start=n - 3 + Lp, len_k=n + Lp), 1.0)
    for o, l in ((O, LSE), (O1, LSE1)):
        check("O", o, want["O"])
        check("LSE", l, want["LSE"])


@pytest.mark.parametrize("store", ["e4m3", "int8"])
def test_an_answer_token_by_token(store):
    """Positions turned, tokens written as they come, attention after each: the cache is that of all at once bit for bit, and so are the
    outputs within the operator's bounds; read back, the banded Sinkhorn attention takes it."""
    say("answer", store)
    g = torch.Generator().manual_seed(6)
    B, Hq, Hk, L, d, W = 2, 4, 4, 50, 64, 20
    freq, amp = ska.ska_rope_frequencies(d)
    q, k, v = (rnd(g, B, h, L, d, dtype=BF16).cuda() for h in (Hq, Hk, Hk))
    Q, K = ska.ska_rope_fwd(q, k, freq.cuda(), amp)
    once = ska.ska_cache_write(ska.ska_cache_empty(B, Hk, L, d, store), K, v)
    O, LSE = ska.ska_cache_attn_fwd(Q, once, W, True)
    want = ref.attn(Q.cpu(), *(ref.values(c.cpu().float(), s.cpu()) for c, s in ((once.K, once.K_scale), (once.V, once.V_scale))), pairs(B, L, L, W, True), 1.0)
    check("O", O, want["O"])
    steps = ska.ska_cache_empty(B, Hk, L, d, store)
    n, out = torch.zeros(B, dtype=torch.int32, device="cuda"), []
    for t in range(L):
        one = slice(t, t + 1)
        Qt, Kt = ska.ska_rope_fwd(q[:, :, one], k[:, :, one], freq.cuda(), amp, start=n)
        ska.ska_cache_write(steps, Kt, v[:, :, one], start=n)
        out.append(ska.ska_cache_attn_fwd(Qt, steps, W, True, start_q=n, len_k=n + 1)[0])
        n = n + 1
    for a, b in zip(steps, once):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    check("O", torch.cat(out, 2), want["O"])
    Kr, Vr = ska.ska_cache_read(steps)
    S, _ = ska.sinkhorn_attn_fwd(Q, Kr, Vr, W, 4, 2, 1.0)
    assert torch.isfinite(S).all() and S.shape == Q.shape
