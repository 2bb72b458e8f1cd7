"""The layer operators (include/sinkhorn_attn_layer.h) on the GPU against their 64-bit definitions, entry by entry within the
bounds of tests/layer_ref.py, at the sizes, masks, strides and streams where they can go wrong."""
import math

import pytest
import torch

import paper_2605_08123_amd as ska

from . import layer_ref as ref

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def rnd(g, *shape, dtype=F32, scale=1.0, shift=0.0):
    return (torch.randn(*shape, generator=g) * scale + shift).to(dtype)


def say(*what):
    print("\n[case]", *what, flush=True)


# ------------------------------------------------------------------ layer norm
NORM = [  # rows, D: one feature to rows that do not fit registers, widths around every change of shape
    (1, 1), (3, 2), (1, 5), (7, 8), (130, 17), (33, 64), (5, 100), (257, 128), (64, 511), (65, 512), (66, 513), (9, 1024), (31, 1283),
    (6, 2047), (4, 2049), (3, 4100), (5, 8192), (2, 8200), (3, 16385), (2, 65536)]


@pytest.mark.parametrize("dtype,wdtype", [(F32, F32), (BF16, F32), (BF16, BF16), (F32, BF16)])
@pytest.mark.parametrize("rows,D", NORM)
def test_layer_norm(rows, D, dtype, wdtype):
    say("layer norm", rows, D, dtype, wdtype)
    g = torch.Generator().manual_seed(rows * 7919 + D)
    for residual in (False, True):
        x, r = rnd(g, rows, D, dtype=dtype, shift=0.5), rnd(g, rows, D, dtype=dtype) if residual else None
        w, b = rnd(g, D, dtype=wdtype, scale=0.3, shift=1.0), rnd(g, D, dtype=wdtype)
        dy, ds = rnd(g, rows, D, dtype=dtype), rnd(g, rows, D, dtype=dtype) if residual else None
        c = lambda t: None if t is None else t.cuda()   # noqa: E731
        Y, S, stats = ska.ska_layer_norm_fwd(c(x), c(w), c(b), residual=c(r))
        s, y, mean, rstd = ref.norm_fwd(x, w, b, r, 1e-5)
        assert torch.equal(S.cpu(), s)
        ref.check("Y", Y, y)
        ref.check("mean", stats[0], mean)
        ref.check("rstd", stats[1], rstd)
        st = torch.stack([mean[0], rstd[0]]).float()
        got = ska.ska_layer_norm_bwd(c(dy), c(s), c(w), c(st), dS=c(ds))
        for name, t, want in zip(("dX", "dweight", "dbias"), got, ref.norm_bwd(dy, s, w, st, ds, wdtype)):
            ref.check(name, t, want)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,D", [(40003, 40), (9001, 512), (5003, 1283), (3001, 2100), (2051, 4200), (1601, 8192), (700, 9000)])
def test_layer_norm_many_rows(rows, D, dtype):
    """More rows than a launch has room for at a time, also in place."""
    say("layer norm, many rows", rows, D, dtype)
    g = torch.Generator().manual_seed(rows + D)
    s, dy, ds = (rnd(g, rows, D, dtype=dtype) for _ in range(3))
    w = rnd(g, D, scale=0.3, shift=1.0)
    _, _, mean, rstd = ref.norm_fwd(s, None, None, None, 1e-5)
    st = torch.stack([mean[0], rstd[0]]).float()
    x = dy.cuda()
    got = ska.ska_layer_norm_bwd(x, s.cuda(), w.cuda(), st.cuda(), dS=ds.cuda())
    for name, t, want in zip(("dX", "dweight", "dbias"), got, ref.norm_bwd(dy, s, w, st, ds, F32)):
        ref.check(name, t, want)
    again = ska.ska_layer_norm_bwd(x, s.cuda(), w.cuda(), st.cuda(), dS=ds.cuda(), dX=x)
    assert all(torch.equal(a, b) for a, b in zip(got, again))


@pytest.mark.parametrize("D", [96, 1000, 20000])
def test_layer_norm_strides_and_places(D):
    """Rows apart, rows that start on any element, results in the inputs' place, no weights, only some of the results."""
    say("layer norm strides", D)
    g = torch.Generator().manual_seed(D)
    for dtype in (F32, BF16):
        wide = rnd(g, 4, 6, D + 13, dtype=dtype).cuda()
        x = wide[:, :, 5:5 + D]
        s, y, mean, rstd = ref.norm_fwd(x.cpu(), None, None, None, 1e-3)
        st = torch.stack([mean[0], rstd[0]]).float().cuda()
        out = torch.full((4, 6, D + 3), 7.0, device="cuda", dtype=dtype)
        ska.ska_layer_norm_fwd(x, eps=1e-3, Y=out[:, :, 2:2 + D])
        ref.check("Y", out[:, :, 2:2 + D], y)
        assert (out[:, :, :2] == 7).all() and (out[:, :, 2 + D:] == 7).all()
        dy, ds = rnd(g, 4, 6, D, dtype=dtype).cuda(), rnd(g, 1, 6, D, dtype=dtype).cuda()
        want = ref.norm_bwd(dy.cpu(), s, None, st.cpu(), None, F32)
        a, w1, b1 = ska.ska_layer_norm_bwd(dy, x, None, st)
        ref.check("dX", a, want[0])
        ref.check("dweight", w1, want[1])
        ref.check("dbias", b1, want[2])
        _, w2, b2 = ska.ska_layer_norm_bwd(dy, x, None, st, want_bias=False)
        assert torch.equal(w1, w2) and b2 is None
        _, w3, b3 = ska.ska_layer_norm_bwd(dy, x, None, st, want_weight=False)
        assert w3 is None and torch.equal(b1, b3)
        # in place: dX over dY, and Y and S over X and the residual
        inplace = dy.clone()
        got, w4, b4 = ska.ska_layer_norm_bwd(inplace, x, None, st, dX=inplace)
        assert torch.equal(got, a) and torch.equal(w1, w4) and torch.equal(b1, b4)
        r = rnd(g, 4, 6, D, dtype=dtype).cuda()
        Y0, S0, _ = ska.ska_layer_norm_fwd(x, residual=r)
        x1, r1 = x.contiguous(), r.clone()
        Y1, S1, _ = ska.ska_layer_norm_fwd(x1, residual=r1, Y=x1, S=r1)
        assert torch.equal(Y0, Y1) and torch.equal(S0, S1)
        # a broadcast gradient on the residual's way
        full = ska.ska_layer_norm_bwd(dy[0], x[0], None, st[:, 0].contiguous(), dS=ds[0, :1].expand(6, D))[0]
        ref.check("dX", full, ref.norm_bwd(dy[0].cpu(), s[0], None, st[:, 0].cpu(), ds[0, :1].expand(6, D).cpu(), F32)[0])


def test_layer_norm_without_rows():
    x = torch.zeros((0, 64), device="cuda")
    w = torch.ones(64, device="cuda")
    Y, _, st = ska.ska_layer_norm_fwd(x, w, w)
    dX, dw, db = ska.ska_layer_norm_bwd(x, x, w, st, dweight=torch.full_like(w, 9.0), dbias=torch.full_like(w, 9.0))
    assert Y.shape == dX.shape == (0, 64) and not dw.any() and not db.any()


# ------------------------------------------------------------------ rotary positions
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,Hq,Hk,L,d,rot", [(1, 1, 0, 1, 2, 2), (2, 3, 1, 1, 64, 64), (1, 2, 2, 5, 64, 32), (2, 8, 4, 130, 128, 64), (1, 4, 2, 77, 32, 10),
                                             (3, 2, 1, 33, 33, 6), (1, 1, 1, 300, 128, 128), (2, 5, 5, 64, 96, 48), (1, 2, 1, 9, 4096, 4096)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rope(B, Hq, Hk, L, d, rot, interleaved, dtype):
    say("rope", B, Hq, Hk, L, d, rot, interleaved, dtype)
    g = torch.Generator().manual_seed(L * 131 + d)
    freq, amp = ska.ska_rope_frequencies(rot, 10000.0, "yarn", 8.0, 4096)
    amp = torch.tensor(amp, dtype=F32).item()
    q, k = rnd(g, B, Hq, L, d, dtype=dtype), rnd(g, B, Hk, L, d, dtype=dtype) if Hk else None
    start = torch.randint(-5, 250000, (B,), generator=g, dtype=torch.int32)
    each = torch.randint(0, 2 ** 31 - 1, (B, L), generator=g, dtype=torch.int32)
    f = freq.cuda()
    for pos, kw in ((torch.arange(L).expand(B, L), {}), (torch.arange(L) + start[:, None], dict(start=start.cuda())), (each, dict(positions=each.cuda()))):
        for back, call in ((False, ska.ska_rope_fwd), (True, ska.ska_rope_bwd)):
            qo, ko = call(q.cuda(), k.cuda() if Hk else None, f, amp, interleaved, **kw)
            ref.check("Q", qo, ref.rope(q, freq, amp, pos, interleaved, back))
            if Hk:
                ref.check("K", ko, ref.rope(k, freq, amp, pos, interleaved, back))
            else:
                assert ko is None


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rope_strides_and_places(interleaved, dtype):
    """A projection's [B, L, H, d], results into it, in place, rows on any element, and broadcast heads: all the same bits."""
    say("rope strides", interleaved, dtype)
    g = torch.Generator().manual_seed(11)
    B, Hq, Hk, L, d = 2, 4, 2, 37, 64
    freq = ska.ska_rope_frequencies(32)[0].cuda()
    q, k = rnd(g, B, Hq, L, d, dtype=dtype).cuda(), rnd(g, B, Hk, L, d, dtype=dtype).cuda()
    a, b = ska.ska_rope_fwd(q, k, freq, 1.25, interleaved)
    qkv = torch.full((B, L, Hq + Hk, d), 3.0, device="cuda", dtype=dtype)
    qkv[:, :, :Hq], qkv[:, :, Hq:] = q.transpose(1, 2), k.transpose(1, 2)
    qv, kv = qkv[:, :, :Hq].transpose(1, 2), qkv[:, :, Hq:].transpose(1, 2)
    c, e = ska.ska_rope_fwd(qv, kv, freq, 1.25, interleaved)
    assert c.is_contiguous() and torch.equal(a, c) and torch.equal(b, e)
    ska.ska_rope_fwd(qv, kv, freq, 1.25, interleaved, Qr=qv, Kr=kv)
    assert torch.equal(a, qv) and torch.equal(b, kv)
    odd = torch.zeros((B, Hq, L, d + 3), device="cuda", dtype=dtype)[..., 1:d + 1]
    odd.copy_(q)
    assert torch.equal(ska.ska_rope_fwd(odd, None, freq, 1.25, interleaved)[0], a)
    one = q[:, :1].expand(B, Hq, L, d)
    assert torch.equal(ska.ska_rope_fwd(one, None, freq, 1.25, interleaved)[0], a[:, :1].expand(B, Hq, L, d))
    empty = torch.zeros((B, Hq, 0, d), device="cuda", dtype=dtype)
    assert ska.ska_rope_fwd(empty, None, freq)[0].shape == (B, Hq, 0, d)


# ------------------------------------------------------------------ softmax attention
def attn_case(B, Hq, Hk, Lq, Lk, d, W, causal=False, eps=1.0, dtype=BF16, start=None, len_q=None, len_k=None, mask_q=None, mask_k=None,
              seed=0, scale=1.0, junk=False):
    say("attention", B, Hq, Hk, Lq, Lk, d, W, causal, eps, dtype, start, len_q, len_k, mask_q is not None, mask_k is not None)
    g = torch.Generator().manual_seed(seed + Lq * 31 + Lk * 17 + d + W)
    q, k, v, do = (rnd(g, B, h, n, d, dtype=dtype, scale=s) for h, n, s in ((Hq, Lq, scale), (Hk, Lk, scale), (Hk, Lk, 1.0), (Hq, Lq, 1.0)))
    i32 = lambda x: None if x is None else torch.tensor(x, dtype=torch.int32)   # noqa: E731
    where = dict(start=i32(start), len_q=i32(len_q), len_k=i32(len_k), mask_q=mask_q, mask_k=mask_k)
    ok = ref.pairs(B, Lq, Lk, W, causal, **where)
    want = ref.attn(q, k, v, ok, eps, do)
    if junk:   # what inactive tokens and padding hold
        dead_q, dead_k = torch.zeros(B, Lq, dtype=torch.bool), torch.zeros(B, Lk, dtype=torch.bool)
        for dead, n, m in ((dead_q, where["len_q"], mask_q), (dead_k, where["len_k"], mask_k)):
            if n is not None:
                dead |= torch.arange(dead.shape[1]) >= n[:, None]
            if m is not None:
                dead |= m == 0
        for x, dead in ((q, dead_q), (do, dead_q), (k, dead_k), (v, dead_k)):
            x[dead[:, None].expand(x.shape[:3])] = torch.tensor([math.nan, math.inf, -math.inf, torch.finfo(dtype).min] * (d // 4), dtype=dtype)
    c = lambda t: None if t is None else t.cuda()   # noqa: E731
    kw = dict(causal=causal, eps=eps, start_q=c(where["start"]), len_q=c(where["len_q"]), len_k=c(where["len_k"]), mask_q=c(mask_q), mask_k=c(mask_k))
    O, LSE = ska.ska_softmax_attn_fwd(c(q), c(k), c(v), W, **kw)
    torch.cuda.synchronize()
    ref.check("O", O, want["O"])
    ref.check("LSE", LSE, want["LSE"])
    o, lse = c(want["O"][0].to(dtype)), c(want["LSE"][0].float())
    grads = ska.ska_softmax_attn_bwd(c(q), c(k), c(v), o, c(do), lse, W, **kw)
    torch.cuda.synchronize()
    for name, x in zip(("dQ", "dK", "dV"), grads):
        ref.check(name, x, want[name])
    return want


SIZES = [  # Hq, Hk, Lq = Lk, W: single tokens, ends inside and on tiles, bands narrower and wider than a tile, all pairs
    (1, 1, 1, 0), (1, 1, 1, 5), (2, 1, 2, 0), (1, 1, 31, 3), (2, 2, 32, 64), (1, 1, 33, 33), (4, 2, 63, 1), (2, 1, 64, 0), (3, 1, 65, 20),
    (1, 1, 127, 128), (2, 2, 129, 31), (8, 2, 200, 64), (5, 1, 257, 300), (1, 1, 515, 65), (2, 2, 700, 128), (4, 4, 300, 16)]


@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("Hq,Hk,L,W", SIZES)
def test_attention_sizes(Hq, Hk, L, W, causal, dtype, d):
    attn_case(1 + L % 2, Hq, Hk, L, L, d, W, causal, eps=0.5 if W else 1.0, dtype=dtype)


@pytest.mark.parametrize("B,Hq,Hk,L,W,causal,dtype,d", [
    (2, 16, 16, 1030, 1030, True, BF16, 64), (2, 16, 16, 1030, 1030, True, F32, 32),   # between one and two wavefronts per SIMD, walks of every length
    (1, 16, 16, 1030, 2000, False, F32, 64), (1, 16, 16, 1030, 2000, False, BF16, 32),   # more than half of one, walks of one length
    (2, 16, 16, 1030, 20, False, F32, 128), (2, 32, 16, 1030, 40, True, F32, 64),   # a band of many rows, single wavefronts for the keys in fp32
    (1, 6, 2, 1600, 1600, False, BF16, 128), (1, 8, 2, 900, 900, True, F32, 128)])
def test_attention_many_rows(B, Hq, Hk, L, W, causal, dtype, d):
    """Enough rows for the other choices of workgroups and of parts of a walk."""
    attn_case(B, Hq, Hk, L, L, d, W, causal, dtype=dtype)


@pytest.mark.parametrize("dtype,d", [(F32, 32), (F32, 128), (BF16, 64), (BF16, 128)])
@pytest.mark.parametrize("Hq,Hk,Lq,Lk,W", [(8, 2, 1, 1000, 1 << 30), (1, 1, 1, 1, 0), (4, 4, 1, 3000, 100), (6, 2, 17, 900, 1 << 25), (2, 1, 5, 5, 7),
                                           (2, 1, 40, 2500, 5000), (4, 1, 1, 20000, 1 << 20), (1, 1, 300, 2, 400), (2, 2, 1500, 3, 1 << 20)])
def test_attention_cached(Hq, Hk, Lq, Lk, W, dtype, d):
    """Other numbers of queries than of keys: the last tokens of ragged caches, and few keys under many queries."""
    B = 3
    lens = [max(1, Lk - 7 * b - (Lk // 3) * (b == 2)) for b in range(B)]
    attn_case(B, Hq, Hk, Lq, Lk, d, W, True, dtype=dtype, start=[max(0, n - Lq) for n in lens], len_k=lens, junk=True)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("L,W", [(70, 5), (200, 200), (333, 40)])
def test_attention_lengths_and_masks(L, W, causal, dtype):
    """Rows that nothing reaches, lengths of zero and one, beyond L and negative; inactive tokens hold NaN, infinities and lowest values."""
    g = torch.Generator().manual_seed(L)
    B = 6
    len_q, len_k = [0, 1, L, L + 9, L // 2, L], [L, L, 1, L // 3, 0, -4]
    attn_case(B, 4, 2, L, L, 64, W, causal, dtype=dtype, len_q=len_q, len_k=len_k, junk=True)
    mq, mk = ((torch.rand(B, L, generator=g) > p).to(torch.uint8) * 200 for p in (0.3, 0.6))
    mq[0], mk[1] = 0, 0
    mk[2, L // 4:] = 0   # a band without a key for later queries
    want = attn_case(B, 2, 2, L, L, 32, W, causal, dtype=dtype, mask_q=mq, mask_k=mk, junk=True)
    assert torch.isinf(want["LSE"][0]).any()
    attn_case(B, 3, 1, L, L, 128, W, causal, dtype=dtype, len_q=[L, 5, L, L - 1, 33, 64], len_k=[L - 3, L, 31, 1, 65, L], mask_q=mq, mask_k=mk,
              start=[0, 3, 0, 40, 1, L], junk=True)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_attention_far_scores(dtype):
    """Scores of hundreds: sums that start at one and end many powers of two higher, along a row and across the parts of a walk."""
    attn_case(1, 2, 1, 257, 257, 64, 300, dtype=dtype, scale=6.0)
    attn_case(1, 2, 1, 2, 4000, 64, 1 << 20, dtype=dtype, scale=6.0, start=[4000])


def test_attention_strides():
    """Heads of a projection, a cache with room to spare, broadcast keys, results into a projection: the same bits."""
    say("attention strides")
    g = torch.Generator().manual_seed(3)
    for dtype in (F32, BF16):
        B, Hq, Hk, L, d, W = 2, 4, 2, 150, 64, 30
        q, k, v, do = (rnd(g, B, h, L, d, dtype=dtype).cuda() for h in (Hq, Hk, Hk, Hq))
        O, LSE = ska.ska_softmax_attn_fwd(q, k, v, W)
        grads = ska.ska_softmax_attn_bwd(q, k, v, O, do, LSE, W)
        t = lambda x: x.transpose(1, 2).contiguous().transpose(1, 2)   # noqa: E731
        room = torch.full((B, Hk, 2 * L, 2 * d), math.nan, device="cuda", dtype=dtype)
        kc, vc = room[:, :, :L, :d], room[:, :, L:, d:]
        kc.copy_(k)
        vc.copy_(v)
        out = torch.empty((B, L, Hq, d), device="cuda", dtype=dtype).transpose(1, 2)
        O2, LSE2 = ska.ska_softmax_attn_fwd(t(q), kc, vc, W, O=out)
        assert torch.equal(O, O2) and torch.equal(LSE, LSE2)
        dq, dk = (torch.empty((B, L, h, d), device="cuda", dtype=dtype).transpose(1, 2) for h in (Hq, Hk))
        dv = torch.empty((B, Hk, L, 2 * d), device="cuda", dtype=dtype)[..., :d]
        got = ska.ska_softmax_attn_bwd(t(q), kc, vc, out, t(do), LSE, W, dQ=dq, dK=dk, dV=dv)
        assert all(torch.equal(x, y) for x, y in zip(grads, got))
        one_k, one_v = k[:1, :1].expand(B, Hk, L, d), v[:1, :1].expand(B, Hk, L, d)
        same = ska.ska_softmax_attn_fwd(q, one_k.contiguous(), one_v.contiguous(), W)
        assert torch.equal(ska.ska_softmax_attn_fwd(q, one_k, one_v, W)[0], same[0])
        single = q[:, :, 3:4].transpose(1, 2).contiguous().transpose(1, 2)   # one token: its stride may be anything
        assert torch.equal(ska.ska_softmax_attn_fwd(single.as_strided(single.shape, (Hq * d, d, 3, 1)), k, v, W)[0],
                           ska.ska_softmax_attn_fwd(single.contiguous(), k, v, W)[0])


def test_attention_misaligned_is_refused():
    x = torch.zeros((1, 1, 8, 72), device="cuda", dtype=BF16)
    with pytest.raises(ska.SinkhornAttnError) as e:
        ska.ska_softmax_attn_fwd(x[..., 4:68], x[..., :64], x[..., :64], 3)
    assert e.value.status == -2
    with pytest.raises(ValueError):
        ska.ska_softmax_attn_fwd(x[..., :64], x[..., :64].float(), x[..., :64], 3)


def test_attention_difference():
    """The kernels' own forward: a directional difference in fp32.  O's bound at either end over 2 h, and h^2 / 6 of a third derivative,
    estimated by the next larger step's difference (four times the error)."""
    say("difference")
    g = torch.Generator().manual_seed(8)
    B, H, L, d, W = 1, 2, 90, 32, 20
    q, k, v, do = (rnd(g, B, H, L, d) for _ in range(4))
    want = ref.attn(q, k, v, ref.pairs(B, L, L, W, False), 1.0, do)
    O, LSE = ska.ska_softmax_attn_fwd(q.cuda(), k.cuda(), v.cuda(), W)
    grads = ska.ska_softmax_attn_bwd(q.cuda(), k.cuda(), v.cuda(), O, do.cuda(), LSE, W)
    x = [q, k, v]
    for n in range(3):
        u = rnd(g, B, H, L, d)

        def diff(h):
            ends = []
            for sign in (1, -1):
                y = list(x)
                y[n] = x[n] + sign * h * u
                ends.append((ska.ska_softmax_attn_fwd(*(t.cuda() for t in y), W)[0].double().cpu() * do.double()).sum().item())
            return (ends[0] - ends[1]) / (2 * h)
        h = 2.0 ** -6
        a, b = diff(h), diff(2 * h)
        noise = ((want["O"][1] * do.abs()).sum() / h + 2.0 ** -24 * (x[n].abs() * u.abs()).sum() / h * 0).item()
        grad = (grads[n].double().cpu() * u.double()).sum().item()
        assert abs(grad - a) <= 2 * abs(a - b) + 2 * noise + 1e-4 * (grads[n].cpu().abs() * u.abs()).sum().item(), (n, grad, a, b, noise)


# ------------------------------------------------------------------ streams, graphs, repeats
def _everything(x):
    """All operators once, as a layer would run them."""
    Y, S, st = ska.ska_layer_norm_fwd(x["x"], x["w"], x["w"], residual=x["r"])
    q = Y.view(x["B"], x["L"], x["H"], x["d"]).transpose(1, 2)
    Qr, Kr = ska.ska_rope_fwd(q, q[:, :x["Hk"]], x["f"], 1.1)
    V = q[:, :x["Hk"]]
    O, LSE = ska.ska_softmax_attn_fwd(Qr, Kr, V, x["W"], causal=x["causal"])
    dQr, dKr, dV = ska.ska_softmax_attn_bwd(Qr, Kr, V, O, O, LSE, x["W"], causal=x["causal"])
    dQ, dK = ska.ska_rope_bwd(dQr, dKr, x["f"], 1.1)
    dx = ska.ska_layer_norm_bwd(dQ.transpose(1, 2).reshape(S.shape), S, x["w"], st, dS=S)
    return [Y, S, st, Qr, Kr, O, LSE, dQ, dK, dV, *dx]


def _inputs(B, H, Hk, L, d, W, causal, dtype=BF16):
    g = torch.Generator().manual_seed(L)
    return dict(B=B, H=H, Hk=Hk, L=L, d=d, W=W, causal=causal, x=rnd(g, B * L, H * d, dtype=dtype).cuda(), r=rnd(g, B * L, H * d, dtype=dtype).cuda(),
                w=rnd(g, H * d, shift=1.0).cuda(), f=ska.ska_rope_frequencies(d)[0].cuda())


def test_other_stream_and_repeats():
    """On a stream of its own, between work on others, and again: the same bits."""
    say("streams")
    x = _inputs(2, 4, 2, 300, 64, 50, True)
    first = _everything(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = _everything(x)
    again = _everything(x)
    torch.cuda.synchronize()
    for a, b, c in zip(first, other, again):
        assert torch.equal(a, b) and torch.equal(a, c)


@pytest.mark.parametrize("shape", [(2, 4, 2, 300, 64, 50, True), (1, 2, 1, 1024, 64, 1024, False)])
def test_graph_replays(shape):
    """Captured (with joined parts in the second), replayed on changed inputs between eager runs: every replay is the eager result."""
    say("graph", shape)
    x = _inputs(*shape)
    _everything(x)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = _everything(x)
    for n in range(4):
        x["x"].copy_(torch.randn(x["x"].shape, generator=torch.Generator().manual_seed(n)).to(BF16).cuda())
        eager = [t.clone() for t in _everything(x)]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, eager):
            assert torch.equal(a, b), n
        assert all(torch.equal(a, b) for a, b in zip(_everything(x), eager))


def test_far_offsets():
    """A cache whose rows lie beyond 2^31 elements and 2^32 bytes: the last keys of a [1, 1, L, d] view with a wide token stride."""
    say("far offsets")
    d, L, stride = 64, 300, 1 << 23   # 300 * 2^23 elements = 5 GB in bf16
    g = torch.Generator().manual_seed(2)
    flat = torch.empty(L * stride, device="cuda", dtype=BF16)
    k = flat.as_strided((1, 1, L, d), (0, 0, stride, 1))
    v = flat[d:].as_strided((1, 1, L, d), (0, 0, stride, 1))
    q, k0, v0 = (rnd(g, 1, h, n, d, dtype=BF16).cuda() for h, n in ((2, L), (1, L), (1, L)))
    k.copy_(k0)
    v.copy_(v0)
    a, b = ska.ska_softmax_attn_fwd(q, k0, v0, 40), ska.ska_softmax_attn_fwd(q, k, v, 40)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    ga, gb = (ska.ska_softmax_attn_bwd(q, kk, vv, a[0], q, a[1], 40) for kk, vv in ((k0, v0), (k, v)))
    assert all(torch.equal(x, y) for x, y in zip(ga, gb))
    f = ska.ska_rope_frequencies(d)[0].cuda()
    assert torch.equal(ska.ska_rope_fwd(k, None, f)[0], ska.ska_rope_fwd(k0, None, f)[0])
    x0, x1 = k0.view(L, d), k.as_strided((L, d), (stride, 1))
    assert torch.equal(ska.ska_layer_norm_fwd(x0)[0], ska.ska_layer_norm_fwd(x1)[0])
