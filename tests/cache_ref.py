"""The operators on caches (include/sinkhorn_attn_cache.h) in 64 bits by their definitions, on the CPU; attention with a bound on what a
correct implementation may differ by (as in tests/layer_ref.py), what is written and read back with none."""
import math

import torch

from .layer_ref import F32, half, pairs

SMALLEST, LARGEST = 2.0 ** -126, float.fromhex("0x1.020406p+121")   # of an int8 row's scale


def e4m3_numbers():
    """The 127 numbers from 0 to 448, in the order of their codes."""
    return torch.tensor([m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7) for e in range(16) for m in range(8)][:127], dtype=torch.float64)


def quantise(x, store):
    """Rows [..., d] (storage tensor) -> codes as float64 numbers, scales as float64 numbers of fp32."""
    f = x.double()
    bad = ~torch.isfinite(f).all(-1, keepdim=True)
    f = torch.where(bad, 0.0, f)
    a = f.abs().amax(-1, keepdim=True)
    if store == "int8":
        s = (a.float() / 127).clamp(SMALLEST, LARGEST).double()   # (one correctly rounded division)
        y = f / s                                            # 24-bit by 24-bit numbers: no quotient but a half is rounded to a half in 53 bits
        c = torch.round(y).clamp(-127, 127)
    else:
        e = torch.full_like(a, -126.0)
        for k in range(-126, 121):
            e = torch.where(448 * 2.0 ** (k - 1) < a, float(k), e)
        s = torch.exp2(e)
        numbers = e4m3_numbers()
        y = (f / s).abs()
        y = torch.where(s == 2.0 ** 120, y.clamp(max=240), y)   # (256 2^120 is infinite)
        mid = (numbers[1:] + numbers[:-1]) / 2
        i = torch.searchsorted(mid, y.contiguous())          # the number below or at a border, even ones' borders belong to them
        i = i + ((y == mid[i.clamp(max=125)]) & (i % 2 == 1))
        c = torch.copysign(numbers[i.clamp(max=126)], f)
    return torch.where(bad, 0.0, c), torch.where(bad, math.nan, s)[..., 0]


def values(codes, scales):
    return codes.double() * scales.double()[..., None]


def prefix_pairs(B, Lq, P, Lp, W, start, len_q, mask_q, mask_p):
    """Which query meets which key of a prefix of Lp places, P of them there."""
    p = P + torch.arange(Lq)[None, :, None] + (0 if start is None else start[:, None, None].long())
    j = torch.arange(Lp)[None, None]
    ok = ((p - j) <= W) & (j < P)
    ok = ok.expand(B, Lq, Lp).clone()
    if len_q is not None:
        ok &= torch.arange(Lq)[None, :, None] < len_q[:, None, None]
    if mask_q is not None:
        ok &= mask_q.bool()[:, :, None]
    if mask_p is not None:
        ok &= mask_p.bool()[None, None]
    return ok


def attn(q, k, v, ok, eps, codes=True):
    """q [B,Hq,Lq,d] storage, k, v [B,Hk,L,d] float64 values (codes: of 8-bit codes), ok [B,Lq,L].  (value, bound) of O and LSE.  Tokens that take part in no pair are
    left out before anything is multiplied."""
    B, Hq, Lq, d = q.shape
    G = Hq // k.shape[1]
    row, key = ok.any(2), ok.any(1)
    clean = lambda x, on: torch.where(on[:, None, :, None], x.double(), 0.0)   # noqa: E731
    qd, kd, vd = clean(q, row), clean(k, key).repeat_interleave(G, 1), clean(v, key).repeat_interleave(G, 1)
    c = 1 / (eps * math.sqrt(d))
    okh = ok[:, None].expand(B, Hq, Lq, ok.shape[2])
    s = torch.where(okh, qd @ kd.transpose(-1, -2) * c, -math.inf)
    top = s.amax(-1, keepdim=True)
    top0 = torch.where(top > -math.inf, top, 0.0)
    e = torch.exp(s - top0)
    total = e.sum(-1, keepdim=True)
    p = e / torch.where(total > 0, total, 1.0)
    lse, o = (top + total.log())[..., 0], p @ vd
    n = ok.sum(2).double()[:, None, :, None]
    # scores: d products (three parts of an fp32 query: 3 d), scaled by the key's scale and the temperature; the exponent as in softmax attention
    mag = (qd.abs() @ kd.abs().transpose(-1, -2)) * c
    e_s = (3 * d + 6) * F32 * mag
    e_exp = e_s + 4 * F32 * (torch.where(okh, s, 0.0).abs() + top0.abs()) + 4 * F32
    worst = torch.where(okh, e_exp, 0.0).amax(-1, keepdim=True)
    # P and the value's scale: in fp32 results all their bits; in bf16 ones of codes three fp16 roundings (P, the scale next to its unit, their
    # product: 2^-11 each, and half of the smallest fp16 number, 2^-25, in P, which is counted in 2^-4, and in the product, where the value
    # is counted in at most twice the largest: 2^-29 + 2^-28, with the row's sum at least 1 in P's units); of bf16 values P as two bf16 numbers, 2^-16.  Three sums of n terms
    parts, tiny = F32, 0.0
    if q.dtype == torch.bfloat16:
        parts, tiny = (3 * 2.0 ** -11, 2.0 ** -27 * n * vd.abs().amax()) if codes else (half(torch.bfloat16) ** 2, 0.0)
    e_o = (p @ vd.abs()) * (parts + 2 * worst + 3 * n * F32 + 12 * F32) * 1.02 + tiny + half(q.dtype) * o.abs()
    # (sums of P before it is rounded, or of two bf16 numbers)
    e_lse = (worst + n * F32 + (F32 if codes else parts))[..., 0] + 4 * F32 * (lse.abs().nan_to_num(posinf=0.0) + top0[..., 0].abs()) + 4 * F32
    return {"O": (o, e_o), "LSE": (lse, e_lse)}


def prefix_attn(q, pk, pv, k, v, W, causal, eps, P=None, start=None, len_q=None, len_k=None, mask_q=None, mask_k=None, mask_p=None, codes=True):
    """pk, pv [Hk,Lp,d], k, v [B,Hk,Lk,d] float64 values."""
    B, Lq, Lp = q.shape[0], q.shape[2], pk.shape[1]
    ok = torch.cat([prefix_pairs(B, Lq, Lp if P is None else P, Lp, W, start, len_q, mask_q, mask_p),
                    pairs(B, Lq, k.shape[2], W, causal, start, len_q, len_k, mask_q, mask_k)], 2)
    both = lambda a, b: torch.cat([a[None].expand(B, *a.shape), b], 2)   # noqa: E731
    return attn(q, both(pk, k), both(pv, v), ok, eps, codes)
