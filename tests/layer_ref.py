"""The layer operators (include/sinkhorn_attn_layer.h) in 64 bits by their definitions, on the CPU, each with a bound on what a
correct implementation may differ by.

The bounds count roundings: half a step of a type relative to what is rounded (`half`), and for fp32 sums of n terms in any
order n half-steps of the sum of magnitudes.  They are worst cases, entry by entry.
"""
import math

import torch

F32 = 2.0 ** -24


def half(dtype):
    return torch.finfo(dtype).eps / 2


# ------------------------------------------------------------------ layer norm
def norm_fwd(x, w, b, r, eps):
    """x, r: storage tensors.  Returns s (storage), and (value, bound) of y, mean, rstd."""
    s = x if r is None else (x.double() + r.double()).to(x.dtype)
    f = s.double()
    D = f.shape[-1]
    mean = f.mean(-1, keepdim=True)
    var = ((f - mean) ** 2).mean(-1, keepdim=True)
    rstd = (var + eps) ** -0.5
    wd = torch.ones(D, dtype=torch.float64) if w is None else w.double()
    bd = torch.zeros(D, dtype=torch.float64) if b is None else b.double()
    h = (f - mean) * rstd
    y = h * wd + bd
    # a sum of D terms, taken over at least 16 running sums (threads of a row, pieces of a thread): D / 16 + 32 additions deep
    n = D / 16 + 32
    e_mean = n * F32 * f.abs().mean(-1, keepdim=True)
    # var: its terms' errors (2 |f - mean| e(f - mean)) and the sum's
    dev = (f - mean).abs()
    e_dev = e_mean + F32 * dev
    e_var = (2 * dev * e_dev + e_dev ** 2).mean(-1, keepdim=True) + (n + 2) * F32 * var
    e_rstd = rstd * (e_var / (2 * (var + eps)) + 4 * F32)
    e_y = half(x.dtype) * y.abs() + wd.abs() * (e_dev * rstd + dev * e_rstd + 3 * F32 * h.abs()) * 1.01 + 2 * F32 * y.abs()
    return s, (y, e_y), (mean[..., 0], e_mean[..., 0] + F32 * mean[..., 0].abs()), (rstd[..., 0], e_rstd[..., 0])


def norm_bwd(dy, s, w, stats, ds, wdtype):
    """(value, bound) of dx, dw, db for the statistics that are given (fp32)."""
    g0, f = dy.double(), s.double()
    D, N = f.shape[-1], f.numel() // f.shape[-1]
    mean, rstd = stats[0].double()[..., None], stats[1].double()[..., None]
    h = (f - mean) * rstd
    wd = torch.ones(D, dtype=torch.float64) if w is None else w.double()
    g = g0 * wd
    m0, m1 = g.mean(-1, keepdim=True), (g * h).mean(-1, keepdim=True)
    dx = rstd * (g - m0 - h * m1)
    n = D / 16 + 32
    e_h = 2 * F32 * h.abs()
    e_g = F32 * g.abs()
    e0 = n * F32 * g.abs().mean(-1, keepdim=True) + e_g.mean(-1, keepdim=True)
    e1 = (n + 4) * F32 * (g * h).abs().mean(-1, keepdim=True)
    e_dx = rstd * (e_g + e0 + h.abs() * e1 + e_h * m1.abs() + 4 * F32 * (g.abs() + m0.abs() + (h * m1).abs())) * 1.01
    if ds is not None:
        dx = dx + ds.double()
    e_dx = e_dx + (half(dy.dtype) + 2 * F32) * dx.abs()
    rows = tuple(range(f.dim() - 1))
    p = g0 * h
    # rows: at most N / 64 + 64 additions deep (a thread's rows one after another, then trees)
    k = N / 64 + 64
    dw, db = p.sum(rows), g0.sum(rows)
    e_dw = (half(wdtype) + F32) * dw.abs() + (k + 4) * F32 * p.abs().sum(rows)
    e_db = (half(wdtype) + F32) * db.abs() + k * F32 * g0.abs().sum(rows)
    return (dx, e_dx), (dw, e_dw), (db, e_db)


# ------------------------------------------------------------------ rotary positions
def rope(x, freq, amplitude, pos, interleaved, back=False):
    """x [B,H,L,d] storage, pos [B,L] integers.  (value, bound)."""
    h = freq.numel()
    f = x.double()
    t = pos.double()[:, None, :, None] * freq * (-1 if back else 1)
    c, s = amplitude * torch.cos(t), amplitude * torch.sin(t)
    out, mag = f.clone(), torch.zeros_like(f)
    i1, i2 = (slice(0, 2 * h, 2), slice(1, 2 * h, 2)) if interleaved else (slice(0, h), slice(h, 2 * h))
    x1, x2 = f[..., i1], f[..., i2]
    out[..., i1], out[..., i2] = x1 * c - x2 * s, x2 * c + x1 * s
    mag[..., i1] = mag[..., i2] = amplitude * (x1.abs() + x2.abs())
    # cosine and sine: the angle's fp32 rounding (pi half-steps), the function's two units, the amplitude's product; the products and the sum
    bound = half(x.dtype) * out.abs() + (math.pi + 4 + 1 + 2 + 1) * F32 * mag
    bound[..., 2 * h:] = 0
    return out, bound


# ------------------------------------------------------------------ softmax attention
def pairs(B, Lq, Lk, W, causal, start=None, len_q=None, len_k=None, mask_q=None, mask_k=None):
    p = torch.arange(Lq)[None, :, None] + (0 if start is None else start[:, None, None].long())
    j = torch.arange(Lk)[None, None]
    ok = ((p - j).abs() <= W).expand(B, Lq, Lk).clone()
    if causal:
        ok &= j <= p
    if len_q is not None:
        ok &= torch.arange(Lq)[None, :, None] < len_q[:, None, None]
    if len_k is not None:
        ok &= j < len_k[:, None, None]
    if mask_q is not None:
        ok &= mask_q.bool()[:, :, None]
    if mask_k is not None:
        ok &= mask_k.bool()[:, None, :]
    return ok


def attn(q, k, v, ok, eps, do=None):
    """Storage tensors; rows that take part in no pair are left out before anything is multiplied.  A dict of (value, bound) of
    O and LSE, with dO also of dQ, dK, dV (for a backward that is given O rounded to the storage type and LSE to fp32)."""
    dt = q.dtype
    B, Hq, Lq, d = q.shape
    Hk, Lk = k.shape[1], k.shape[2]
    G = Hq // Hk
    row, key = ok.any(2), ok.any(1)
    clean = lambda x, on: torch.where(on[:, None, :, None], x.double(), 0.0)   # noqa: E731
    qd, kd, vd = clean(q, row), clean(k, key).repeat_interleave(G, 1), clean(v, key).repeat_interleave(G, 1)
    c = 1 / (eps * math.sqrt(d))
    s = qd @ kd.transpose(-1, -2) * c
    okh = ok[:, None].expand(B, Hq, Lq, Lk)
    s = torch.where(okh, s, -math.inf)
    top = s.amax(-1, keepdim=True)
    top0 = torch.where(top > -math.inf, top, 0.0)
    e = torch.exp(s - top0)
    total = e.sum(-1, keepdim=True)
    some = total > 0
    p = e / torch.where(some, total, 1.0)
    lse = (top + total.log())[..., 0]
    o = p @ vd
    # scores: d products and sums, scaled; exponent: one rounding of score and maximum in units of 2, the exponential two units
    n = ok.sum(2).double()[:, None, :, None]
    mag = (qd.abs() @ kd.abs().transpose(-1, -2)) * c
    e_s = (d + 4) * F32 * mag
    e_exp = e_s + 4 * F32 * (torch.where(okh, s, 0.0).abs() + top0.abs()) + 4 * F32
    worst = torch.where(okh, e_exp, 0.0).amax(-1, keepdim=True)
    # P unnormalised in the storage type's precision for the second product, sums of n terms in fp32
    e_o = (p @ vd.abs()) * (half(dt) * (dt != torch.float32) + 2 * worst + 3 * n * F32 + 8 * F32) * 1.02 + half(dt) * o.abs()
    e_lse = (worst + n * F32)[..., 0] + 4 * F32 * (lse.abs().nan_to_num(posinf=0.0) + top0[..., 0].abs()) + 4 * F32
    out = {"O": (o, e_o), "LSE": (lse, e_lse)}
    if do is None:
        return out
    g = clean(do, row)
    z = g @ vd.transpose(-1, -2)
    delta = (g * o).sum(-1, keepdim=True)
    ds = p * (z - delta)
    r2 = half(dt) * (dt != torch.float32)   # roundings of P and dS to the storage type
    # P of the backward from an LSE rounded to fp32
    e_p = p * (e_s + 6 * F32 * (torch.where(okh, s, 0.0).abs() + torch.where(some, lse[..., None], 0.0).abs()) + 4 * F32) * 1.02
    e_z = (d + 2) * F32 * (g.abs() @ vd.abs().transpose(-1, -2))
    e_delta = (half(dt) + (d + 2) * F32) * (g.abs() * o.abs()).sum(-1, keepdim=True)
    e_ds = e_p * (z - delta).abs() + p * (e_z + e_delta + 2 * F32 * (z.abs() + delta.abs())) * 1.02 + r2 * ds.abs() + 2 * F32 * ds.abs()
    fold = lambda x: x.view(B, Hk, G, Lk, d).sum(2)   # noqa: E731
    t = lambda x: x.transpose(-1, -2)                 # noqa: E731
    cols = okh.sum(2).double().view(B, Hk, G, Lk).sum(2)[..., None]
    dq, dk, dv = ds @ kd * c, fold(t(ds) @ qd) * c, fold(t(p) @ g)
    e_dq = (e_ds @ kd.abs() + (n + 3) * F32 * (ds.abs() @ kd.abs())) * c * 1.02 + half(dt) * dq.abs()
    e_dk = (fold(t(e_ds) @ qd.abs()) + (cols + 3) * F32 * fold(t(ds).abs() @ qd.abs())) * c * 1.02 + half(dt) * dk.abs()
    e_dv = (fold(t(e_p + r2 * p) @ g.abs()) + (cols + 3) * F32 * fold(t(p) @ g.abs())) * 1.02 + half(dt) * dv.abs()
    out.update(dQ=(dq, e_dq), dK=(dk, e_dk), dV=(dv, e_dv))
    return out


def check(name, got, ref, floor=1e-30):
    """Entry by entry within the bound; equal where the reference is infinite."""
    value, bound = ref
    got = got.double().cpu()
    assert got.shape == value.shape, (name, got.shape, value.shape)
    inf = torch.isinf(value)
    assert torch.equal(got[inf], value[inf]), name
    off = torch.where(inf, 0.0, (got - torch.where(inf, 0.0, value)).abs())
    over = ~(off <= torch.where(inf, 0.0, bound) + floor)
    if over.any():
        at = tuple(over.nonzero()[0].tolist())
        raise AssertionError(f"{name}: {int(over.sum())} of {over.numel()} entries off, first at {at}: {got[at]} for {value[at]}, bound {bound[at]}")
