"""Thin Python binding of the C ABI in include/sinkhorn_attn_layer.h: the operators of an attention layer around the banded
Sinkhorn attention.

Argument marshalling only, as in `binding`: torch supplies device memory and the current HIP stream.  Heads are [B, H, L, d]
tensors of any strides whose features lie next to each other (a projection's [B, L, H, d] transposed is one).
"""
from __future__ import annotations

import ctypes

import torch

from .binding import SKA_BF16, SKA_F32, SKA_OK, SinkhornAttnError, load

ROPE_SCALINGS = {"none": 0, "linear": 1, "ntk": 2, "yarn": 3}

_CODES = {torch.float32: SKA_F32, torch.bfloat16: SKA_BF16}
_vp, _i, _f, _ll, _sz, _d = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_longlong, ctypes.c_size_t, ctypes.c_double


class Strides(ctypes.Structure):
    """Elements between items, heads and tokens (ska_strides)."""
    _fields_ = [("b", _ll), ("h", _ll), ("l", _ll)]


_bound = None


def _lib():
    global _bound
    if _bound is None:
        lib = load()
        lib.ska_layer_norm_fwd.restype = _i
        lib.ska_layer_norm_fwd.argtypes = [_vp, _ll, _vp, _ll, _vp, _vp, _vp, _ll, _vp, _ll, _vp, _ll, _i, _f, _i, _i, _vp]
        lib.ska_layer_norm_workspace_bytes.restype = _sz
        lib.ska_layer_norm_workspace_bytes.argtypes = [_ll, _i]
        lib.ska_layer_norm_bwd.restype = _i
        lib.ska_layer_norm_bwd.argtypes = [_vp, _ll, _vp, _ll, _vp, _vp, _vp, _ll, _vp, _ll, _vp, _vp, _ll, _i, _i, _i, _vp, _sz, _vp]
        lib.ska_rope_frequencies.restype = _i
        lib.ska_rope_frequencies.argtypes = [_i, _d, _i, _d, _i, _vp, _vp]
        for f in (lib.ska_rope_fwd, lib.ska_rope_bwd):
            f.restype = _i
            f.argtypes = [_vp] * 9 + [_f, _vp, _vp] + [_i] * 8 + [_vp]
        lib.ska_softmax_attn_workspace_bytes.restype = _sz
        lib.ska_softmax_attn_workspace_bytes.argtypes = [_i] * 10
        lib.ska_softmax_attn_fwd.restype = _i
        lib.ska_softmax_attn_fwd.argtypes = [_vp] * 14 + [_i] * 8 + [_f, _i, _vp, _sz, _vp]
        lib.ska_softmax_attn_bwd.restype = _i
        lib.ska_softmax_attn_bwd.argtypes = [_vp] * 22 + [_i] * 8 + [_f, _i, _vp, _sz, _vp]
        _bound = lib
    return _bound


def _code(t: torch.Tensor) -> int:
    c = _CODES.get(t.dtype)
    if c is None:
        raise TypeError(f"unsupported dtype {t.dtype}")
    return c


def _on_gpu(x: torch.Tensor, name: str):
    if not x.is_cuda:
        raise ValueError(f"{name} must live on the GPU")
    if x.device.index != torch.cuda.current_device():
        raise ValueError(f"{name} lives on {x.device}, the current device is cuda:{torch.cuda.current_device()}")


def _plain(x, shape, dtype, name):
    """Pointer of an optional contiguous tensor."""
    if x is None:
        return None
    _on_gpu(x, name)
    if tuple(x.shape) != tuple(shape) or x.dtype != dtype or not x.is_contiguous():
        raise ValueError(f"{name}: expected contiguous {tuple(shape)} {dtype}, got {tuple(x.shape)} {x.dtype}")
    return x.data_ptr()


def _heads(x, shape, dtype, name):
    """Pointer and strides of a [B, H, L, d] tensor."""
    _on_gpu(x, name)
    if tuple(x.shape) != tuple(shape) or x.dtype != dtype:
        raise ValueError(f"{name}: expected {tuple(shape)} {dtype}, got {tuple(x.shape)} {x.dtype}")
    b, h, l, f = x.stride()
    if f != 1 and shape[3] > 1:
        raise ValueError(f"{name}: the features of a token must lie next to each other")
    return x.data_ptr(), ctypes.byref(Strides(b, h, l))   # (the reference keeps it alive)


def _stream() -> int:
    return torch.cuda.current_stream().cuda_stream


def _done(rc):
    if rc != SKA_OK:
        raise SinkhornAttnError(rc)


def _workspace(given, need, device):
    if given is not None:
        _on_gpu(given, "workspace")
        return given.data_ptr(), given.numel() * given.element_size(), given
    if not need:
        return None, 0, None
    w = torch.empty(need, device=device, dtype=torch.uint8)
    return w.data_ptr(), need, w


# ------------------------------------------------------------------ layer norm
def _rows(x, like, name):
    """Pointer and row distance of a tensor of `like`'s shape and type whose leading dimensions are evenly spaced rows."""
    _on_gpu(x, name)
    if x.shape != like.shape or x.dtype != like.dtype:
        raise ValueError(f"{name}: expected {tuple(like.shape)} {like.dtype}, got {tuple(x.shape)} {x.dtype}")
    shape, stride = x.shape, x.stride()
    if x.dim() < 1 or shape[-1] < 1:
        raise ValueError(f"{name}: needs features in its last dimension")
    if stride[-1] != 1 and shape[-1] > 1:
        raise ValueError(f"{name}: the features of a row must lie next to each other")
    if x.is_contiguous():
        return x.data_ptr(), shape[-1]
    ld, rows = None, 1   # dimensions from the last row dimension outwards: each steps over the whole of the ones inside it
    for n, s in zip(reversed(shape[:-1]), reversed(stride[:-1])):
        if n == 1:
            continue
        if ld is None:
            ld = s
        elif s != ld * rows:
            raise ValueError(f"{name}: rows must be evenly spaced")
        rows *= n
    return x.data_ptr(), shape[-1] if ld is None else ld


def ska_layer_norm_fwd(X, weight=None, bias=None, residual=None, eps=1e-5, Y=None, S=None, stats=None):
    """Layer norm over the last dimension of X, or of X + residual.  weight, bias: [D], of X's type or float32.
    Returns (Y, S, stats): S the sum (X itself without a residual), stats [2, rows...] float32, as the backward takes them."""
    xp, ldx = _rows(X, X, "X")
    D = X.shape[-1]
    w = weight if weight is not None else bias
    wp = _plain(weight, (D,), w.dtype, "weight") if w is not None else None
    bp = _plain(bias, (D,), w.dtype, "bias") if w is not None else None
    Y = torch.empty(X.shape, device=X.device, dtype=X.dtype) if Y is None else Y
    yp, ldy = _rows(Y, X, "Y")
    rp = sp = None
    ldr = lds = 0
    if residual is not None:
        rp, ldr = _rows(residual, X, "residual")
        S = torch.empty(X.shape, device=X.device, dtype=X.dtype) if S is None else S
        sp, lds = _rows(S, X, "S")
    else:
        if S is not None:
            raise ValueError("S is the sum with a residual: there is none")
        S = X
    shape = (2,) + tuple(X.shape[:-1])
    stats = torch.empty(shape, device=X.device, dtype=torch.float32) if stats is None else stats
    _done(_lib().ska_layer_norm_fwd(xp, ldx, rp, ldr, wp, bp, sp, lds, yp, ldy, _plain(stats, shape, torch.float32, "stats"),
                                    X.numel() // D, D, eps, _code(X), SKA_F32 if w is None else _code(w), _stream()))
    return Y, S, stats


def ska_layer_norm_workspace_bytes(N, D) -> int:
    return int(_lib().ska_layer_norm_workspace_bytes(N, D))


def ska_layer_norm_bwd(dY, S, weight, stats, dS=None, want_weight=True, want_bias=True, dX=None, dweight=None, dbias=None,
                       workspace=None):
    """Gradient of ska_layer_norm_fwd: S, stats as it returned them, dS the gradient that reaches S on the residual's way.
    Returns (dX, dweight, dbias): dX is that of X and of the residual; the others are None where they are not wanted."""
    gp, ldg = _rows(dY, S, "dY")
    sp, lds = _rows(S, S, "S")
    D = S.shape[-1]
    N = S.numel() // D
    wt = torch.float32 if weight is None else weight.dtype
    wp = _plain(weight, (D,), wt, "weight")
    rp, ldr = _rows(dS, S, "dS") if dS is not None else (None, 0)
    dX = torch.empty(S.shape, device=S.device, dtype=S.dtype) if dX is None else dX
    xp, ldx = _rows(dX, S, "dX")
    if want_weight and dweight is None:
        dweight = torch.empty(D, device=S.device, dtype=wt)
    if want_bias and dbias is None:
        dbias = torch.empty(D, device=S.device, dtype=wt)
    dwp, dbp = _plain(dweight, (D,), wt, "dweight"), _plain(dbias, (D,), wt, "dbias")
    lib = _lib()
    ws, n, keep = _workspace(workspace, lib.ska_layer_norm_workspace_bytes(N, D) if dwp or dbp else 0, S.device)
    _done(lib.ska_layer_norm_bwd(gp, ldg, sp, lds, wp, _plain(stats, (2,) + tuple(S.shape[:-1]), torch.float32, "stats"), rp, ldr, xp, ldx,
                                 dwp, dbp, N, D, _code(S), SKA_F32 if weight is None else _code(weight), ws, n, _stream()))
    return dX, dweight, dbias


# ------------------------------------------------------------------ rotary positions
def ska_rope_frequencies(rot, base=10000.0, scaling="none", factor=1.0, trained_length=1):
    """(radians per position of each of the rot / 2 pairs, float64 on the host; amplitude).  scaling: "none", "linear",
    "ntk" or "yarn" (sinkhorn_attn_layer.h), for contexts `factor` times as long as trained_length."""
    if scaling not in ROPE_SCALINGS:
        raise ValueError(f"scaling: one of {sorted(ROPE_SCALINGS)}, got {scaling!r}")
    freq = torch.empty(max(int(rot), 0) // 2, dtype=torch.float64)
    amplitude = _d()
    _done(_lib().ska_rope_frequencies(int(rot), float(base), ROPE_SCALINGS[scaling], float(factor), int(trained_length),
                                      freq.data_ptr() if freq.numel() else None, ctypes.addressof(amplitude)))
    return freq, amplitude.value


def _rope(call, Q, K, freq, amplitude, interleaved, start, positions, Qo, Ko, names):
    if Q.dim() != 4:
        raise ValueError(f"{names[0]}: expected [B, H, L, d], got {tuple(Q.shape)}")
    B, Hq, L, d = Q.shape
    qp, qs = _heads(Q, Q.shape, Q.dtype, names[0])
    Qo = torch.empty(Q.shape, device=Q.device, dtype=Q.dtype) if Qo is None else Qo
    op, os = _heads(Qo, Q.shape, Q.dtype, names[2])
    kp = kop = ks = kos = None
    Hk = 0
    if K is not None:
        Hk = K.shape[1] if K.dim() == 4 else 0
        kp, ks = _heads(K, (B, Hk, L, d), Q.dtype, names[1])
        Ko = torch.empty(K.shape, device=Q.device, dtype=Q.dtype) if Ko is None else Ko
        kop, kos = _heads(Ko, K.shape, Q.dtype, names[3])
    elif Ko is not None:
        raise ValueError(f"{names[3]} without {names[1]}")
    if freq.dim() != 1:
        raise ValueError(f"freq: expected one dimension, got {tuple(freq.shape)}")
    fp = _plain(freq, freq.shape, torch.float64, "freq")
    _done(call(qp, qs, op, os, kp, ks, kop, kos, fp, amplitude, _plain(start, (B,), torch.int32, "start"),
               _plain(positions, (B, L), torch.int32, "positions"), B, Hq, Hk, L, d, 2 * freq.shape[0], int(bool(interleaved)), _code(Q),
               _stream()))
    return Qo, Ko


def ska_rope_fwd(Q, K, freq, amplitude=1.0, interleaved=False, start=None, positions=None, Qr=None, Kr=None):
    """Rotary positions of Q [B,Hq,L,d] and K [B,Hk,L,d] (or None).  freq: float64 CUDA tensor of the turned pairs
    (ska_rope_frequencies).  Token l of item b stands at positions[b][l], start[b] + l, or l (int32 CUDA tensors [B,L], [B]).
    Returns (Qr, Kr), contiguous [B,H,L,d] unless given."""
    return _rope(_lib().ska_rope_fwd, Q, K, freq, amplitude, interleaved, start, positions, Qr, Kr, ("Q", "K", "Qr", "Kr"))


def ska_rope_bwd(dQr, dKr, freq, amplitude=1.0, interleaved=False, start=None, positions=None, dQ=None, dK=None):
    """Gradient of ska_rope_fwd.  Returns (dQ, dK)."""
    return _rope(_lib().ska_rope_bwd, dQr, dKr, freq, amplitude, interleaved, start, positions, dQ, dK, ("dQr", "dKr", "dQ", "dK"))


# ------------------------------------------------------------------ softmax attention on a band
def ska_softmax_attn_workspace_bytes(backward, B, Hq, Hk, Lq, Lk, d, W, causal=False, dtype=SKA_BF16) -> int:
    return int(_lib().ska_softmax_attn_workspace_bytes(int(bool(backward)), B, Hq, Hk, Lq, Lk, d, W, int(bool(causal)), dtype))


def _sizes(Q, K):
    if Q.dim() != 4 or K.dim() != 4:
        raise ValueError(f"Q, K: expected [B, H, L, d], got {tuple(Q.shape)}, {tuple(K.shape)}")
    B, Hq, Lq, d = Q.shape
    return B, Hq, K.shape[1], Lq, K.shape[2], d


def ska_softmax_attn_fwd(Q, K, V, W, causal=False, eps=1.0, len_q=None, len_k=None, mask_q=None, mask_k=None, start_q=None,
                         O=None, LSE=None, workspace=None):
    """Softmax attention of Q [B,Hq,Lq,d] on K, V [B,Hk,Lk,d] over the band |start_q + i - j| <= W (causal: j <= start_q + i
    only), scores / (eps sqrt d).  len_q, len_k, start_q: int32 CUDA tensors [B]; mask_q, mask_k: uint8 [B,Lq], [B,Lk]
    (nonzero = active).  Returns (O, LSE [B,Hq,Lq] float32); a query without a key: 0, -inf."""
    B, Hq, Hk, Lq, Lk, d = _sizes(Q, K)
    dt, code = Q.dtype, _code(Q)
    qp, qs = _heads(Q, Q.shape, dt, "Q")
    kp, ks = _heads(K, (B, Hk, Lk, d), dt, "K")
    vp, vs = _heads(V, (B, Hk, Lk, d), dt, "V")
    O = torch.empty(Q.shape, device=Q.device, dtype=dt) if O is None else O
    op, os = _heads(O, Q.shape, dt, "O")
    LSE = torch.empty((B, Hq, Lq), device=Q.device, dtype=torch.float32) if LSE is None else LSE
    lib = _lib()
    W, causal = int(W), int(bool(causal))
    ws, n, keep = _workspace(workspace, lib.ska_softmax_attn_workspace_bytes(0, B, Hq, Hk, Lq, Lk, d, W, causal, code), Q.device)
    _done(lib.ska_softmax_attn_fwd(
        qp, qs, kp, ks, vp, vs, op, os, _plain(LSE, (B, Hq, Lq), torch.float32, "LSE"), _plain(start_q, (B,), torch.int32, "start_q"),
        _plain(len_q, (B,), torch.int32, "len_q"), _plain(len_k, (B,), torch.int32, "len_k"), _plain(mask_q, (B, Lq), torch.uint8, "mask_q"),
        _plain(mask_k, (B, Lk), torch.uint8, "mask_k"), B, Hq, Hk, Lq, Lk, d, W, causal, eps, code, ws, n, _stream()))
    return O, LSE


def ska_softmax_attn_bwd(Q, K, V, O, dO, LSE, W, causal=False, eps=1.0, len_q=None, len_k=None, mask_q=None, mask_k=None,
                         start_q=None, dQ=None, dK=None, dV=None, workspace=None):
    """Gradient of ska_softmax_attn_fwd (O, LSE as it returned them, the same other arguments).  Returns (dQ, dK, dV)."""
    B, Hq, Hk, Lq, Lk, d = _sizes(Q, K)
    dt, code = Q.dtype, _code(Q)
    kv = (B, Hk, Lk, d)
    ptrs = []
    for name, x, shape in (("Q", Q, Q.shape), ("K", K, kv), ("V", V, kv), ("O", O, Q.shape), ("dO", dO, Q.shape)):
        ptrs += _heads(x, shape, dt, name)
    dQ = torch.empty(Q.shape, device=Q.device, dtype=dt) if dQ is None else dQ
    dK = torch.empty(kv, device=Q.device, dtype=dt) if dK is None else dK
    dV = torch.empty(kv, device=Q.device, dtype=dt) if dV is None else dV
    outs = []
    for name, x, shape in (("dQ", dQ, Q.shape), ("dK", dK, kv), ("dV", dV, kv)):
        outs += _heads(x, shape, dt, name)
    lib = _lib()
    W, causal = int(W), int(bool(causal))
    ws, n, keep = _workspace(workspace, lib.ska_softmax_attn_workspace_bytes(1, B, Hq, Hk, Lq, Lk, d, W, causal, code), Q.device)
    _done(lib.ska_softmax_attn_bwd(
        *ptrs, _plain(LSE, (B, Hq, Lq), torch.float32, "LSE"), *outs, _plain(start_q, (B,), torch.int32, "start_q"),
        _plain(len_q, (B,), torch.int32, "len_q"), _plain(len_k, (B,), torch.int32, "len_k"), _plain(mask_q, (B, Lq), torch.uint8, "mask_q"),
        _plain(mask_k, (B, Lk), torch.uint8, "mask_k"), B, Hq, Hk, Lq, Lk, d, W, causal, eps, code, ws, n, _stream()))
    return dQ, dK, dV
