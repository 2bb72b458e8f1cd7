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


# (A call of a microsecond's work is bound by what follows here: sizes are compared as they are, contiguous tensors pass no
# strides, and the device and its stream are asked for once.)
_device = torch.cuda.current_device


def _raw_stream(dev):
    # (looked for when a call needs it: not every build of torch has it, and host-side calls need none)
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return torch.cuda.current_stream(dev).cuda_stream if raw is None else raw(dev)


def _int32(x) -> int:
    """The nearest 32-bit integer: ctypes keeps the lower bits of what does not fit, and W = 2**32 would be 0."""
    x = int(x)
    return x if -0x80000000 <= x <= 0x7fffffff else 0x7fffffff if x > 0 else -0x80000000


def _here(x: torch.Tensor, name: str) -> int:
    """The current device's number, which x must live on."""
    if not x.is_cuda:
        raise ValueError(f"{name} must live on the GPU")
    dev = _device()
    if x.get_device() != dev:
        raise ValueError(f"{name} lives on {x.device}, the current device is cuda:{dev}")
    return dev


def _wrong(x, shape, dtype, dev, name, contiguous=""):
    if not x.is_cuda:
        raise ValueError(f"{name} must live on the GPU")
    if x.get_device() != dev:
        raise ValueError(f"{name} lives on {x.device}, the other tensors on cuda:{dev}")
    raise ValueError(f"{name}: expected {contiguous}{tuple(shape)} {dtype}, got {tuple(x.shape)} {x.dtype}")


def _plain(x, shape, dtype, dev, name):
    """Pointer of an optional contiguous tensor."""
    if x is None:
        return None
    if x.get_device() != dev or x.shape != shape or x.dtype != dtype or not x.is_contiguous():
        _wrong(x, shape, dtype, dev, name, "contiguous ")
    return x.data_ptr()


def _heads(x, shape, dtype, dev, name):
    """Pointer and strides of a [B, H, L, d] tensor (no strides: contiguous)."""
    if x.get_device() != dev or x.shape != shape or x.dtype != dtype:
        _wrong(x, shape, dtype, dev, name)
    if x.is_contiguous():
        return x.data_ptr(), None
    b, h, l, f = x.stride()
    if f != 1 and shape[3] > 1:
        raise ValueError(f"{name}: the features of a token must lie next to each other")
    return x.data_ptr(), ctypes.byref(Strides(b, h, l))   # (the reference keeps it alive)


def _like(x):
    """A contiguous tensor of x's shape and type."""
    return torch.empty_like(x) if x.is_contiguous() else x.new_empty(x.shape)


def _done(rc):
    if rc != SKA_OK:
        raise SinkhornAttnError(rc)


def _workspace(given, need, like, dev):
    """Pointer and bytes of the caller's workspace or of one of this call, and what keeps it alive until the launch."""
    if given is not None:
        if given.get_device() != dev or not given.is_contiguous():
            raise ValueError("workspace: expected a contiguous tensor on the current device")
        return given.data_ptr(), given.numel() * given.element_size(), given
    if not need:
        return None, 0, None
    w = like.new_empty(need, dtype=torch.uint8)
    return w.data_ptr(), need, w


# ------------------------------------------------------------------ layer norm
def _rows(x, shape, dtype, dev, name):
    """Pointer and row distance of a tensor whose leading dimensions are evenly spaced rows."""
    if x.get_device() != dev or x.shape != shape or x.dtype != dtype:
        _wrong(x, shape, dtype, dev, name)
    if x.is_contiguous():
        return x.data_ptr(), shape[-1]
    stride = x.stride()
    if stride[-1] != 1 and shape[-1] > 1:
        raise ValueError(f"{name}: the features of a row must lie next to each other")
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


def _features(x, name):
    if x.dim() < 1 or x.shape[-1] < 1:
        raise ValueError(f"{name}: needs features in its last dimension")
    return x.shape[-1]


def ska_layer_norm_fwd(X, weight=None, bias=None, residual=None, eps=1e-5, Y=None, S=None, stats=None):
    """Layer norm over the last dimension of X, or of X + residual.  weight, bias: [D], of X's type or float32.
    Returns (Y, S, stats): S the sum (X itself without a residual), stats [2, rows...] float32, as the backward takes them."""
    dev, shape, dt, D = _here(X, "X"), X.shape, X.dtype, _features(X, "X")
    xp, ldx = _rows(X, shape, dt, dev, "X")
    w = weight if weight is not None else bias
    wp = bp = None
    if w is not None:
        wp, bp = _plain(weight, (D,), w.dtype, dev, "weight"), _plain(bias, (D,), w.dtype, dev, "bias")
    if Y is None:
        Y = _like(X)
    yp, ldy = _rows(Y, shape, dt, dev, "Y")
    rp = sp = None
    ldr = lds = 0
    if residual is not None:
        rp, ldr = _rows(residual, shape, dt, dev, "residual")
        if S is None:
            S = _like(X)
        sp, lds = _rows(S, shape, dt, dev, "S")
    elif S is not None:
        raise ValueError("S is the sum with a residual: there is none")
    else:
        S = X
    sshape = (2,) + shape[:-1]
    if stats is None:
        stats = X.new_empty(sshape, dtype=torch.float32)
    _done(_lib().ska_layer_norm_fwd(xp, ldx, rp, ldr, wp, bp, sp, lds, yp, ldy, _plain(stats, sshape, torch.float32, dev, "stats"),
                                    X.numel() // D, D, eps, _code(X), SKA_F32 if w is None else _code(w), _raw_stream(dev)))
    return Y, S, stats


def ska_layer_norm_workspace_bytes(N, D) -> int:
    return int(_lib().ska_layer_norm_workspace_bytes(N, D))


def ska_layer_norm_bwd(dY, S, weight, stats, dS=None, want_weight=True, want_bias=True, dX=None, dweight=None, dbias=None,
                       workspace=None):
    """Gradient of ska_layer_norm_fwd: S, stats as it returned them, dS the gradient that reaches S on the residual's way.
    Returns (dX, dweight, dbias): dX is that of X and of the residual; the others are None where they are not wanted, and of the
    weight's type, without a weight of that of the dweight or dbias given, else float32."""
    dev, shape, dt, D = _here(S, "S"), S.shape, S.dtype, _features(S, "S")
    gp, ldg = _rows(dY, shape, dt, dev, "dY")
    sp, lds = _rows(S, shape, dt, dev, "S")
    N = S.numel() // D
    w = weight if weight is not None else dweight if dweight is not None else dbias
    wt = torch.float32 if w is None else w.dtype
    wp = _plain(weight, (D,), wt, dev, "weight")
    rp, ldr = _rows(dS, shape, dt, dev, "dS") if dS is not None else (None, 0)
    if dX is None:
        dX = _like(S)
    xp, ldx = _rows(dX, shape, dt, dev, "dX")
    if want_weight and dweight is None:
        dweight = S.new_empty(D, dtype=wt) if weight is None else torch.empty_like(weight)
    if want_bias and dbias is None:
        dbias = S.new_empty(D, dtype=wt) if weight is None else torch.empty_like(weight)
    dwp, dbp = _plain(dweight, (D,), wt, dev, "dweight"), _plain(dbias, (D,), wt, dev, "dbias")
    lib = _lib()
    ws, n, keep = _workspace(workspace, lib.ska_layer_norm_workspace_bytes(N, D) if dwp or dbp else 0, S, dev)
    _done(lib.ska_layer_norm_bwd(gp, ldg, sp, lds, wp, _plain(stats, (2,) + shape[:-1], torch.float32, dev, "stats"), rp, ldr, xp, ldx,
                                 dwp, dbp, N, D, _code(S), SKA_F32 if w is None else _code(w), ws, n, _raw_stream(dev)))
    return dX, dweight, dbias


# ------------------------------------------------------------------ rotary positions
def ska_rope_frequencies(rot, base=10000.0, scaling="none", factor=1.0, trained_length=1):
    """(radians per position of each of the rot / 2 pairs, float64 on the host; amplitude).  scaling: "none", "linear",
    "ntk" or "yarn" (sinkhorn_attn_layer.h), for contexts `factor` times as long as trained_length."""
    if scaling not in ROPE_SCALINGS:
        raise ValueError(f"scaling: one of {sorted(ROPE_SCALINGS)}, got {scaling!r}")
    freq = torch.empty(max(int(rot), 0) // 2, dtype=torch.float64)
    amplitude = _d()
    _done(_lib().ska_rope_frequencies(_int32(rot), float(base), ROPE_SCALINGS[scaling], float(factor), _int32(trained_length),
                                      freq.data_ptr() if freq.numel() else None, ctypes.addressof(amplitude)))
    return freq, amplitude.value


def _rope(call, Q, K, freq, amplitude, interleaved, start, positions, Qo, Ko, names):
    if Q.dim() != 4:
        raise ValueError(f"{names[0]}: expected [B, H, L, d], got {tuple(Q.shape)}")
    dev, shape, dt = _here(Q, names[0]), Q.shape, Q.dtype
    B, Hq, L, d = shape
    qp, qs = _heads(Q, shape, dt, dev, names[0])
    if Qo is None:
        Qo = _like(Q)
    op, os = _heads(Qo, shape, dt, dev, names[2])
    kp = kop = ks = kos = None
    Hk = 0
    if K is not None:
        Hk = K.shape[1] if K.dim() == 4 else 0
        kshape = (B, Hk, L, d)
        kp, ks = _heads(K, kshape, dt, dev, names[1])
        if Ko is None:
            Ko = _like(K)
        kop, kos = _heads(Ko, kshape, dt, dev, names[3])
    elif Ko is not None:
        raise ValueError(f"{names[3]} without {names[1]}")
    if freq.dim() != 1:
        raise ValueError(f"freq: expected one dimension, got {tuple(freq.shape)}")
    pairs = freq.shape[0]
    _done(call(qp, qs, op, os, kp, ks, kop, kos, _plain(freq, (pairs,), torch.float64, dev, "freq"), amplitude,
               _plain(start, (B,), torch.int32, dev, "start"), _plain(positions, (B, L), torch.int32, dev, "positions"), B, Hq, Hk, L, d,
               2 * pairs, 1 if interleaved else 0, _code(Q), _raw_stream(dev)))
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
    return int(_lib().ska_softmax_attn_workspace_bytes(int(bool(backward)), B, Hq, Hk, Lq, Lk, d, _int32(W), int(bool(causal)), dtype))


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
    dev, qshape, kshape, dt, code = _here(Q, "Q"), Q.shape, (B, Hk, Lk, d), Q.dtype, _code(Q)
    qp, qs = _heads(Q, qshape, dt, dev, "Q")
    kp, ks = _heads(K, kshape, dt, dev, "K")
    vp, vs = _heads(V, kshape, dt, dev, "V")
    if O is None:
        O = _like(Q)
    op, os = _heads(O, qshape, dt, dev, "O")
    if LSE is None:
        LSE = Q.new_empty((B, Hq, Lq), dtype=torch.float32)
    lib = _lib()
    W, causal, i32, u8 = _int32(W), 1 if causal else 0, torch.int32, torch.uint8
    ws, n, keep = _workspace(workspace, lib.ska_softmax_attn_workspace_bytes(0, B, Hq, Hk, Lq, Lk, d, W, causal, code), Q, dev)
    _done(lib.ska_softmax_attn_fwd(
        qp, qs, kp, ks, vp, vs, op, os, _plain(LSE, (B, Hq, Lq), torch.float32, dev, "LSE"), _plain(start_q, (B,), i32, dev, "start_q"),
        _plain(len_q, (B,), i32, dev, "len_q"), _plain(len_k, (B,), i32, dev, "len_k"), _plain(mask_q, (B, Lq), u8, dev, "mask_q"),
        _plain(mask_k, (B, Lk), u8, dev, "mask_k"), B, Hq, Hk, Lq, Lk, d, W, causal, eps, code, ws, n, _raw_stream(dev)))
    return O, LSE


def ska_softmax_attn_bwd(Q, K, V, O, dO, LSE, W, causal=False, eps=1.0, len_q=None, len_k=None, mask_q=None, mask_k=None,
                         start_q=None, dQ=None, dK=None, dV=None, workspace=None):
    """Gradient of ska_softmax_attn_fwd (O, LSE as it returned them, the same other arguments).  Returns (dQ, dK, dV)."""
    B, Hq, Hk, Lq, Lk, d = _sizes(Q, K)
    dev, qshape, kshape, dt, code = _here(Q, "Q"), Q.shape, (B, Hk, Lk, d), Q.dtype, _code(Q)
    qp, qs = _heads(Q, qshape, dt, dev, "Q")
    kp, ks = _heads(K, kshape, dt, dev, "K")
    vp, vs = _heads(V, kshape, dt, dev, "V")
    op, os = _heads(O, qshape, dt, dev, "O")
    gp, gs = _heads(dO, qshape, dt, dev, "dO")
    if dQ is None:
        dQ = _like(Q)
    if dK is None:
        dK = _like(K)
    if dV is None:
        dV = _like(V)
    dqp, dqs = _heads(dQ, qshape, dt, dev, "dQ")
    dkp, dks = _heads(dK, kshape, dt, dev, "dK")
    dvp, dvs = _heads(dV, kshape, dt, dev, "dV")
    lib = _lib()
    W, causal, i32, u8 = _int32(W), 1 if causal else 0, torch.int32, torch.uint8
    ws, n, keep = _workspace(workspace, lib.ska_softmax_attn_workspace_bytes(1, B, Hq, Hk, Lq, Lk, d, W, causal, code), Q, dev)
    _done(lib.ska_softmax_attn_bwd(
        qp, qs, kp, ks, vp, vs, op, os, gp, gs, _plain(LSE, (B, Hq, Lq), torch.float32, dev, "LSE"), dqp, dqs, dkp, dks, dvp, dvs,
        _plain(start_q, (B,), i32, dev, "start_q"), _plain(len_q, (B,), i32, dev, "len_q"), _plain(len_k, (B,), i32, dev, "len_k"),
        _plain(mask_q, (B, Lq), u8, dev, "mask_q"), _plain(mask_k, (B, Lk), u8, dev, "mask_k"), B, Hq, Hk, Lq, Lk, d, W, causal, eps, code,
        ws, n, _raw_stream(dev)))
    return dQ, dK, dV
