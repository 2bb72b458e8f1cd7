"""Thin Python binding of the C ABI in include/sinkhorn_attn_cache.h: caches in 8 bits and softmax attention on caches and shared
prefixes.  Argument marshalling only, as in `layer`.
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple

import torch

from .binding import load
from .layer import (_code, _done, _f, _heads, _here, _i, _int32, _ll, _plain, _raw_stream, _sz, _vp, _workspace, _wrong)

SKA_E4M3, SKA_INT8 = 2, 3
CACHE_STORES = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}
_STORES = {torch.float8_e4m3fn: SKA_E4M3, torch.int8: SKA_INT8}


class KVCache(NamedTuple):
    """Codes [B,Hk,L,d] (float8_e4m3fn or int8) and float32 scales [B,Hk,L] of keys and values.  Views are fine: of some items,
    heads or places (`KVCache(*(x[:2] for x in cache))`)."""
    K: torch.Tensor
    V: torch.Tensor
    K_scale: torch.Tensor
    V_scale: torch.Tensor


class ScaleStrides(ctypes.Structure):
    """Floats between items and heads (ska_scale_strides)."""
    _fields_ = [("b", _ll), ("h", _ll)]


_bound = None


def _lib():
    global _bound
    if _bound is None:
        lib = load()
        lib.ska_cache_write.restype = lib.ska_cache_read.restype = _i
        lib.ska_cache_write.argtypes = lib.ska_cache_read.argtypes = [_vp] * 14 + [_i] * 7 + [_vp]
        lib.ska_cache_attn_workspace_bytes.restype = lib.ska_prefix_attn_workspace_bytes.restype = _sz
        lib.ska_cache_attn_workspace_bytes.argtypes = [_i] * 10
        lib.ska_prefix_attn_workspace_bytes.argtypes = [_i] * 11
        lib.ska_cache_attn_fwd.restype = lib.ska_prefix_attn_fwd.restype = _i
        lib.ska_cache_attn_fwd.argtypes = [_vp] * 18 + [_i] * 8 + [_f, _i, _i, _vp, _sz, _vp]
        lib.ska_prefix_attn_fwd.argtypes = [_vp] * 28 + [_i] * 9 + [_f, _i, _i, _vp, _sz, _vp]
        _bound = lib
    return _bound


def _scales(x, shape, dev, name):
    """Pointer and strides of [B,Hk,L] scales (no strides: contiguous)."""
    if x.get_device() != dev or x.shape != shape or x.dtype is not torch.float32:
        _wrong(x, shape, torch.float32, dev, name)
    if x.is_contiguous():
        return x.data_ptr(), None
    b, h, l = x.stride()
    if l != 1 and shape[2] > 1:
        raise ValueError(f"{name}: the scales of a head's tokens must lie next to each other")
    return x.data_ptr(), ctypes.byref(ScaleStrides(b, h))


def _store(x, name):
    c = _STORES.get(x.dtype)
    if c is None:
        raise TypeError(f"{name}: codes are float8_e4m3fn or int8, got {x.dtype}")
    return c


def _kept(kept, shape, dev, name):
    """The eight pointers of keys and values that are kept as codes (shape: [B,Hk,L,d])."""
    K, V, Ks, Vs = kept
    if K.is_contiguous() and V.is_contiguous() and Ks.is_contiguous() and Vs.is_contiguous() and \
            K.get_device() == V.get_device() == Ks.get_device() == Vs.get_device() == dev and K.dtype is V.dtype and \
            Ks.dtype is Vs.dtype is torch.float32 and K.shape == V.shape == shape and Ks.shape == Vs.shape == shape[:3]:
        return K.data_ptr(), None, Ks.data_ptr(), None, V.data_ptr(), None, Vs.data_ptr(), None
    kp, ks = _heads(K, shape, K.dtype, dev, f"{name}.K")
    vp, vs = _heads(V, shape, K.dtype, dev, f"{name}.V")
    ksp, kss = _scales(Ks, shape[:3], dev, f"{name}.K_scale")
    vsp, vss = _scales(Vs, shape[:3], dev, f"{name}.V_scale")
    return kp, ks, ksp, kss, vp, vs, vsp, vss


def ska_cache_empty(B, Hk, L, d, store="e4m3", device=None) -> KVCache:
    """A cache for L tokens of B items, of codes "e4m3" or "int8" (sinkhorn_attn_cache.h), its places not written."""
    if store not in CACHE_STORES:
        raise ValueError(f"store: one of {sorted(CACHE_STORES)}, got {store!r}")
    device = torch.device("cuda") if device is None else device
    codes = [torch.empty((B, Hk, L, d), dtype=CACHE_STORES[store], device=device) for _ in range(2)]
    return KVCache(*codes, *(torch.empty((B, Hk, L), dtype=torch.float32, device=device) for _ in range(2)))


def _queries(Q, qshape, dev):
    """_heads of a tensor that is checked against nothing but its own shape."""
    return (Q.data_ptr(), None) if Q.is_contiguous() else _heads(Q, qshape, Q.dtype, dev, "Q")


def _four(x, name):
    if x.dim() != 4:
        raise ValueError(f"{name}: expected [B, H, L, d], got {tuple(x.shape)}")
    return x.shape


def ska_cache_write(cache, K, V, start=None, len_new=None):
    """Quantises K, V [B,Hk,L,d] into the cache: token l of item b goes to place start[b] + l, for l < len_new[b] (int32 CUDA tensors
    [B]; 0, L).  Other places are left as they were; tokens without a place are not written.  Returns the cache."""
    B, Hk, Lc, d = _four(cache[0], "cache.K")
    dev, L, dt = _here(K, "K"), _four(K, "K")[2], K.dtype
    shape, store = (B, Hk, L, d), _store(cache[0], "cache.K")
    kp, ks = _heads(K, shape, dt, dev, "K")
    vp, vs = _heads(V, shape, dt, dev, "V")
    _done(_lib().ska_cache_write(kp, ks, vp, vs, *_kept(cache, (B, Hk, Lc, d), dev, "cache"), _plain(start, (B,), torch.int32, dev, "start"),
                                 _plain(len_new, (B,), torch.int32, dev, "len_new"), B, Hk, L, Lc, d, _code(K), store, _raw_stream(dev)))
    return cache


def ska_cache_read(cache, L=None, start=None, len_k=None, dtype=torch.bfloat16, K=None, V=None):
    """The values that L places from start[b] on (all of them; 0) stand for, zeros where a place is not below len_k[b] (int32 CUDA tensors
    [B]).  Returns (K, V) [B,Hk,L,d] of `dtype`, contiguous unless given."""
    B, Hk, Lc, d = _four(cache[0], "cache.K")
    dev, store = _here(cache[0], "cache.K"), _store(cache[0], "cache.K")
    if L is None:
        L = _four(K, "K")[2] if K is not None else _four(V, "V")[2] if V is not None else Lc
    shape = (B, Hk, L, d)
    if K is None and V is None:
        K = cache[2].new_empty(shape, dtype=dtype)
        V = torch.empty_like(K)
        kp, ks, vp, vs = K.data_ptr(), None, V.data_ptr(), None
    else:
        if K is None:
            K = V.new_empty(shape)
        if V is None:
            V = K.new_empty(shape)
        kp, ks = _heads(K, shape, K.dtype, dev, "K")
        vp, vs = _heads(V, shape, K.dtype, dev, "V")
    _done(_lib().ska_cache_read(*_kept(cache, (B, Hk, Lc, d), dev, "cache"), kp, ks, vp, vs, _plain(start, (B,), torch.int32, dev, "start"),
                                _plain(len_k, (B,), torch.int32, dev, "len_k"), B, Hk, L, Lc, d, _code(K), store, _raw_stream(dev)))
    return K, V


# Workspaces by sizes: asking the library costs as much as a check of two tensors
_needs = {}


def _need(f, *sizes):
    n = _needs.get((f, sizes))
    if n is None:
        if len(_needs) > 4096:
            _needs.clear()
        n = _needs[f, sizes] = getattr(_lib(), f)(*sizes)
    return n


def ska_cache_attn_workspace_bytes(B, Hq, Hk, Lq, Lc, d, W, causal=False, dtype=1, store=SKA_E4M3) -> int:
    return int(_lib().ska_cache_attn_workspace_bytes(B, Hq, Hk, Lq, Lc, d, _int32(W), int(bool(causal)), dtype, store))


def ska_cache_attn_fwd(Q, cache, W, causal=False, eps=1.0, start_q=None, len_q=None, len_k=None, mask_q=None, mask_k=None, O=None,
                       LSE=None, workspace=None):
    """ska_softmax_attn_fwd of Q [B,Hq,Lq,d] (float32 or bfloat16) on a cache in 8 bits (KVCache, or its four tensors).  Returns (O, LSE)."""
    qshape, kshape = _four(Q, "Q"), _four(cache[0], "cache.K")
    B, Hq, Lq, d = qshape
    _, Hk, Lc, _ = kshape
    dev, dt, code, store = _here(Q, "Q"), Q.dtype, _code(Q), _store(cache[0], "cache.K")
    qp, qs = _queries(Q, qshape, dev)
    if O is None:
        O = torch.empty_like(Q) if qs is None else Q.new_empty(qshape)
        op, os = O.data_ptr(), None
    else:
        op, os = _heads(O, qshape, dt, dev, "O")
    if LSE is None:
        LSE = Q.new_empty((B, Hq, Lq), dtype=torch.float32)
        lp = LSE.data_ptr()
    else:
        lp = _plain(LSE, (B, Hq, Lq), torch.float32, dev, "LSE")
    W, causal, i32, u8 = _int32(W), 1 if causal else 0, torch.int32, torch.uint8
    ws, n, keep = _workspace(workspace, _need("ska_cache_attn_workspace_bytes", B, Hq, Hk, Lq, Lc, d, W, causal, code, store), Q, dev)
    _done(_lib().ska_cache_attn_fwd(
        qp, qs, *_kept(cache, (B, Hk, Lc, d), dev, "cache"), op, os, lp,
        _plain(start_q, (B,), i32, dev, "start_q"), _plain(len_q, (B,), i32, dev, "len_q"), _plain(len_k, (B,), i32, dev, "len_k"),
        _plain(mask_q, (B, Lq), u8, dev, "mask_q"), _plain(mask_k, (B, Lc), u8, dev, "mask_k"), B, Hq, Hk, Lq, Lc, d, W, causal, eps, code, store,
        ws, n, _raw_stream(dev)))
    return O, LSE


def ska_prefix_attn_workspace_bytes(B, Hq, Hk, Lq, Lp, Lk, d, W, causal=False, dtype=1, store=SKA_E4M3) -> int:
    return int(_lib().ska_prefix_attn_workspace_bytes(B, Hq, Hk, Lq, Lp, Lk, d, _int32(W), int(bool(causal)), dtype, store))


def _side(kept, shape, Q, dev, name):
    """The eight pointers of one side, and its storage type: keys and values in the queries' type, or a cache in 8 bits."""
    if len(kept) == 2:
        kp, ks = _heads(kept[0], shape, Q.dtype, dev, f"{name}.K")
        vp, vs = _heads(kept[1], shape, Q.dtype, dev, f"{name}.V")
        return (kp, ks, None, None, vp, vs, None, None), _code(Q)
    if len(kept) != 4:
        raise ValueError(f"{name}: expected (K, V) or a KVCache, got {len(kept)} tensors")
    return _kept(kept, shape, dev, name), _store(kept[0], f"{name}.K")


def _shared(kept, Hk, Lp, d, Q, dev):
    """_side of the prefix, whose tensors have no first dimension."""
    shape, dt = (Hk, Lp, d), Q.dtype
    if len(kept) == 2:
        K, V = kept
        if K.is_contiguous() and V.is_contiguous() and K.get_device() == V.get_device() == dev and K.dtype is V.dtype is dt and K.shape == V.shape == shape:
            return (K.data_ptr(), None, None, None, V.data_ptr(), None, None, None), _code(Q)
    elif len(kept) == 4:
        K, V, Ks, Vs = kept
        if K.is_contiguous() and V.is_contiguous() and Ks.is_contiguous() and Vs.is_contiguous() and \
                K.get_device() == V.get_device() == Ks.get_device() == Vs.get_device() == dev and K.dtype is V.dtype and \
                Ks.dtype is Vs.dtype is torch.float32 and K.shape == V.shape == shape and Ks.shape == Vs.shape == (Hk, Lp):
            return (K.data_ptr(), None, Ks.data_ptr(), None, V.data_ptr(), None, Vs.data_ptr(), None), _store(K, "prefix.K")
    return _side([x.unsqueeze(0) for x in kept], (1, Hk, Lp, d), Q, dev, "prefix")


def ska_prefix_attn_fwd(Q, prefix, own, W, causal=True, eps=1.0, len_p=None, start_q=None, len_q=None, len_k=None, mask_q=None, mask_k=None,
                        mask_p=None, O=None, LSE=None, workspace=None):
    """Softmax attention of Q [B,Hq,Lq,d] on a prefix that all items share, [Hk,Lp,d], and on each item's own keys behind it,
    [B,Hk,Lk,d]: each (K, V) in Q's type, or both a KVCache (the prefix's without the first dimension).  The prefix is at positions
    0 ... P - 1, an item's key j at P + j, its query i at P + start_q + i; P is len_p (int32 CUDA tensor [1]) or Lp.  The band and the other
    arguments as in ska_softmax_attn_fwd; mask_p: uint8 [Lp].  Returns (O, LSE)."""
    qshape, kshape = _four(Q, "Q"), _four(own[0], "own.K")
    B, Hq, Lq, d = qshape
    _, Hk, Lk, _ = kshape
    dev, dt, code = _here(Q, "Q"), Q.dtype, _code(Q)
    if prefix[0].dim() != 3:
        raise ValueError(f"prefix.K: expected [Hk, Lp, d], got {tuple(prefix[0].shape)}")
    Lp = prefix[0].shape[1]
    before, store = _shared(prefix, Hk, Lp, d, Q, dev)
    behind, other = _side(own, (B, Hk, Lk, d), Q, dev, "own")
    if store != other or len(prefix) != len(own):
        raise ValueError("prefix and own: expected the same kind of storage")
    qp, qs = _queries(Q, qshape, dev)
    if O is None:
        O = torch.empty_like(Q) if qs is None else Q.new_empty(qshape)
        op, os = O.data_ptr(), None
    else:
        op, os = _heads(O, qshape, dt, dev, "O")
    if LSE is None:
        LSE = Q.new_empty((B, Hq, Lq), dtype=torch.float32)
        lp = LSE.data_ptr()
    else:
        lp = _plain(LSE, (B, Hq, Lq), torch.float32, dev, "LSE")
    W, causal, i32, u8 = _int32(W), 1 if causal else 0, torch.int32, torch.uint8
    ws, n, keep = _workspace(workspace, _need("ska_prefix_attn_workspace_bytes", B, Hq, Hk, Lq, Lp, Lk, d, W, causal, code, store), Q, dev)
    _done(_lib().ska_prefix_attn_fwd(
        qp, qs, *before, *behind, op, os, lp, _plain(len_p, (1,), i32, dev, "len_p"),
        _plain(start_q, (B,), i32, dev, "start_q"), _plain(len_q, (B,), i32, dev, "len_q"), _plain(len_k, (B,), i32, dev, "len_k"),
        _plain(mask_q, (B, Lq), u8, dev, "mask_q"), _plain(mask_k, (B, Lk), u8, dev, "mask_k"), _plain(mask_p, (Lp,), u8, dev, "mask_p"),
        B, Hq, Hk, Lq, Lp, Lk, d, W, causal, eps, code, store, ws, n, _raw_stream(dev)))
    return O, LSE
