"""Host-side checks of the operators on caches: symbols, refusals before anything is launched, and the 64-bit reference (no GPU)."""
import ctypes
import math
import os
import re

import pytest
import torch

import paper_2605_08123_amd as ska
from paper_2605_08123_amd import binding, cache, layer

from . import cache_ref as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = ctypes.c_void_p(1 << 20)   # never dereferenced
ODD = ctypes.c_void_p((1 << 20) + 8)
OFF = ctypes.c_void_p((1 << 20) + 2)
EINVAL, EUNSUPPORTED, EWORKSPACE = binding.SKA_EINVAL, binding.SKA_EUNSUPPORTED, binding.SKA_EWORKSPACE
F32, BF16, E4M3, INT8 = 0, 1, 2, 3


def by(s):
    return None if s is None else ctypes.byref((layer.Strides if len(s) == 3 else cache.ScaleStrides)(*s))


def test_library_exports_every_declared_symbol():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "sinkhorn_attn_cache.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(ska_\w+)\s*\(", text)))
    assert names == ["ska_cache_attn_fwd", "ska_cache_attn_workspace_bytes", "ska_cache_read", "ska_cache_write", "ska_prefix_attn_fwd",
                     "ska_prefix_attn_workspace_bytes"]
    for n in names:
        args = re.search(rf"\b{n}\s*\((.*?)\)", text, re.S).group(1).count(",") + 1
        assert len(getattr(cache._lib(), n).argtypes) == args, n


def test_write_and_read_refusals():
    lib = cache._lib()

    def call(k=P, v=P, kc=P, ksc=P, vc=P, vsc=P, ks=None, kcs=None, kss=None, B=1, Hk=2, L=8, Lc=64, d=64, dt=BF16, store=E4M3):
        return (lib.ska_cache_write(k, by(ks), v, None, kc, by(kcs), ksc, by(kss), vc, None, vsc, None, None, None, B, Hk, L, Lc, d, dt, store, None),
                lib.ska_cache_read(kc, by(kcs), ksc, by(kss), vc, None, vsc, None, k, by(ks), v, None, None, None, B, Hk, L, Lc, d, dt, store, None))
    for bad in (dict(k=None), dict(v=None), dict(kc=None), dict(ksc=None), dict(vc=None), dict(vsc=None), dict(B=0), dict(Hk=0), dict(L=-1), dict(Lc=0),
                dict(ks=(1024, -64, 64)), dict(kcs=(1024, -64, 64)), dict(kss=(-1, 64))):
        assert call(**bad) == (EINVAL, EINVAL), bad
    for bad in (dict(d=48), dict(d=256), dict(dt=2), dict(store=F32), dict(store=4), dict(L=(1 << 24) + 1), dict(Lc=(1 << 24) + 1), dict(B=65536),
                dict(k=ODD), dict(ks=(1024, 512, 68)), dict(kc=ctypes.c_void_p((1 << 20) + 4)), dict(kcs=(8192, 4096, 66)), dict(ksc=OFF),
                dict(kcs=(1 << 40, 1 << 36, 1 << 27))):
        assert call(**bad) == (EUNSUPPORTED, EUNSUPPORTED), bad
    # a dimension that is not stepped over in what is written, and may be in what is read
    assert call(kcs=(8192, 0, 64))[0] == call(kcs=(8192, 4096, 0))[0] == call(kss=(128, 0))[0] == EINVAL
    assert call(ks=(1024, 0, 64))[1] == EINVAL
    assert call(L=0, k=None, v=None) == (0, 0)


def _attn(lib, prefix, q=P, k=P, v=P, ksc=P, vsc=P, pk=P, psc=P, o=P, lse=P, qs=None, os_=None, ks=None, kss=None, pks=None, B=1, Hq=4, Hk=2, Lq=4, Lp=64, Lk=64,
          d=64, W=8, eps=1.0, dt=BF16, store=E4M3, ws=P, n=1 << 40):
    own = (k, by(ks), ksc, by(kss), v, None, vsc, None)
    if not prefix:
        return lib.ska_cache_attn_fwd(q, by(qs), *own, o, by(os_), lse, None, None, None, None, None, B, Hq, Hk, Lq, Lk, d, W, 0, eps, dt, store, ws, n, None)
    return lib.ska_prefix_attn_fwd(q, by(qs), pk, by(pks), psc, None, pk, None, psc, None, *own, o, by(os_), lse, None, None, None, None, None, None, None, B, Hq,
                                   Hk, Lq, Lp, Lk, d, W, 0, eps, dt, store, ws, n, None)


def test_attention_refusals():
    lib = cache._lib()
    for prefix in (False, True):
        f = lambda **kw: _attn(lib, prefix, **kw)   # noqa: E731
        for bad in (dict(q=None), dict(k=None), dict(v=None), dict(ksc=None), dict(vsc=None), dict(o=None), dict(lse=None), dict(B=0), dict(Hq=0), dict(Hk=0),
                    dict(Hq=3), dict(Lq=0), dict(Lk=0), dict(W=-1), dict(eps=0.0), dict(eps=-1.0), dict(eps=math.nan), dict(eps=math.inf),
                    dict(qs=(1024, -64, 64)), dict(ks=(-16, 64, 64)), dict(kss=(64, -64)), dict(os_=(1024, 0, 64)), dict(ws=ctypes.c_void_p((1 << 20) + 4))):
            assert f(**bad) == EINVAL, (prefix, bad)
        for bad in (dict(d=48), dict(d=256), dict(dt=2), dict(store=4), dict(store=F32, dt=BF16), dict(store=BF16, dt=F32), dict(Lq=(1 << 24) + 1),
                    dict(Lk=(1 << 24) + 1), dict(B=32768), dict(q=ODD), dict(k=ODD), dict(o=ODD), dict(ksc=OFF), dict(qs=(1024, 256, 60)),
                    dict(ks=(8192, 4096, 72)), dict(Lq=1 << 24, Hq=32), dict(eps=1e38), dict(eps=1e-45)):
            assert f(**bad) == EUNSUPPORTED, (prefix, bad)
    f = lambda **kw: _attn(lib, True, **kw)   # noqa: E731
    for bad in (dict(pk=None), dict(psc=None), dict(Lp=0), dict(store=BF16), dict(store=F32, dt=F32), dict(pks=(0, -64, 64))):   # (scales without codes)
        assert f(**bad) == EINVAL, bad
    for bad in (dict(Lp=(1 << 24) + 1), dict(pk=ODD), dict(B=16384, Hq=64, Lq=4096)):
        assert f(**bad) == EUNSUPPORTED, bad
    # keys and values in the queries' type are for the prefix operator; elsewhere softmax_attn takes them
    for t in (F32, BF16):
        assert _attn(lib, False, dt=t, store=t, ksc=None, vsc=None) == EUNSUPPORTED
    # many keys for few queries: parts, and a workspace
    need = ska.ska_cache_attn_workspace_bytes(1, 4, 2, 1, 65536, 64, 1 << 20, True)
    assert need > 0
    for kw in (dict(ws=None), dict(n=need - 1)):
        assert _attn(lib, False, Lq=1, Lk=65536, W=1 << 20, **kw) == EWORKSPACE
    assert ska.ska_prefix_attn_workspace_bytes(1, 4, 2, 1, 65536, 64, 64, 1 << 20) > 0 and f(Lq=1, Lp=65536, W=1 << 20, ws=None) == EWORKSPACE
    assert ska.ska_cache_attn_workspace_bytes(1, 4, 2, 1, 65536, 48, 8) == 0 and ska.ska_prefix_attn_workspace_bytes(1, 4, 2, 1, 0, 64, 64, 8) == 0


def test_binding_refusals():
    q, k = torch.zeros((1, 4, 2, 64)), torch.zeros((1, 2, 8, 64))
    c = ska.ska_cache_empty(1, 2, 8, 64, device="cpu")
    assert c.K.dtype == torch.float8_e4m3fn and c.V_scale.shape == (1, 2, 8)
    assert ska.ska_cache_empty(1, 2, 8, 64, "int8", device="cpu").V.dtype == torch.int8
    with pytest.raises(ValueError, match="store"):
        ska.ska_cache_empty(1, 2, 8, 64, "int4", device="cpu")
    for call in (lambda: ska.ska_cache_write(c, k, k), lambda: ska.ska_cache_read(c), lambda: ska.ska_cache_attn_fwd(q, c, 4),
                 lambda: ska.ska_prefix_attn_fwd(q, (k[0], k[0]), (k, k), 4)):
        with pytest.raises(ValueError, match="GPU"):
            call()
    with pytest.raises(ValueError, match="expected"):
        ska.ska_cache_attn_fwd(q[0], c, 4)
    assert ska.KVCache(*(x[:, :1] for x in c)).K.shape == (1, 1, 8, 64)


def test_reference_numbers():
    """The e4m3 numbers are those that torch's type has, and the nearest code is torch's rounding."""
    numbers = ref.e4m3_numbers()
    assert torch.equal(torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double(), numbers)
    x = torch.randn(200, 64, generator=torch.Generator().manual_seed(1))
    x[:, 0] = 448.0                                                       # scales of 1
    x[:120, 1:8] = ((numbers[:120] + numbers[1:121]) / 2).float()[:, None]   # borders
    c, s = ref.quantise(x, "e4m3")
    assert (s == 1).all() and torch.equal(c.float(), x.to(torch.float8_e4m3fn).float())
    for a, want in ((448.0, 1.0), (448.1, 2.0), (224.0, 0.5), (225.0, 1.0), (3e38, 2.0 ** 120), (1e-40, 2.0 ** -126), (0.0, 2.0 ** -126)):
        assert ref.quantise(torch.tensor([[a, 0.0]]), "e4m3")[1].item() == want, a


def test_reference_of_a_prefix():
    """A prefix and own keys against the same keys in one cache: positions, band and causal end are the same."""
    g = torch.Generator().manual_seed(3)
    r = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)   # noqa: E731
    q, pk, pv, k, v = r(2, 4, 3, 8), r(2, 5, 8), r(2, 5, 8), r(2, 2, 7, 8), r(2, 2, 7, 8)
    start, len_k = torch.tensor([2, 0]), torch.tensor([5, 3])
    for W, causal in ((100, True), (4, True), (3, False)):
        got = ref.prefix_attn(q.float(), pk, pv, k, v, W, causal, 1.0, start=start, len_k=len_k)
        both = lambda a, b: torch.cat([a[None].expand(2, *a.shape), b], 2)   # noqa: E731
        ok = ref.pairs(2, 3, 12, W, causal, start=start + 5, len_k=len_k + 5)
        want = ref.attn(q.float(), both(pk, k), both(pv, v), ok, 1.0)
        for name in ("O", "LSE"):
            torch.testing.assert_close(got[name][0], want[name][0], rtol=0, atol=0)
