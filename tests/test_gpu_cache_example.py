"""The example layer's answers from caches in 8 bits and behind a shared prompt."""
import math
import os
import sys

import pytest
import torch

import paper_2605_08123_amd as ska

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))


def whole(layer, x, r, store):
    """All tokens at once in fp32, keys and values as the cache stands for them."""
    p = layer.params
    Y, _, _ = ska.ska_layer_norm_fwd(x, p["norm"], p["norm_bias"], residual=r)
    q, k, v = layer._heads(Y @ p["qkv"])
    Q, K = ska.ska_rope_fwd(q, k, layer.freq, layer.amplitude)
    B, _, L, d = K.shape
    K, V = ska.ska_cache_read(ska.ska_cache_write(ska.ska_cache_empty(B, layer.Hk, L, d, store), K, v), dtype=torch.float32)
    G, i = layer.Hq // layer.Hk, torch.arange(L, device="cuda")
    off = (i[None] > i[:, None]) | (i[None] < i[:, None] - layer.W)
    a = (Q.float() @ K.repeat_interleave(G, 1).transpose(-1, -2).contiguous() / math.sqrt(d)).masked_fill(off, -math.inf).softmax(-1)
    return (a @ V.repeat_interleave(G, 1)).transpose(1, 2).reshape(B, L, -1) @ p["out"].float()


@pytest.mark.parametrize("store", ["e4m3", "int8"])
@pytest.mark.parametrize("W", [17, 1 << 20])
@pytest.mark.parametrize("P", [0, 25])
def test_tokens_against_all_at_once(P, W, store):
    """What differs are roundings to bf16: of attention's result and the output's, and of the projections, whose matrix products sum
    in another order for one token (a step now and then, of about four tensors): a handful of 2^-9."""
    from attention_layer import AttentionLayer
    print("\n[case] example", P, W, store, flush=True)
    layer = AttentionLayer("softmax", 128, 4, 2, 32, W, causal=True, rot=32)
    g = torch.Generator(device="cuda").manual_seed(0)
    B, L = 3, 60
    x, r = (torch.randn((B, L, 128), generator=g, device="cuda").bfloat16() for _ in range(2))
    x[:, :P], r[:, :P] = x[:1, :P], r[:1, :P]
    want = whole(layer, x, r, store)
    prefix, outs = None, []
    if P:
        prompt = ska.ska_cache_empty(1, 2, P, 32, store)
        out, _ = layer.token(x[:1, :P], r[:1, :P], prompt, torch.zeros(1, device="cuda", dtype=torch.int32))
        outs.append(out.expand(B, -1, -1))
        prefix = ska.KVCache(*(y[0] for y in prompt))
    cache, n = ska.ska_cache_empty(B, 2, L - P, 32, store), torch.zeros(B, device="cuda", dtype=torch.int32)
    for t in range(P, L):
        outs.append(layer.token(x[:, t:t + 1], r[:, t:t + 1], cache, n, prefix)[0])
        n = n + 1
    got = torch.cat(outs, 1).float()
    off = ((got - want).norm() / want.norm()).item()
    print(off)
    assert off < 6 * 2.0 ** -9


def test_it_runs(monkeypatch, capsys):
    import attention_layer
    monkeypatch.setattr(sys, "argv", ["attention_layer.py", "--steps", "1"])
    attention_layer.main()
    out = capsys.readouterr().out
    print(out)
    assert out.count("largest difference") == 5
