"""The example layer's answers from caches in the storage type behind a prompt that all sequences share."""
import math

import pytest
import torch

import paper_2605_08123_amd as ska

from . import test_gpu_cache_example   # noqa: F401 (the path of the examples)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("W", [17, 1 << 20])
@pytest.mark.parametrize("P", [0, 25])
@pytest.mark.parametrize("n", [1, 3])
def test_tokens_behind_a_plain_prompt(n, P, W):
    """n tokens at a time, the prompt as keys and values in bf16.  Roundings as for caches in 8 bits: a handful of 2^-9."""
    from attention_layer import AttentionLayer
    print("\n[case] example, plain", n, P, W, flush=True)
    layer = AttentionLayer("softmax", 128, 4, 2, 32, W, causal=True, rot=32)
    g = torch.Generator(device="cuda").manual_seed(0)
    B, L = 3, P + 36
    x, r = (torch.randn((B, L, 128), generator=g, device="cuda").bfloat16() for _ in range(2))
    x[:, :P], r[:, :P] = x[:1, :P], r[:1, :P]
    p = layer.params
    Y, _, _ = ska.ska_layer_norm_fwd(x, p["norm"], p["norm_bias"], residual=r)
    Q, K, V = layer._heads(Y @ p["qkv"])
    Q, K = ska.ska_rope_fwd(Q, K, layer.freq, layer.amplitude)
    i = torch.arange(L, device="cuda")
    off = (i[None] > i[:, None]) | (i[None] < i[:, None] - W)
    a = (Q.float() @ K.float().repeat_interleave(2, 1).transpose(-1, -2).contiguous() / math.sqrt(32)).masked_fill(off, -math.inf).softmax(-1)
    want = (a @ V.float().repeat_interleave(2, 1)).transpose(1, 2).reshape(B, L, -1) @ p["out"].float()
    new = lambda b, L: [torch.zeros((b, 2, L, 32), device="cuda", dtype=torch.bfloat16) for _ in range(2)]   # noqa: E731
    prefix, outs = None, []
    if P:
        prompt = new(1, P)
        outs.append(layer.token(x[:1, :P], r[:1, :P], prompt, torch.zeros(1, device="cuda", dtype=torch.int32))[0].expand(B, -1, -1))
        prefix = tuple(y[0] for y in prompt)
    cache, length = new(B, L - P), torch.zeros(B, device="cuda", dtype=torch.int32)
    for t in range(P, L, n):
        outs.append(layer.token(x[:, t:t + n].contiguous(), r[:, t:t + n].contiguous(), cache, length, prefix)[0])
        length = length + n
    got = torch.cat(outs, 1).float()
    off = ((got - want).norm() / want.norm()).item()
    print(off)
    assert off < 6 * 2.0 ** -9


def test_a_prompt_of_another_kind_is_refused():
    from attention_layer import AttentionLayer
    layer = AttentionLayer("softmax", 128, 4, 2, 32, 17, causal=True, rot=32)
    x = torch.zeros((2, 1, 128), device="cuda", dtype=torch.bfloat16)
    length = torch.zeros(2, device="cuda", dtype=torch.int32)
    plain = [torch.full((2, 2, 8, 32), 3.0, device="cuda", dtype=torch.bfloat16) for _ in range(2)]
    codes = ska.ska_cache_empty(2, 2, 8, 32)
    for y in codes:
        y.view(torch.uint8).fill_(3)
    for cache, prefix in ((plain, ska.KVCache(*(y[0] for y in codes))), (codes, tuple(y[0] for y in plain))):
        with pytest.raises(ValueError, match="storage"):
            layer.token(x, x, cache, length, prefix)
    assert all((y == 3).all() for y in plain) and all((y.view(torch.uint8) == 3).all() for y in codes)   # (nothing was appended)
