"""The example layer: its gradients against torch's own of the same layer in fp32, its training, its single tokens."""
import math
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_gradients_of_the_softmax_layer():
    """Relative 2-norms.  The layer rounds about a dozen intermediate tensors to bf16 (2^-8 at worst, about half of that in the
    2-norm), each gradient passing through at most all of them: 12 * 2^-9."""
    from attention_layer import AttentionLayer
    B, L, D, Hq, Hk, d, W = 2, 200, 128, 4, 2, 32, 50
    layer = AttentionLayer("softmax", D, Hq, Hk, d, W, causal=True, rot=16)
    g = torch.Generator(device="cuda").manual_seed(4)
    x, r, dout, dS = (torch.randn((B, L, D), generator=g, device="cuda").bfloat16() for _ in range(4))
    out, S, saved = layer.forward(x, r)
    dx, grads = layer.backward(dout, dS, saved)
    p = {k: v.cpu().float().requires_grad_() for k, v in layer.params.items()}
    s = S.cpu().float().requires_grad_()
    y = torch.nn.functional.layer_norm(s, (D,), p["norm"], p["norm_bias"])
    qkv = (y @ p["qkv"]).view(B, L, Hq + 2 * Hk, d).transpose(1, 2)
    angle = torch.arange(L).double()[:, None] * layer.freq.cpu()
    c, n = angle.cos().float(), angle.sin().float()

    def turn(t):
        a, b, rest = t[..., :8], t[..., 8:16], t[..., 16:]
        return torch.cat([a * c - b * n, b * c + a * n, rest], -1)
    q, k, v = turn(qkv[:, :Hq]), turn(qkv[:, Hq:Hq + Hk]), qkv[:, Hq + Hk:]
    i = torch.arange(L)
    off = (i[None] > i[:, None]) | (i[None] < i[:, None] - W)
    a = (q @ k.repeat_interleave(2, 1).transpose(-1, -2) / math.sqrt(d)).masked_fill(off, -math.inf).softmax(-1)
    want = (a @ v.repeat_interleave(2, 1)).transpose(1, 2).reshape(B, L, -1) @ p["out"]
    loss = (want * dout.cpu().float()).sum() + (s * dS.cpu().float()).sum()
    names = ["norm", "norm_bias", "qkv", "out"]
    ref = torch.autograd.grad(loss, [s] + [p[k] for k in names])
    rel = lambda a, b: ((a.cpu().float() - b).norm() / b.norm()).item()   # noqa: E731
    for name, got, b in zip(["output", "x"] + names, [out, dx] + [grads[k] for k in names], [want.detach()] + list(ref)):
        e = rel(got, b)
        print(name, e)
        assert e < 12 * 2.0 ** -9, (name, e)


@pytest.mark.parametrize("kind", ["sinkhorn", "softmax"])
def test_training(kind):
    from attention_layer import train
    losses = train(kind, steps=8, L=512)
    print(kind, losses)
    assert all(math.isfinite(x) for x in losses) and losses[-1] < 0.9 * losses[0]


def test_tokens_one_by_one():
    """Against all at once: a handful of roundings of values of a few units."""
    from attention_layer import AttentionLayer
    layer = AttentionLayer("softmax", 128, 4, 2, 32, 17, causal=True, rot=32, scaling="yarn", factor=4.0, trained_length=64)
    g = torch.Generator(device="cuda").manual_seed(0)
    B, L = 3, 60
    x, r = (torch.randn((B, L, 128), generator=g, device="cuda").bfloat16() for _ in range(2))
    whole, _, _ = layer.forward(x, r)
    cache = [torch.full((B, 2, L, 32), math.nan, device="cuda", dtype=torch.bfloat16) for _ in range(2)]
    length = torch.zeros(B, device="cuda", dtype=torch.int32)
    outs = []
    for t in range(L):
        outs.append(layer.token(x[:, t:t + 1], r[:, t:t + 1], cache, length)[0])
        length = length + 1
    got = torch.cat(outs, 1).float()
    assert (got - whole.float()).norm() < 6 * 2.0 ** -9 * whole.float().norm()
