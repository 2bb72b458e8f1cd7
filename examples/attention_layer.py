"""A pre-norm attention layer from the library's operators, trained and answering.

    S = x + r,  Y = layer norm(S),  q, k, v = Y Wqkv,  q, k turned by their positions,  O = attention(q, k, v),  out = O Wo

with the paper's banded Sinkhorn attention or softmax attention on the same band, forward and backward by hand (the library has
no autograd functions; projections are plain matrix products), and the softmax layer's form for single tokens against a
cache.  Run on a GPU: python examples/attention_layer.py
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2605_08123_amd as ska  # noqa: E402


class AttentionLayer:
    """kind: "sinkhorn" (as many key heads as query heads, not causal) or "softmax"."""

    def __init__(self, kind, D, Hq, Hk, d, W, causal=False, rot=None, base=10000.0, scaling="none", factor=1.0, trained_length=1,
                 T=8, R=2, eps=1.0, seed=0):
        if kind not in ("sinkhorn", "softmax") or (kind == "sinkhorn" and (Hq != Hk or causal)):
            raise ValueError("sinkhorn attention has one key head per query head and no causal form")
        g = torch.Generator(device="cuda").manual_seed(seed)
        rnd = lambda *s: (torch.randn(*s, generator=g, device="cuda") * s[0] ** -0.5).bfloat16()   # noqa: E731
        self.kind, self.Hq, self.Hk, self.d, self.W, self.causal, self.T, self.R, self.eps = kind, Hq, Hk, d, W, causal, T, R, eps
        self.params = {"norm": torch.ones(D, device="cuda"), "norm_bias": torch.zeros(D, device="cuda"),
                       "qkv": rnd(D, (Hq + 2 * Hk) * d), "out": rnd(Hq * d, D)}
        freq, self.amplitude = ska.ska_rope_frequencies(rot or d, base, scaling, factor, trained_length)
        self.freq = freq.cuda()

    def _heads(self, qkv):
        """[B, L, (Hq + 2 Hk) d] -> views [B, H, L, d] of q, k, v."""
        B, L, _ = qkv.shape
        x = qkv.view(B, L, self.Hq + 2 * self.Hk, self.d).transpose(1, 2)
        return x[:, :self.Hq], x[:, self.Hq:self.Hq + self.Hk], x[:, self.Hq + self.Hk:]

    def forward(self, x, r):
        """x, r [B, L, D] bf16 -> the layer's output, the sum that goes on beside it, and what the backward needs."""
        p = self.params
        Y, S, stats = ska.ska_layer_norm_fwd(x, p["norm"], p["norm_bias"], residual=r)
        q, k, v = self._heads(Y @ p["qkv"])
        Q, K = ska.ska_rope_fwd(q, k, self.freq, self.amplitude)      # reads the projection's layout, writes [B, H, L, d]
        if self.kind == "softmax":
            O = torch.empty((Q.shape[0], Q.shape[2], self.Hq, self.d), device=Q.device, dtype=Q.dtype).transpose(1, 2)
            O, state = ska.ska_softmax_attn_fwd(Q, K, v, self.W, self.causal, self.eps, O=O)
        else:
            v = v.contiguous()
            O, state = ska.sinkhorn_attn_fwd(Q, K, v, self.W, self.T, self.R, self.eps)
        flat = O.transpose(1, 2).reshape(*x.shape[:2], -1)
        return flat @ p["out"], S, (Y, S, stats, Q, K, v, O, state, flat)

    def backward(self, dout, dS, saved):
        """Gradients of x (and of r, the same) and of the parameters."""
        p, (Y, S, stats, Q, K, v, O, state, flat) = self.params, saved
        B, L, D = S.shape
        rows = lambda t: t.reshape(B * L, -1)   # noqa: E731
        grads = {"out": rows(flat).t() @ rows(dout)}
        dO = (dout @ p["out"].t()).view(B, L, self.Hq, self.d).transpose(1, 2)
        dqkv = torch.empty((B, L, (self.Hq + 2 * self.Hk) * self.d), device=S.device, dtype=S.dtype)
        dq, dk, dv = self._heads(dqkv)
        if self.kind == "softmax":
            dQ, dK, _ = ska.ska_softmax_attn_bwd(Q, K, v, O, dO, state, self.W, self.causal, self.eps, dV=dv)
        else:
            dQ, dK, dV = ska.sinkhorn_attn_bwd(Q, K, v, O, dO.contiguous(), state, self.W, self.T, self.R, self.eps)
            dv.copy_(dV)
        ska.ska_rope_bwd(dQ, dK, self.freq, self.amplitude, dQ=dq, dK=dk)   # back into the projection's layout
        grads["qkv"] = rows(Y).t() @ rows(dqkv)
        dx, grads["norm"], grads["norm_bias"] = ska.ska_layer_norm_bwd(dqkv @ p["qkv"].t(), S, p["norm"], stats, dS=dS)
        return dx, grads

    def token(self, x, r, cache, length):
        """One more token per sequence (softmax, causal): x, r [B, 1, D]; cache: keys and values [B, Hk, L, d], of which length [B]
        (int32) tokens are there and to which this one is appended.  -> output and sum."""
        p = self.params
        Y, S, _ = ska.ska_layer_norm_fwd(x, p["norm"], p["norm_bias"], residual=r)
        q, k, v = self._heads(Y @ p["qkv"])
        Q, K = ska.ska_rope_fwd(q, k, self.freq, self.amplitude, start=length)
        b = torch.arange(x.shape[0], device=x.device)
        cache[0][b, :, length.long()], cache[1][b, :, length.long()] = K[:, :, 0], v[:, :, 0]
        O, _ = ska.ska_softmax_attn_fwd(Q, cache[0], cache[1], self.W, True, self.eps, len_k=length + 1, start_q=length)
        return O.transpose(1, 2).reshape(x.shape[0], 1, -1) @ p["out"], S


def train(kind, steps=12, B=2, L=1024, D=256, H=4, d=64, W=128, rate=30.0, seed=1):
    """Fits the layer to another one's outputs; returns the loss per step."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x, r = (torch.randn((B, L, D), generator=g, device="cuda").bfloat16() for _ in range(2))
    layer, goal = (AttentionLayer(kind, D, H, H, d, W, seed=s) for s in (2, 3))
    want, _, _ = goal.forward(x, r)
    losses = []
    for _ in range(steps):
        out, S, saved = layer.forward(x, r)
        off = out.float() - want.float()
        losses.append(off.square().mean().item())
        _, grads = layer.backward((off * (2 / off[0, 0].numel())).bfloat16(), torch.zeros_like(S), saved)
        for name, p in layer.params.items():
            p.copy_((p.float() - rate / (B * L) * grads[name].float()).to(p.dtype))
    return losses


def main():
    a = argparse.ArgumentParser()
    a.add_argument("--steps", type=int, default=12)
    steps = a.parse_args().steps
    for kind in ("sinkhorn", "softmax"):
        print(kind, "loss per step:", " ".join(f"{x:.4f}" for x in train(kind, steps)))
    layer = AttentionLayer("softmax", 256, 8, 2, 64, 1 << 20, causal=True)
    g = torch.Generator(device="cuda").manual_seed(0)
    B, L = 3, 40
    x, r = (torch.randn((B, L, 256), generator=g, device="cuda").bfloat16() for _ in range(2))
    whole, _, _ = layer.forward(x, r)
    cache = [torch.zeros((B, 2, L, 64), device="cuda", dtype=torch.bfloat16) for _ in range(2)]
    length = torch.zeros(B, device="cuda", dtype=torch.int32)
    off = 0.0
    for t in range(L):
        out, _ = layer.token(x[:, t:t + 1], r[:, t:t + 1], cache, length)
        length += 1
        off = max(off, (out[:, 0].float() - whole[:, t].float()).abs().max().item())
    print(f"token by token against all at once: largest difference {off:.4f} (outputs of size {whole.float().abs().mean().item():.2f})")


if __name__ == "__main__":
    main()
