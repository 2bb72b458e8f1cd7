"""Calls of the layer operators with arguments at the ends of their ranges, on the GPU."""
import sys

import pytest
import torch

import paper_2605_08123_amd as ska

from . import layer_ref as ref

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("W", [2 ** 31, 2 ** 32, sys.maxsize])
def test_a_band_of_everything(W):
    print("\n[case] W", W, flush=True)
    g = torch.Generator().manual_seed(1)
    q, k, v = (torch.randn(1, 2, 130, 64, generator=g).to(BF16).cuda() for _ in range(3))
    O, LSE = ska.ska_softmax_attn_fwd(q, k, v, W, causal=True)
    want = ska.ska_softmax_attn_fwd(q, k, v, 130, causal=True)
    assert torch.equal(O, want[0]) and torch.equal(LSE, want[1])
    for a, b in zip(ska.ska_softmax_attn_bwd(q, k, v, O, q, LSE, W, causal=True), ska.ska_softmax_attn_bwd(q, k, v, O, q, LSE, 130, causal=True)):
        assert torch.equal(a, b)
