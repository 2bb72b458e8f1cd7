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


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,D", [(33, 100), (5, 9000)])
def test_gradient_of_a_bias_without_a_weight(rows, D, dtype):
    """A norm with a bf16 bias alone, which the forward takes: its gradient in the bias's type."""
    print("\n[case] bias alone", rows, D, dtype, flush=True)
    g = torch.Generator().manual_seed(D)
    s, dy = (torch.randn(rows, D, generator=g).to(dtype) for _ in range(2))
    b = torch.randn(D, generator=g).to(BF16)
    Y, _, _ = ska.ska_layer_norm_fwd(s.cuda(), bias=b.cuda())
    _, y, mean, rstd = ref.norm_fwd(s, None, b, None, 1e-5)
    ref.check("Y", Y, y)
    st = torch.stack([mean[0], rstd[0]]).float()
    want = ref.norm_bwd(dy, s, None, st, None, BF16)
    into = torch.empty(D, dtype=BF16, device="cuda")
    dX, dw, db = ska.ska_layer_norm_bwd(dy.cuda(), s.cuda(), None, st.cuda(), want_weight=False, dbias=into)
    assert dw is None and db is into
    ref.check("dX", dX, want[0])
    ref.check("dbias", db, want[2])
    _, dw, db = ska.ska_layer_norm_bwd(dy.cuda(), s.cuda(), None, st.cuda(), dweight=into)
    assert dw is into and db.dtype == BF16
    ref.check("dweight", dw, want[1])
    ref.check("dbias", db, want[2])
    _, dw, db = ska.ska_layer_norm_bwd(dy.cuda(), s.cuda(), None, st.cuda())
    assert dw.dtype == db.dtype == F32


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("start", [2 ** 31 - 1, 2 ** 31 - 3, -2 ** 31])
def test_rope_starts_at_the_ends_of_32_bits(start, dtype):
    """Tokens that follow a start near 2^31 stand beyond it."""
    print("\n[case] rope start", start, dtype, flush=True)
    B, H, L, d = 2, 2, 9, 64
    q = torch.randn(B, H, L, d, generator=torch.Generator().manual_seed(3)).to(dtype)
    freq, amp = ska.ska_rope_frequencies(d)
    at = torch.tensor([start, 5], dtype=torch.int32)
    got, _ = ska.ska_rope_fwd(q.cuda(), None, freq.cuda(), amp, start=at.cuda())
    ref.check("Q", got, ref.rope(q, freq, amp, torch.arange(L) + at.long()[:, None], False))
