"""Layer operators at documented sizes that take more threads than one launch can have (2^32 in a dimension).  Inputs are broadcast, so
that the results alone fill memory."""
import pytest
import torch

import paper_2605_08123_amd as ska

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(autouse=True)
def memory():
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


def rows(x, n=1 << 20):
    return ((i, x[i:i + n]) for i in range(0, x.shape[0], n))


def test_rope_of_many_tokens():
    """2^24 tokens of 257 slots (single features): two launches."""
    L, d = 1 << 24, 258
    print("\n[case] rope", L, d, flush=True)
    x = torch.randn(1, 1, 1, d, generator=torch.Generator().manual_seed(1)).to(BF16).cuda()
    freq = torch.tensor([0.37], dtype=torch.float64, device="cuda")
    out = ska.ska_rope_fwd(x.expand(1, 1, L, d), None, freq, 1.0)[0][0, 0]
    torch.cuda.synchronize()
    x1, x2 = x[0, 0, 0, 0].double(), x[0, 0, 0, 1].double()
    for i, part in rows(out):
        assert (part[:, 2:] == x[0, 0, 0, 2:]).all(), i
        t = torch.arange(i, i + part.shape[0], device="cuda", dtype=torch.float64) * freq
        c, s = t.cos(), t.sin()
        for y, want in ((part[:, 0], x1 * c - x2 * s), (part[:, 1], x2 * c + x1 * s)):
            # half a step of bf16 and a dozen of fp32 for the angle, the functions and the products
            assert ((y.double() - want).abs() <= 2.0 ** -8 * want.abs() + 12 * 2.0 ** -24 * (x1.abs() + x2.abs())).all(), i
