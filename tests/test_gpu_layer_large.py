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


def norm_row(x, w, b):
    """A row's layer norm in 64 bits, and its backward's (mean, rstd)."""
    f = x.double()
    mean, rstd = f.mean(), (f.var(unbiased=False) + 1e-5).rsqrt()
    return (f - mean) * rstd * w.double() + b.double(), mean, rstd


@pytest.mark.parametrize("N,D", [((1 << 26) + 5, 257),      # a wavefront's row
                                 ((1 << 24) + 3, 2056)])    # a block's
def test_layer_norm_of_many_rows(N, D):
    print("\n[case] layer norm", N, D, flush=True)
    g = torch.Generator().manual_seed(2)
    x, w, b = torch.randn(1, D, generator=g).to(BF16).cuda(), torch.randn(D, generator=g).cuda(), torch.randn(D, generator=g).cuda()
    Y, _, stats = ska.ska_layer_norm_fwd(x.expand(N, D), w, b)
    torch.cuda.synchronize()
    want, mean, rstd = norm_row(x[0], w, b)
    assert ((Y[0].double() - want).abs() <= 2.0 ** -8 * want.abs() + 1e-4).all()
    for i, part in rows(Y):
        assert (part == Y[0]).all(), i
    assert (stats == stats[:, :1]).all()
    assert abs(stats[0, 0].item() - mean.item()) < 1e-6 and abs(stats[1, 0].item() - rstd.item()) < 1e-5


def test_layer_norm_gradient_of_many_wide_rows():
    """Rows that no block holds in registers, one to a block of 1024 threads."""
    N, D = (1 << 22) + 2, 8200
    print("\n[case] layer norm gradient", N, D, flush=True)
    g = torch.Generator().manual_seed(3)
    s, dy = (torch.randn(1, D, generator=g).to(BF16).cuda() for _ in range(2))
    _, mean, rstd = norm_row(s[0], torch.ones(D, device="cuda"), torch.zeros(D, device="cuda"))
    stats = torch.stack([mean, rstd]).float()[:, None].expand(2, N).contiguous()
    dX, dw, db = ska.ska_layer_norm_bwd(dy.expand(N, D), s.expand(N, D), None, stats, want_weight=False, want_bias=False)
    torch.cuda.synchronize()
    h, gd = (s[0].double() - mean) * rstd, dy[0].double()
    want = rstd * (gd - gd.mean() - h * (gd * h).mean())
    assert ((dX[0].double() - want).abs() <= 2.0 ** -8 * want.abs() + 1e-4).all() and dw is None and db is None
    for i, part in rows(dX, 1 << 18):
        assert (part == dX[0]).all(), i
