"""Attention behind a prefix with so many query rows that the join of its parts takes 2^32 threads."""
import math

import pytest
import torch

import paper_2605_08123_amd as ska

from . import cache_ref as ref
from .layer_ref import check
from .test_gpu_cache import ALL, BF16, case, say

pytestmark = pytest.mark.gpu


def test_join_of_2_to_the_26_rows():
    """d = 128, two parts: 64 threads a row.  All items are the same, by strides of 0; their 2^26 rows and the parts take 87 GB."""
    B, Lq, Lp, Lk, d = 4096, 1 << 14, 64, 32, 128
    need = ska.ska_prefix_attn_workspace_bytes(B, 1, 1, Lq, Lp, Lk, d, ALL, True, 1, 1)
    say("many rows", B, Lq, d, need)
    assert need >= 2 * B * Lq * (d + 1) * 4
    torch.cuda.empty_cache()
    assert torch.cuda.mem_get_info()[0] > need + B * Lq * d * 2 + (8 << 30)
    g = torch.Generator().manual_seed(0)
    q, k, v = case(g, 1, 1, 1, Lq, Lk, d, BF16)
    _, pk, pv = case(g, 1, 1, 1, 1, Lp, d, BF16)
    O = torch.full((B, 1, Lq, d), math.nan, device="cuda", dtype=BF16)
    LSE = torch.full((B, 1, Lq), math.nan, device="cuda")
    many = lambda x: x.cuda().expand(B, -1, -1, -1)   # noqa: E731
    ska.ska_prefix_attn_fwd(many(q), (pk[0].cuda(), pv[0].cuda()), (many(k), many(v)), ALL, O=O, LSE=LSE)
    want = ref.prefix_attn(q, pk[0].double(), pv[0].double(), k.double(), v.double(), ALL, True, 1.0, codes=False)
    check("O", O[:1], want["O"])
    check("LSE", LSE[:1], want["LSE"])
    for b in range(0, B, 64):   # 32 rows to a workgroup, which do not pass an item's end: the same bits for all
        assert (O[b:b + 64] == O[:1]).all() and (LSE[b:b + 64] == LSE[:1]).all(), b
    del O, LSE
    torch.cuda.empty_cache()
