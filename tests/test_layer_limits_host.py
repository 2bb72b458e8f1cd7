"""The layer operators' binding and the limits of their sizes and arguments that hold before anything is launched (no GPU)."""
import os
import subprocess
import sys

import torch

import paper_2605_08123_amd as ska
from paper_2605_08123_amd import binding, layer

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_softmax_sizes_fit_a_launch():
    """2^24 - 8 blocks of 128 rows: a refused size has no workspace and its calls are SKA_EUNSUPPORTED."""
    most, rows = (1 << 24) - 8, 1 << 24
    need = lambda n, Lq, Lk=1, G=1, back=True, W=8: ska.ska_softmax_attn_workspace_bytes(back, 1, n * G, n, Lq, Lk, 32, W)   # noqa: E731
    full = most // (rows // 128)      # 127 problems of 2^24 rows, and one more
    assert need(full, rows) > 0 and need(full, 1, rows) > 0 and need(full, rows // 4, 1, 4) > 0
    assert need(full + 1, rows) == 0 and need(full + 1, 1, rows) == 0 and need(full + 1, rows // 4, 1, 4) == 0
    assert need(65535, 128 * 256) > 0 and need(65535, 128 * 256 + 1) == 0
    # the forward's blocks are the queries' alone: one token against a cache of any documented size
    assert need(full + 1, 1, rows, back=False, W=rows) > 0 and need(full + 1, 1, rows, W=rows) == 0
    lib, P = layer._lib(), 1 << 20   # (not read: the size is refused first)
    args = [1, full + 1, full + 1, rows, 1, 32, 8, 0, 1.0, binding.SKA_BF16]
    assert lib.ska_softmax_attn_fwd(P, None, P, None, P, None, P, None, P, *[None] * 5, *args, P, 1 << 60, None) == binding.SKA_EUNSUPPORTED
    assert lib.ska_softmax_attn_bwd(P, None, P, None, P, None, P, None, P, None, P, P, None, P, None, P, *[None] * 6, *args, P, 1 << 60,
                                    None) == binding.SKA_EUNSUPPORTED


def test_import_without_the_raw_stream():
    """A build of torch without its function for the raw stream: the package is imported, host-side calls work."""
    code = ("import torch; del torch._C._cuda_getCurrentRawStream\n"
            "import paper_2605_08123_amd as ska\n"
            "assert ska.ska_rope_frequencies(8)[0].numel() == 4 and ska.ska_layer_norm_workspace_bytes(8, 64) > 0\n")
    res = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert res.returncode == 0, res.stderr


def test_the_stream_without_the_raw_function(monkeypatch):
    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream")
    monkeypatch.setattr(torch.cuda, "current_stream", lambda dev: type("Stream", (), {"cuda_stream": 40 + dev}))
    assert layer._raw_stream(2) == 42


def test_numbers_beyond_32_bits():
    """A band as wide as can be said is everything, not what its lower 32 bits say; below 0 it is refused."""
    need = lambda W, back=False: ska.ska_softmax_attn_workspace_bytes(back, 1, 4, 2, 1, 65536, 64, W)   # noqa: E731
    assert need(1 << 20) > need(0) == 0
    for W in (2 ** 31, 2 ** 32, 2 ** 32 + 5, sys.maxsize, 2 ** 80):
        assert need(W) == need(1 << 20), W
    for W in (-1, -2 ** 31 - 1, -2 ** 32, -2 ** 32 + 7):
        assert need(W) == 0 and need(W, True) == 0 < need(0, True), W
    far = ska.ska_rope_frequencies(64, scaling="yarn", factor=4.0, trained_length=2 ** 31 - 1)[0]
    assert torch.equal(ska.ska_rope_frequencies(64, scaling="yarn", factor=4.0, trained_length=2 ** 32 + 4096)[0], far)


def test_softmax_scale_is_a_number():
    """1 / (eps sqrt d) of 0 or beyond fp32 made masked scores 0 times -inf.  (Without the workspace that both need: nothing is launched.)"""
    lib, P = layer._lib(), 1 << 20

    def calls(eps, d):
        args = [1, 2, 2, 1, 65536, d, 1 << 20, 0, eps, binding.SKA_BF16, None, 0, None]
        return [lib.ska_softmax_attn_fwd(P, None, P, None, P, None, P, None, P, *[None] * 5, *args),
                lib.ska_softmax_attn_bwd(P, None, P, None, P, None, P, None, P, None, P, P, None, P, None, P, *[None] * 6, *args)]
    for d in (32, 64, 128):
        for eps in (3e38, 2e37, 1e-40, 1e-45):
            assert calls(eps, d) == [binding.SKA_EUNSUPPORTED] * 2, (eps, d)
        for eps in (1e36, 1.0, 1e-30, 1e-37):
            assert calls(eps, d) == [binding.SKA_EWORKSPACE] * 2, (eps, d)
