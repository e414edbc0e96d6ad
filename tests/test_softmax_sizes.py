"""How large a workspace the softmax loss asks for (no GPU)."""
import pytest
import torch

from paper_2009_06693_amd import binding as B

MB, GB = 1 << 20, 1 << 30


def _size(n, V, d, k=1, dtype=torch.bfloat16, grad=True):
    return B.nd_softmax_loss_workspace_bytes(n, V, d, k, dtype, grad)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("d", [64, 128, 200, 256])
def test_small_calls_ask_for_little(d, dtype):
    """Room for as many parts as the work is cut into, not as many as the chip could take."""
    assert _size(1, 1, d, dtype=dtype) < 4 * MB
    assert _size(20, 300, d, 3, dtype) < 16 * MB
    # w and its gradient's parts, once each in 32 bits and as a copy
    assert _size(1, 57000, d, dtype=dtype) < 57000 * 256 * 12 + 8 * MB


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("n,V,d", [(16384, 65536, 512), (8192, 130000, 512), (2049, 57000, 1000), (32768, 32768, 1024),
                                   (20000, 300000, 512), (16384, 233000, 300), (4096, 4096, 128)])
def test_scores_and_probabilities_are_bounded(n, V, d, dtype):
    """4 GB of scores where they are kept, and 512 MB of probabilities (fp32: in the scores' place); the rest is rows: those of x
    and w, and parts of the gradients in 32 bits."""
    b = 4 if dtype == torch.float32 else 2
    rows = (n + V + 1024) * (d + 64)
    # gathered x, a copy of w and the sums over labels, once each; parts of dx and dw: at most 64 shares of 256 rows a compute unit
    rest = rows * (b + 4 + 4) + 2 * 512 * 256 * 128 * 4 + 64 * n + 64 * MB
    probabilities = 512 * MB
    assert _size(n, V, d, 1, dtype) <= 4 * GB + probabilities + rest
    kept = (n + 255) // 256 * 256 * ((V + 255) // 256 * 256) * 4 <= 4 * GB
    if not kept:
        assert _size(n, V, d, 1, dtype) <= probabilities + rest


def test_a_gradient_asks_for_no_less_than_the_loss():
    for dtype in (torch.float32, torch.bfloat16):
        for n, V, d in ((1, 1, 8), (9, 1000, 64), (5000, 3000, 128), (700, 90000, 300)):
            assert _size(n, V, d, 2, dtype, True) > _size(n, V, d, 2, dtype, False) > 0
