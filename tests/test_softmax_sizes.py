"""How large a workspace the softmax loss asks for (no GPU)."""
import pytest
import torch

from paper_2009_06693_amd import binding as B

MB = 1 << 20


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


def test_a_gradient_asks_for_no_less_than_the_loss():
    for dtype in (torch.float32, torch.bfloat16):
        for n, V, d in ((1, 1, 8), (9, 1000, 64), (5000, 3000, 128), (700, 90000, 300)):
            assert _size(n, V, d, 2, dtype, True) > _size(n, V, d, 2, dtype, False) > 0
