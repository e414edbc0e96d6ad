"""The softmax loss writes nothing behind the workspace it asks for, whatever part of it the work takes."""
import pytest
import torch

from paper_2009_06693_amd import binding as B

from rows_util import TYPES, Loss

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BEHIND = 1 << 20


def _inputs(n, V, d, k, dtype, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = (torch.randn(n, d, generator=g, device=DEV) * (2.0 / d ** 0.5)).to(dtype)
    w = torch.randn(V, d, generator=g, device=DEV).to(dtype)
    labels = torch.randint(0, V, (n, k), generator=g, device=DEV).int()
    return x, w, labels, (torch.rand(n, generator=g, device=DEV) + 0.5) / n


def _check(n, V, d, k, kind):
    dtype = TYPES[kind]
    args = _inputs(n, V, d, k, dtype, n + V)
    size = B.nd_softmax_loss_workspace_bytes(n, V, d, k, dtype, True)
    ws = torch.full((size + BEHIND,), 0xA5, dtype=torch.uint8, device=DEV)
    loss, lse = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    dx, dw = torch.empty_like(args[0]), torch.empty_like(args[1])
    print(f"[workspace] n={n} V={V} d={d} k={k} {kind}: {size} bytes", flush=True)
    B.nd_softmax_loss_grad(*args, loss, lse, dx, dw, ws[:size])
    assert bool((ws[size:] == 0xA5).all())
    Loss(*args).check(loss, lse, dx, dw)


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("n,V", [(1, 1), (1, 57), (1, 5000), (20, 300), (64, 64), (65, 257), (300, 1000), (1000, 300), (257, 20000),
                                 (2000, 90)])
def test_rows_of_sweeps(n, V, d, kind):
    _check(n, V, d, 2, kind)


@pytest.mark.parametrize("kind,n,V,d", [("bf16", 4600, 70000, 520), ("f16", 2100, 140000, 600), ("f32", 1200, 3000, 200)])
def test_kept_scores_whose_probabilities_come_in_pieces(n, V, d, kind):
    _check(n, V, d, 2, kind)
