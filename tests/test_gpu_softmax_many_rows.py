"""The softmax loss over so many rows that their places come from a scan of their own, and either side of where that begins
(blocks of 128 rows, 2,048 of them)."""
import pytest
import torch

from paper_2009_06693_amd import binding as B

from rows_util import TYPES, Loss

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("kind,n,grad", [("f16", 2048 * 128, True), ("f16", 2048 * 128 + 1, True), ("bf16", 4097 * 128 + 5, False),
                                         ("f32", 2500 * 128 - 3, True), ("bf16", 9000 * 128 + 77, False)])
def test_places_of_many_rows(kind, n, grad):
    V, d, k, dtype = 40, 16, 2, TYPES[kind]
    g = torch.Generator().manual_seed(n)
    x, w = (torch.randn(n, d, generator=g) * 0.5).to(dtype).to(DEV), torch.randn(V, d, generator=g).to(dtype).to(DEV)
    labels = torch.randint(-1, V, (n, k), generator=g).int()
    labels[torch.rand(n, generator=g) < 0.3] = -1
    labels[5000:9000] = -1       # blocks without a label
    labels = labels.to(DEV)
    x[labels.amax(1) < 0] = float("nan")
    weight = ((torch.rand(n, generator=g) + 0.5) / n).to(DEV)
    print(f"[many] n={n} {kind}", flush=True)
    op = B.SoftmaxLoss(n, V, d, k, dtype, grad=grad)
    op.workspace.fill_(0xFF)
    out = op.grad(x, w, labels, weight) if grad else op.loss(x, w, labels)
    op.status()
    Loss(x, w, labels, weight).check(*out)
    # a label that is no vertex, in the last block
    labels[n - 1, 0] = V
    op.loss(x, w, labels) if not grad else op.grad(x, w, labels, weight)
    with pytest.raises(B.NdError) as e:
        op.status()
    assert e.value.code == B.ND_ERR_BAD_ROOT
