"""Gradients of rows that the model fits already: a label's probability times the labels there are is close to how often it is
one, and what is left of the two is the gradient.

Every product and sum of a score is exact in fp32 here (labels' rows are rows of a Hadamard matrix, the others' numbers are
+-1/4, x is a small multiple of the sum of the labels' rows), so that what a label weighs may be off by the exponentials and
their sum in fp32 alone, and by nothing that a 16-bit type rounds: half a step of the type, 2^-9 of p in bf16, is what the
difference of p = 0.998 and 1 is.
"""
import math

import pytest
import torch

from paper_2009_06693_amd import binding as B

from rows_util import TYPES, U32, assert_within, half_step, rounded

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TARGETS = (0.9, 0.99, 0.999, 0.9999)


def _hadamard(size):
    h = torch.ones(1, 1, dtype=torch.float64)
    while h.shape[0] < size:
        h = torch.cat([torch.cat([h, h], 1), torch.cat([h, -h], 1)], 0)
    return h


def _inputs(n, V, d, k, dtype, seed, repeat=False):
    """(x, w, labels, row_weight): row i's labels together have a probability near TARGETS[i % 4]."""
    g = torch.Generator().manual_seed(seed)
    side = 1 << int(math.log2(d))
    count = min(side - 1, V, 90)
    # neighbours in a block of vertices, the first and the last vertex, and some anywhere
    at = torch.cat([torch.arange(count // 2), torch.tensor([V - 1]), torch.randperm(V, generator=g)])
    at = torch.tensor(list(dict.fromkeys(at.tolist()))[:count])
    w = torch.randint(0, 2, (V, d), generator=g).double() * 0.5 - 0.25
    w[at] = 0.0
    w[at, :side] = _hadamard(side)[1:count + 1]
    pick = torch.stack([torch.randperm(count, generator=g)[:k] for _ in range(n)])
    if repeat:  # some labels twice
        pick[::2, 0] = pick[::2, k - 1]
    labels = at[pick].int()
    x = torch.zeros(n, d, dtype=torch.float64)
    steps = (1.0,) if k > 16 else tuple(a / 8 for a in range(8, 16))  # few bits: k times 15 of them are exact in bf16
    for i in range(n):
        rows = torch.zeros(V, dtype=torch.float64)
        rows[labels[i].long().unique()] = 1.0
        sums = rows @ w
        products = w @ sums
        best = None
        for e in range(1, 9):
            for a in steps:
                s = products * (a * 2.0 ** -e)
                p = float(torch.softmax(s, 0)[rows > 0].sum())
                miss = abs(math.log((1 - p + 1e-12) / (1 - TARGETS[i % 4])))
                if float(s.max()) < 30 and (best is None or miss < best[0]):
                    best = (miss, a * 2.0 ** -e)
        x[i] = sums * best[1]
    xt, wt = x.to(dtype), w.to(dtype)
    assert torch.equal(xt.double(), x) and torch.equal(wt.double(), w)
    return xt, wt, labels, torch.rand(n, generator=g) + 0.5


class Fitted:
    """The formulas in 64 bits with what may be off."""

    def __init__(self, x, w, labels, row_weight):
        n, V, dtype = x.shape[0], w.shape[0], x.dtype
        k = labels.shape[1]
        xd, wd, g = x.double(), w.double(), row_weight.double()[:, None]
        held = torch.zeros(n, V, dtype=torch.float64).scatter_add_(1, labels.long(), torch.ones(n, k, dtype=torch.float64))
        s = xd @ wd.T
        lse = torch.logsumexp(s, 1)
        p = (s - lse[:, None]).exp()
        self.held, self.p = held, p
        rate = g * (k * p - held)
        self.dx, self.dw = rate @ wd, rate.T @ xd
        # Scores are exact.  An exponential: its argument, the product with log2 e, itself (4 and 8 half steps); the sum of V of
        # them; the quotient.  All relative, of k p and of the count next to it.
        de = (4 * (s.abs().max(1).values + lse.abs()) + 8) * U32
        dp = (2 * de + (V + 16) * U32)[:, None]
        u = half_step(dtype)
        # a vertex that is no label: what it weighs is rounded to the type (fp16: in steps of 2^-39 k of the largest weight)
        under = float(g.max()) * k * 2.0 ** -38 if dtype == torch.float16 else 0.0
        off = torch.where(held > 0, g * (k * p + held) * dp, g * k * p * (dp + u + 4 * U32) + under)
        # sums in fp32: their terms' sizes, with what the labels' rows are when they are taken off
        size = g * (k * p + held)
        self.dx_tol = rounded(self.dx, off @ wd.abs() + (k + 24) * U32 * (size @ wd.abs()), dtype)
        self.dw_tol = rounded(self.dw, off.T @ xd.abs() + (n / 4 + 24) * U32 * (size.T @ xd.abs()), dtype)


def _call(args, dx=True, dw=True):
    x, w, labels, row_weight = args
    n, d = x.shape
    V = w.shape[0]
    loss, lse = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    gx = torch.full_like(x, float("nan")) if dx else None
    gw = torch.full_like(w, float("nan")) if dw else None
    ws = torch.full((B.nd_softmax_loss_workspace_bytes(n, V, d, labels.shape[1], x.dtype, True),), 0xFF, dtype=torch.uint8,
                    device=DEV)
    B.nd_softmax_loss_grad(x, w, labels, row_weight, loss, lse, gx, gw, ws)
    torch.cuda.synchronize()
    return loss, lse, gx, gw


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("d", [40, 128, 256, 300, 520])
@pytest.mark.parametrize("k,repeat", [(1, False), (10, False), (10, True)])
def test_rows_that_are_fitted(k, repeat, d, kind):
    n, V = 96, 400
    args = _inputs(n, V, d, k, TYPES[kind], seed=d + k, repeat=repeat)
    want = Fitted(*args)
    total = (want.p * (want.held > 0)).sum(1)
    assert float(total.max()) > 0.999 and float(total.min()) < 0.95
    print(f"[fitted] n={n} V={V} d={d} k={k} {kind}", flush=True)
    loss, lse, dx, dw = _call([t.to(DEV) for t in args])
    assert_within(dx, want.dx, want.dx_tol, "dx")
    assert_within(dw, want.dw, want.dw_tol, "dw")


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("n,V,d,k", [(300, 20011, 128, 10), (70, 20000, 256, 5), (40, 9001, 64, 40), (260, 7001, 300, 3),
                                     (129, 7001, 520, 1), (3, 30000, 100, 1), (600, 91, 128, 10)])
def test_fitted_rows_over_more_vertices(n, V, d, k, kind):
    """Rows' labels in parts of the vertices that different workgroups sweep; either gradient alone has the same numbers."""
    args = _inputs(n, V, d, k, TYPES[kind], seed=n + V, repeat=k == 5)
    want = Fitted(*args)
    print(f"[fitted] n={n} V={V} d={d} k={k} {kind}", flush=True)
    args = [t.to(DEV) for t in args]
    _, _, dx, dw = _call(args)
    assert_within(dx, want.dx, want.dx_tol, "dx")
    assert_within(dw, want.dw, want.dw_tol, "dw")
    assert torch.equal(_call(args, dw=False)[2], dx)
    alone = _call(args, dx=False)[3]
    assert_within(alone, want.dw, want.dw_tol, "dw alone")


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("d", [128, 300, 520])
def test_fitted_rows_with_weights_of_either_sign(d, kind):
    n, V = 96, 400
    x, w, labels, row_weight = _inputs(n, V, d, 2, TYPES[kind], seed=d)
    row_weight[::3] *= -1
    row_weight[::5] = 0
    # the allowances go by sizes
    want = Fitted(x, w, labels, row_weight.abs())
    signed = Fitted(x, w, labels, row_weight)
    u = half_step(x.dtype)
    _, _, dx, dw = _call([t.to(DEV) for t in (x, w, labels, row_weight)])
    assert_within(dx, signed.dx, want.dx_tol, "dx")
    assert_within(dw, signed.dw, want.dw_tol + signed.dw.abs() * u, "dw")


@pytest.mark.parametrize("kind", ["bf16", "f16"])
def test_a_vertex_that_is_every_rows_label(kind):
    """And the only vertex there is: what is left is nothing."""
    for d in (64, 128, 256, 300, 520):
        n = 70
        g = torch.Generator().manual_seed(d)
        x = torch.randint(-4, 5, (n, d), generator=g).to(TYPES[kind]).to(DEV)
        w = torch.ones(1, d, dtype=TYPES[kind], device=DEV)
        labels = torch.zeros(n, 3, dtype=torch.int32, device=DEV)
        weight = (torch.rand(n, generator=g) + 0.3).to(DEV)
        _, _, dx, dw = _call([x, w, labels, weight])
        # rate = 3 - 3 p, p the quotient of a number and itself; the sum over 70 rows in fp32 on top
        assert float(dx.abs().max()) <= 3 * 1.3 * 8 * U32, d
        assert float(dw.abs().max()) <= 3 * 1.3 * 4 * n * (n / 4 + 24) * U32, d
