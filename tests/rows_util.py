"""Plain 64-bit forms of the calls on rows, and what rounding may make of them.

u(T) is half a step of type T relative to a value; fp32 sums of t terms are off by at most t * 2^-24 of the sum of their
sizes.
"""
import torch

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
U32 = 2.0 ** -24


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def smallest(dtype):
    """Half the distance of the type's numbers next to zero."""
    return torch.finfo(dtype).smallest_normal * half_step(dtype)


def assert_within(got, want, tol, what=""):
    got = got.detach().cpu().double()
    want, tol = want.cpu(), tol.cpu()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    err = (got - want).abs()
    bad = ~(err <= tol)
    if bool(bad.any()):
        at = tuple(int(i) for i in bad.nonzero()[0])
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} off; first at {at}: got {float(got[at])}, want "
                             f"{float(want[at])}, off {float(err[at]):.3g}, allowed {float(tol[at]):.3g}")


def rounded(want, tol, dtype):
    """The allowance after rounding to the type."""
    u = half_step(dtype)
    return tol * (1 + u) + want.abs() * u + smallest(dtype)


class Loss:
    """The loss and its gradient in 64 bits, with allowances, from inputs as they are (on their device)."""

    def __init__(self, x, w, labels, row_weight=None):
        dtype = x.dtype
        n, d = x.shape
        V = w.shape[0]
        labels = labels.view(n, -1).long()
        k = labels.shape[1]
        counts = (labels >= 0) & (labels < V)
        c = counts.sum(1).double()
        live = c > 0
        xd = torch.where(live[:, None], x.double(), 0.0)  # rows without labels count nothing, whatever they hold
        wd = w.double()
        g = torch.ones(n, dtype=torch.float64, device=x.device) if row_weight is None else row_weight.double()
        g = torch.where(live, g, 0.0)
        held = torch.zeros(n, V + 1, dtype=torch.float64, device=x.device)
        held.scatter_add_(1, torch.where(counts, labels, V), torch.ones_like(labels, dtype=torch.float64))
        held = held[:, :V]
        s = xd @ wd.T
        size = xd.abs() @ wd.abs().T                        # sum of the products' sizes
        lse = torch.logsumexp(s, 1)
        p = (s - lse[:, None]).exp()
        rate = g[:, None] * (c[:, None] * p - held)
        self.lse = torch.where(live, lse, 0.0)
        self.loss = torch.where(live, c * lse - (held * s).sum(1), 0.0)
        self.dx, self.dw = rate @ wd, rate.T @ xd
        # a product's sum of d terms, twice that for the order and rounding inside a matrix instruction
        ds = 2 * (d + 2) * U32 * size.max(1).values
        # exp of a difference: the difference, its product with log2 e and the exponential each round
        de = ds + 4 * U32 * (s.abs().max(1).values + lse.abs()) + 8 * U32
        dlse = de + (V + 8) * U32                           # and the sum over V terms, relative, is absolute in the logarithm
        self.lse_tol = torch.where(live, dlse + 4 * U32 * lse.abs(), 0.0)
        self.loss_tol = torch.where(live, c * self.lse_tol + (held * size).sum(1) * 2 * (d + 2) * U32
                                    + (k + 4) * U32 * (c * lse.abs() + (held * s.abs()).sum(1)), 0.0)
        dp = de + dlse                                      # relative, of a probability
        u = half_step(dtype)
        some = g.abs()[:, None] * (c[:, None] * p + held)   # what is added up, without signs
        # probabilities are rounded to the type; in fp16 they end at 2^-24 of 2^15 / (largest weight * labels), half of that
        # is lost
        under = (g.abs().max() * k * 2.0 ** -39 * 2) if dtype == torch.float16 else torch.zeros((), device=x.device)
        # exponentials, products and sums in fp32 below its smallest normal number may be 0: so much is lost of a probability,
        # times weight and labels, and of every term of a sum
        least = 2.0 ** -126
        under = under + least * (1 + g.abs().max() * k)
        tol = (some * (2 * dp[:, None])) + (some * (u + 4 * U32)) + under * live[:, None]
        self.dx_tol = rounded(self.dx, tol @ wd.abs() + (V + k + 16) * (U32 * (some @ wd.abs()) + least), dtype)
        self.dx_tol = torch.where(live[:, None], self.dx_tol, 0.0)
        self.dw_tol = rounded(self.dw, tol.T @ xd.abs() + (n + 16) * (U32 * (some.T @ xd.abs()) + least), dtype)

    def check(self, loss, lse, dx=None, dw=None, what=""):
        assert_within(lse, self.lse, self.lse_tol, f"{what} lse")
        assert_within(loss, self.loss, self.loss_tol, f"{what} loss")
        if dx is not None:
            assert_within(dx, self.dx, self.dx_tol, f"{what} dx")
        if dw is not None:
            assert_within(dw, self.dw, self.dw_tol, f"{what} dw")


def groups_of(keys, V):
    """(sorted_slots, ids, start) of a stable grouping of the keys that are not negative."""
    order = torch.sort(keys.long(), stable=True)
    slots = order.indices[int((keys < 0).sum()):]
    sizes = torch.bincount(keys[keys >= 0].long(), minlength=V)
    ids = sizes.nonzero().view(-1)
    start = torch.zeros(ids.numel() + 1, dtype=torch.int64)
    start[1:] = sizes[ids].cumsum(0)
    return slots.int(), ids.int(), start.int()


def weighted_rows(z, index, weights, n, m):
    """(sums, sums of sizes) over a row's slots."""
    index = index.view(n, m).long()
    take = (index >= 0) & (index < z.shape[0])
    f = torch.where(take, 1.0 if weights is None else weights.view(n, m).double(), 0.0)
    rows = torch.where(take[:, :, None], z.double()[index.clamp(0, max(z.shape[0] - 1, 0))], 0.0) if z.shape[0] else \
        torch.zeros(n, m, z.shape[1], dtype=torch.float64)
    return (f[:, :, None] * rows).sum(1), (f[:, :, None] * rows).abs().sum(1)


def group_sums(x, slots, start, weights, m):
    """(sums, sums of sizes) per group."""
    slots = slots.long()
    rows = x.double()[slots // m]
    if weights is not None:
        rows = rows * weights.double()[slots][:, None]
    groups = start.numel() - 1
    of = torch.repeat_interleave(torch.arange(groups), (start[1:] - start[:-1]).long())
    out = torch.zeros(groups, x.shape[1], dtype=torch.float64)
    return out.index_add(0, of, rows[:of.numel()]), out.index_add(0, of, rows[:of.numel()].abs())
