"""Sums per group over a part of a grouping: offsets that do not begin at 0, with the pairs of the whole grouping.

Numbers are whole, so that every sum is exact, whatever its order.
"""
import pytest
import torch

from paper_2009_06693_amd import binding as B

from rows_util import TYPES

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _case(sizes, d, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    P = sum(sizes)
    start = torch.tensor([0] + sizes, dtype=torch.int64).cumsum(0).int()
    x = torch.randint(-2, 3, (P, d), generator=g).to(dtype)
    return x, torch.randperm(P, generator=g).int(), start


def _want(x, slots, start, dtype):
    per = x.double()[slots.long()].cumsum(0)
    per = torch.cat([torch.zeros(1, x.shape[1], dtype=torch.float64), per])
    return (per[start[1:].long()] - per[start[:-1].long()]).to(dtype)


SIZES = [[3, 4, 5, 2], [5, 15, 20, 1], [100, 50, 50], [64, 64, 64, 64], [1000, 3, 0, 9, 2000, 0], [0, 0, 7, 1, 0, 30], [1] * 700,
         [7] * 90, [40000, 11, 30000, 6]]


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: f"{len(s)}x{s[0]}")
@pytest.mark.parametrize("fill", [0, 0xFF])
def test_groups_from_the_middle_of_a_grouping(fill, sizes, kind):
    """Whatever the workspace holds, and into rows of a table as well."""
    d, dtype = 24, TYPES[kind]
    x, slots, start = _case(sizes, d, dtype, seed=len(sizes))
    n = len(sizes)
    ws = torch.empty(B.nd_rows_group_sum_workspace_bytes(slots.numel(), d), dtype=torch.uint8, device=DEV)
    for a, b in {(1, n), (n // 2, n), (1, 2), (n - 1, n), (n // 3 + 1, n - 1), (0, 1)}:
        if a >= b:
            continue
        part = start[a:b + 1]
        print(f"[slices] {kind} groups {a} to {b} of {n}, pairs from {int(part[0])}", flush=True)
        want = _want(x, slots, part, dtype)
        out = torch.full((b - a, d), float("nan"), dtype=dtype, device=DEV)
        ws.fill_(fill)
        B.nd_rows_group_sum(x.to(DEV), slots.to(DEV), part.to(DEV), 1, out=out, workspace=ws)
        assert torch.equal(out.cpu(), want)
        rows = torch.arange(a, b, dtype=torch.int32) * 2 + 1
        whole = torch.zeros(2 * n + 3, d, dtype=dtype)
        whole[rows.long()] = want
        out = torch.full_like(whole, float("nan"), device=DEV)
        ws.fill_(fill)
        B.nd_rows_group_sum(x.to(DEV), slots.to(DEV), part.to(DEV), 1, group_rows=rows.to(DEV), out=out, workspace=ws)
        assert torch.equal(out.cpu(), whole)


def test_rows_shorter_than_a_piece_and_of_many_columns():
    for d in (1, 3, 2048 + 8, 8192):
        x, slots, start = _case([30, 200, 9, 301, 4], d, torch.float32, seed=d)
        part = start[1:5]
        ws = torch.full((B.nd_rows_group_sum_workspace_bytes(slots.numel(), d),), 0xFF, dtype=torch.uint8, device=DEV)
        print(f"[slices] d={d}", flush=True)
        got = B.nd_rows_group_sum(x.to(DEV), slots.to(DEV), part.to(DEV), 1, workspace=ws)
        assert torch.equal(got.cpu(), _want(x, slots, part, torch.float32))


def test_live_counts_with_a_first_offset():
    """As many pairs and groups as the device says, from the middle on."""
    d = 16
    x, slots, start = _case([50, 60, 70, 80], d, torch.float32, seed=2)
    part = start[1:5].clone()
    counts = torch.tensor([200, 3], dtype=torch.int64, device=DEV)  # 20 of the last group's pairs
    out = torch.full((3, d), float("nan"), device=DEV)
    ws = torch.full((B.nd_rows_group_sum_workspace_bytes(slots.numel(), d),), 0xFF, dtype=torch.uint8, device=DEV)
    B.nd_rows_group_sum(x.to(DEV), slots.to(DEV), part.to(DEV), 1, counts=counts, out=out, workspace=ws)
    part[-1] = 200
    assert torch.equal(out.cpu(), _want(x, slots, part, torch.float32))
    # offsets that begin behind the live pairs: groups without pairs
    counts[0] = 40
    out.fill_(float("nan"))
    ws.fill_(0xFF)
    B.nd_rows_group_sum(x.to(DEV), slots.to(DEV), part.to(DEV), 1, counts=counts, out=out, workspace=ws)
    assert not bool(out.any())
