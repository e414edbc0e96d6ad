"""Rows in the order of the transit groups, back with weights, summed per group, and the weights' gradient, against plain
64-bit forms."""
import numpy as np
import pytest
import torch

from paper_2009_06693_amd import binding as B
from paper_2009_06693_amd import inputs

from rows_util import TYPES, U32, Loss, assert_within, group_sums, groups_of, half_step, rounded, weighted_rows

pytestmark = pytest.mark.gpu
DEV = "cuda:0"

# rows, slots per row, keys, numbers per row
SHAPES = [(1, 1, 1, 1), (1, 1, 1, 128), (3, 2, 4, 7), (64, 2, 8, 128), (100, 3, 5, 33), (257, 10, 1000, 100), (1000, 1, 3, 64),
          (31, 40, 6, 1024), (5, 7, 9, 8192), (40, 25, 2000, 2047), (2000, 4, 1, 16), (700, 9, 300, 256)]


def _inputs(n, m, V, d, dtype, seed, null=0.1):
    g = torch.Generator().manual_seed(seed)
    keys = (torch.rand(n * m, generator=g).pow(2) * V).int().clamp(max=V - 1)
    keys[torch.rand(n * m, generator=g) < null] = -1
    return (torch.randn(n, d, generator=g).to(dtype), keys, torch.rand(n * m, generator=g) - 0.3,
            torch.randn(n, d, generator=g).to(dtype), g)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("n,m,V,d", SHAPES)
def test_there_and_back(n, m, V, d, kind):
    dtype = TYPES[kind]
    x, keys, weights, dy, g = _inputs(n, m, V, d, dtype, seed=n + d)
    slots, _, _ = groups_of(keys, V)
    print(f"[rows] n={n} m={m} V={V} d={d} {kind} pairs={slots.numel()}", flush=True)
    sd, wd = slots.to(DEV), weights.to(DEV)
    place = B.nd_group_positions(sd, n * m)
    want = torch.full((n * m,), -1, dtype=torch.int32)
    want[slots.long()] = torch.arange(slots.numel(), dtype=torch.int32)
    assert torch.equal(place.cpu(), want)
    parents = slots.long() // m
    assert torch.equal(B.nd_rows_by_transit(x.to(DEV), sd, m).cpu(), x[parents])
    exact = x.double()[parents] * weights.double()[slots.long()][:, None]
    assert_within(B.nd_rows_by_transit(x.to(DEV), sd, m, wd), exact, rounded(exact, exact.abs() * U32, dtype), "weighted")
    z = torch.randn(slots.numel(), d, generator=g).to(dtype)
    for f in (None, weights):
        sums, sizes = weighted_rows(z, want, f, n, m)
        got = B.nd_rows_to_samples(z.to(DEV), place, m, None if f is None else wd)
        assert_within(got, sums, rounded(sums, (m + 1) * U32 * sizes, dtype), "back")
    dots = torch.zeros(n * m, dtype=torch.float64)
    sizes = torch.zeros(n * m, dtype=torch.float64)
    dots[slots.long()] = (dy.double()[parents] * z.double()).sum(1)
    sizes[slots.long()] = (dy.double()[parents] * z.double()).abs().sum(1)
    assert_within(B.nd_rows_weight_grad(dy.to(DEV), z.to(DEV), place, m), dots, (d + 2) * U32 * sizes, "weights' gradient")


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("n,m,V,d", SHAPES)
def test_sums_over_sampled_vertices_and_their_gradient(n, m, V, d, kind):
    dtype = TYPES[kind]
    dy, vertices, weights, _, g = _inputs(n, m, V, d, dtype, seed=3 * n + d)
    table = torch.randn(V, d, generator=g).to(dtype)
    slots, ids, start = groups_of(vertices, V)
    print(f"[rows] table n={n} m={m} V={V} d={d} {kind}", flush=True)
    vd, wd = vertices.to(DEV), weights.to(DEV)
    sums, sizes = weighted_rows(table, vertices, weights, n, m)
    assert_within(B.nd_rows_to_samples(table.to(DEV), vd, m, wd), sums, rounded(sums, (m + 1) * U32 * sizes, dtype))
    places = vertices.long()
    live = places >= 0
    rows = dy.double().repeat_interleave(m, 0)
    prod = torch.where(live[:, None], rows * table.double()[places.clamp(min=0)], 0.0)
    assert_within(B.nd_rows_weight_grad(dy.to(DEV), table.to(DEV), vd, m), prod.sum(1), (d + 2) * U32 * prod.abs().sum(1))
    args = (dy.to(DEV), slots.to(DEV), start.to(DEV), m)
    for f, fd in ((weights, wd), (None, None)):
        sums, sizes = group_sums(dy, slots, start, f, m)
        terms = (start[1:] - start[:-1]).double()[:, None] + 3
        tol = rounded(sums, terms * U32 * sizes, dtype)
        assert_within(B.nd_rows_group_sum(*args, fd), sums, tol, "sums")
        whole, allowed = torch.zeros(V, d, dtype=torch.float64), torch.zeros(V, d, dtype=torch.float64)
        whole[ids.long()], allowed[ids.long()] = sums, tol
        out = torch.full((V, d), float("nan"), dtype=dtype, device=DEV)
        assert_within(B.nd_rows_group_sum(*args, fd, group_rows=ids.to(DEV), out=out), whole, allowed, "table")


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("n,m,d", [(1, 65536, 128), (2, 1000, 5), (3, 9, 2056), (1, 8, 64), (65, 17, 200), (16500, 12, 128),
                                   (140000, 9, 3)])
def test_slots_of_few_rows_and_of_many(n, m, d, kind):
    dtype = TYPES[kind]
    g = torch.Generator().manual_seed(n + m)
    V = 97
    table, dy = torch.randn(V, d, generator=g).to(dtype).to(DEV), torch.randn(n, d, generator=g).to(dtype).to(DEV)
    index = torch.randint(-1, V + 1, (n * m,), generator=g).int().to(DEV)
    weights = (torch.rand(n * m, generator=g) - 0.3).to(DEV)
    print(f"[rows] slots n={n} m={m} d={d} {kind}", flush=True)
    # sums over the slots of equal vertices first: 64-bit weights per row and vertex
    live = (index >= 0) & (index < V)
    at = torch.arange(n * m, device=DEV) // m * V + index.long().clamp(0, V - 1)
    for w in (weights, None):
        f = (torch.ones_like(weights) if w is None else weights).double() * live
        per = torch.zeros(n * V, dtype=torch.float64, device=DEV).index_add_(0, at, f).view(n, V)
        size = torch.zeros(n * V, dtype=torch.float64, device=DEV).index_add_(0, at, f.abs()).view(n, V)
        want, sizes = per @ table.double(), size @ table.double().abs()
        got = B.nd_rows_to_samples(table, index, m, w)
        assert_within(got, want, rounded(want, (m + 1) * U32 * sizes, dtype), "sums")
    dots, sizes = dy.double() @ table.double().T, dy.double().abs() @ table.double().abs().T
    want, allowed = dots.view(-1)[at] * live, (d + 2) * U32 * sizes.view(-1)[at]
    assert_within(B.nd_rows_weight_grad(dy, table, index, m), want, allowed, "weights' gradient")


@pytest.mark.parametrize("sizes", [[1], [64], [65], [63, 1], [64, 64], [1, 63, 1, 128, 5], [0, 3, 0, 0, 200, 0], [1000, 1], [1] * 300,
                                   [129] * 20, [20000, 7], [5, 70000]])
def test_groups_that_end_inside_and_across_tiles(sizes):
    """Whole numbers: every sum is exact, whatever its order."""
    d = 24
    P = sum(sizes)
    start = torch.tensor([0] + list(np.cumsum(sizes)), dtype=torch.int32)
    g = torch.Generator().manual_seed(P)
    x = torch.randint(-8, 9, (P, d), generator=g).float()
    slots = torch.randperm(P, generator=g).int()
    want, _ = group_sums(x, slots, start, None, 1)
    print(f"[rows] groups of {sizes[:6]}", flush=True)
    got = B.nd_rows_group_sum(x.to(DEV), slots.to(DEV), start.to(DEV), 1)
    assert torch.equal(got.cpu().double(), want)
    rows = torch.arange(len(sizes), dtype=torch.int32) * 3 + 2
    whole = torch.zeros(3 * len(sizes) + 4, d, dtype=torch.float64)
    whole[rows.long()] = want
    got = B.nd_rows_group_sum(x.to(DEV), slots.to(DEV), start.to(DEV), 1, group_rows=rows.to(DEV), num_rows=whole.shape[0])
    assert torch.equal(got.cpu().double(), whole)


@pytest.mark.parametrize("kind", list(TYPES))
def test_rows_at_strides_and_odd_addresses(kind):
    n, m, V, d = 90, 3, 40, 52
    dtype = TYPES[kind]
    x, keys, weights, dy, g = _inputs(n, m, V, d, dtype, seed=2)
    slots, ids, start = groups_of(keys, V)
    z = torch.randn(slots.numel(), d, generator=g).to(dtype)

    def placed(rows, pad=5, shift=3):
        big = torch.full((rows.shape[0] * (d + pad) + shift,), float("nan"), dtype=dtype, device=DEV)
        view = torch.as_strided(big, rows.shape, (d + pad, 1), shift)
        view.copy_(rows)
        return view

    sd, wd = slots.to(DEV), weights.to(DEV)
    place = B.nd_group_positions(sd, n * m)

    def same(call, rows, out):
        a = call(*(t.to(DEV) for t in rows), None)
        v = placed(torch.zeros(out))
        base = v._base if v._base is not None else v
        call(*(placed(t) for t in rows), v)
        assert torch.equal(v, a)
        assert int(base.isnan().sum()) == base.numel() - v.numel()
    same(lambda t, o: B.nd_rows_by_transit(t, sd, m, wd, out=o), [x], (slots.numel(), d))
    same(lambda t, o: B.nd_rows_to_samples(t, place, m, wd, out=o), [z], (n, d))
    same(lambda t, o: B.nd_rows_group_sum(t, sd, start.to(DEV), m, wd, out=o), [dy], (ids.numel(), d))
    assert torch.equal(B.nd_rows_weight_grad(placed(dy), placed(z), place, m),
                       B.nd_rows_weight_grad(dy.to(DEV), z.to(DEV), place, m))


@pytest.mark.parametrize("kind", list(TYPES))
def test_what_lies_behind_the_live_pairs_is_left(kind):
    """Counts on the device, as nd_group_by_transit leaves them: rows behind them are neither read as pairs nor written."""
    n, m, V, d = 50, 4, 30, 40
    dtype = TYPES[kind]
    x, keys, weights, _, _ = _inputs(n, m, V, d, dtype, seed=4, null=0.4)
    slots, ids, start = groups_of(keys, V)
    P, U = slots.numel(), ids.numel()
    full = torch.full((n * m,), 7, dtype=torch.int32)
    full[:P] = slots
    starts = torch.full((n * m + 1,), -3, dtype=torch.int32)
    starts[:U + 1] = start
    counts = torch.tensor([P, U], dtype=torch.int64, device=DEV)
    fd = full.to(DEV)
    place = B.nd_group_positions(fd, n * m, counts)
    assert torch.equal(place, B.nd_group_positions(slots.to(DEV), n * m))
    out = torch.full((n * m, d), float("nan"), dtype=dtype, device=DEV)
    B.nd_rows_by_transit(x.to(DEV), fd, m, counts=counts, out=out)
    assert torch.equal(out[:P].cpu(), x[slots.long() // m]) and bool(out[P:].isnan().all())
    out = torch.full((n * m, d), float("nan"), dtype=dtype, device=DEV)
    B.nd_rows_group_sum(x.to(DEV), fd, starts.to(DEV), m, weights.to(DEV), counts=counts, out=out)
    assert torch.equal(out[:U], B.nd_rows_group_sum(x.to(DEV), slots.to(DEV), start.to(DEV), m, weights.to(DEV)))
    assert bool(out[U:].isnan().all())


def test_places_and_slots_out_of_range_count_nothing():
    z = torch.full((4, 16), float("nan"), device=DEV)
    z[1] = 2.0
    index = torch.tensor([1, -1, 4, -7, 2 ** 31 - 1, 1], dtype=torch.int32, device=DEV)
    weights = torch.tensor([1.0, float("inf"), float("nan"), 1.0, 1.0, 0.5], device=DEV)
    out = B.nd_rows_to_samples(z, index, 3, weights)
    assert torch.equal(out[0], torch.full((16,), 2.0, device=DEV)) and torch.equal(out[1], torch.full((16,), 1.0, device=DEV))
    dw = B.nd_rows_weight_grad(torch.ones(2, 16, device=DEV), z, index, 3)
    assert dw.tolist() == [32.0, 0.0, 0.0, 0.0, 0.0, 32.0]
    slots = torch.tensor([5, 6, -1, 0], dtype=torch.int32, device=DEV)  # of two rows with three slots each
    x = torch.ones(2, 16, device=DEV)
    assert B.nd_rows_by_transit(x, slots, 3).sum(1).tolist() == [16.0, 0.0, 0.0, 16.0]
    start = torch.tensor([0, 3, 4], dtype=torch.int32, device=DEV)
    assert B.nd_rows_group_sum(x, slots, start, 3).sum(1).tolist() == [16.0, 16.0]
    assert B.nd_group_positions(slots, 6).tolist() == [3, -1, -1, -1, -1, 0]


def test_nothing_to_do():
    none = torch.empty(0, dtype=torch.int32, device=DEV)
    x = torch.ones(3, 16, device=DEV)
    assert B.nd_group_positions(none, 4).tolist() == [-1] * 4
    assert B.nd_group_positions(none, 0).numel() == 0
    assert B.nd_rows_by_transit(x, none, 2).shape == (0, 16)
    assert B.nd_rows_to_samples(x, none, 2).shape == (0, 16)
    assert B.nd_rows_weight_grad(x[:0], x, none, 2).numel() == 0
    # no row to bring back: zeros
    assert not bool(B.nd_rows_to_samples(x[:0], torch.full((4,), -1, dtype=torch.int32, device=DEV), 2).any())
    start = torch.zeros(1, dtype=torch.int32, device=DEV)
    assert B.nd_rows_group_sum(x, none, start, 2).shape == (0, 16)
    assert not bool(B.nd_rows_group_sum(x, none, torch.zeros(4, dtype=torch.int32, device=DEV), 2).any())
    whole = torch.full((5, 16), 9.0, device=DEV)
    B.nd_rows_group_sum(x, none, start, 2, group_rows=none, out=whole)
    assert not bool(whole.any())


def test_replays_of_a_graph_and_another_stream():
    n, m, V, d = 300, 5, 60, 128
    x, keys, weights, dy, _ = _inputs(n, m, V, d, torch.bfloat16, seed=6)
    slots, ids, start = groups_of(keys, V)
    x, weights, dy, slots, ids, start = (t.to(DEV) for t in (x, weights, dy, slots, ids, start))

    def both(stream=None):
        place = B.nd_group_positions(slots, n * m, stream=stream)
        xs = B.nd_rows_by_transit(x, slots, m, stream=stream)
        return [place, xs, B.nd_rows_to_samples(xs, place, m, weights, stream=stream),
                B.nd_rows_weight_grad(dy, xs, place, m, stream=stream),
                B.nd_rows_group_sum(dy, slots, start, m, weights, group_rows=ids, num_rows=V, stream=stream)]
    want = [t.clone() for t in both()]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both()
    for _ in range(3):
        for t in got:
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        both()
        torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = both(side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_more_workgroups_than_a_launch_is_given():
    """Rows of one piece each, more of them than one round of the largest launch takes."""
    n, d = (1 << 20) * 256 + 1000, 8            # 16 bytes per row: 256 rows per workgroup
    x = torch.arange(d, device=DEV).to(torch.bfloat16).repeat(4, 1) + torch.arange(4, device=DEV).to(torch.bfloat16)[:, None]
    index = (torch.arange(n, device=DEV, dtype=torch.int32) * 5) % 4
    print(f"[rows] {n} rows", flush=True)

    def is_right(rows):  # a part at a time: torch's own indexing fails on more
        step = 1 << 22
        return all(torch.equal(rows[a:a + step], x[index[a:a + step].long()]) for a in range(0, n, step))
    out = B.nd_rows_to_samples(x, index, 1)
    assert is_right(out)
    assert torch.equal(B.nd_rows_weight_grad(out, x, index, 1)[-3000:], (out[-3000:].float() ** 2).sum(1))
    del out
    assert is_right(B.nd_rows_by_transit(x, (index * 3 + 2).clamp(max=11), 3))


def test_a_step_of_walk_embeddings_as_it_is_made():
    """Walks, their centres' rows, the loss of the next vertices, and both gradients on the table, against the formulas."""
    g = inputs.small_graph(10, 12000, seed=11)
    dg = B.nd_graph_create(g.row_offsets, g.col_indices)
    s = B.Sampler(dg, B.ND_PPR, B.nd_params_init(num_steps=8, term_prob=0.1), g.V)
    steps = s.run(torch.arange(g.V, dtype=torch.int32, device=DEV), 21)
    centres, labels = steps[1], torch.stack([steps[0], steps[2], steps[3]], dim=1).contiguous()
    V, d = g.V, 64
    gen = torch.Generator().manual_seed(8)
    table, contexts = ((torch.randn(V, d, generator=gen) * 0.5).to(DEV) for _ in range(2))
    weight = torch.full((V,), 1.0 / (3 * V), device=DEV)
    # ended walks have no centre: their contexts do not count
    labels[centres < 0] = -1
    rows = B.nd_rows_to_samples(table, centres, 1)
    loss, lse, drows, dcontexts = B.SoftmaxLoss(V, V, d, 3, torch.float32, grad=True).grad(rows, contexts, labels, weight)
    st, slots, ids, start, P, U = B.nd_group_by_transit(centres, V)
    dtable = B.nd_rows_group_sum(drows, slots, start, 1, group_rows=ids, num_rows=V)
    c = centres.cpu().long()
    assert bool((c < 0).any()) and torch.equal(rows.cpu(), torch.where((c >= 0)[:, None], table.cpu()[c.clamp(min=0)], 0.0))
    want = Loss(rows.cpu(), contexts.cpu(), labels.cpu(), weight.cpu())
    want.check(loss, lse, drows, dcontexts)
    live = c >= 0
    whole = torch.zeros(V, d, dtype=torch.float64).index_add(0, c[live], want.dx[live])
    size = torch.zeros(V, d, dtype=torch.float64).index_add(0, c[live], want.dx[live].abs())
    allowed = torch.zeros(V, d, dtype=torch.float64).index_add(0, c[live], want.dx_tol[live])
    held = torch.bincount(c[live], minlength=V).double()[:, None]
    assert_within(dtable, whole, allowed * (1 + V * U32) + (held + 3) * U32 * size + whole.abs() * half_step(torch.float32))


def test_an_aggregator_over_sampled_neighbours_with_keys():
    """k-hop neighbours under three types: rows in type order, a product per type, the weighted mean back, all gradients."""
    g = inputs.small_graph(10, 12000, seed=11)
    dg = B.nd_graph_create(g.row_offsets, g.col_indices)
    m, types, d = 6, 3, 32
    s = B.Sampler(dg, B.ND_KHOP, B.nd_params_init(num_steps=1, fanout=[m]), 200)
    hop = s.run(torch.arange(200, dtype=torch.int32, device=DEV), 5)[0]
    keys = torch.where(hop >= 0, hop % types, -1)
    st, slots, ids, start, P, U = B.nd_group_by_transit(keys, types)
    gen = torch.Generator().manual_seed(3)
    features = torch.randn(200, d, generator=gen)
    mats = torch.randn(types, d, d, generator=gen) / d ** 0.5
    weights = torch.rand(200 * m, generator=gen)
    dy = torch.randn(200, d, generator=gen)
    # the plain form with torch's own gradients, in 64 bits
    f64, w64 = features.double().requires_grad_(), weights.double().requires_grad_()
    k = keys.cpu().view(200, m)
    per = torch.stack([f64 @ mats[t].double() for t in range(types)])
    y = sum(torch.where((k[:, j] >= 0)[:, None], w64.view(200, m)[:, j, None] * per[k[:, j].clamp(min=0), torch.arange(200)], 0.0)
            for j in range(m))
    y.backward(dy.double())
    # as the calls make it
    place = B.nd_group_positions(slots, 200 * m)
    xs = B.nd_rows_by_transit(features.to(DEV), slots, m)
    z = torch.empty_like(xs)
    for i in range(U):
        z[start[i]:start[i + 1]] = xs[start[i]:start[i + 1]] @ mats[int(ids[i])].to(DEV)
    out = B.nd_rows_to_samples(z, place, m, weights.to(DEV))
    dz = B.nd_rows_by_transit(dy.to(DEV), slots, m, weights.to(DEV))
    dxs = torch.empty_like(dz)
    for i in range(U):
        dxs[start[i]:start[i + 1]] = dz[start[i]:start[i + 1]] @ mats[int(ids[i])].to(DEV).T.contiguous()
    dx = B.nd_rows_to_samples(dxs, place, m)
    dw = B.nd_rows_weight_grad(dy.to(DEV), z, place, m)
    # products of 32 numbers of size 1 in fp32 (library), then sums of 6 or of 32: below 100 terms of size 10 in all
    tol = 100 * 10 * U32
    for a, b in ((out, y.detach()), (dx, f64.grad), (dw, w64.grad)):
        assert float((a.cpu().double() - b).abs().max()) <= tol * 4


def test_refusals():
    x = torch.zeros(4, 8, device=DEV)
    slots = torch.zeros(6, dtype=torch.int32, device=DEV)
    start = torch.tensor([0, 6], dtype=torch.int32, device=DEV)
    for call in (lambda: B.nd_rows_by_transit(x.double(), slots, 2), lambda: B.nd_rows_by_transit(x, slots.long(), 2),
                 lambda: B.nd_rows_by_transit(x.cpu(), slots, 2), lambda: B.nd_rows_by_transit(x, slots, 2, x.view(-1).half()),
                 lambda: B.nd_rows_to_samples(x, slots.float(), 2), lambda: B.nd_rows_to_samples(x[0], slots, 2),
                 lambda: B.nd_group_positions(slots, 6, counts=start), lambda: B.nd_group_positions(slots[::2], 6)):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: B.nd_rows_by_transit(x.t(), slots, 2), lambda: B.nd_rows_by_transit(x, slots, 2, x[0, :7]),
                 lambda: B.nd_rows_by_transit(x, slots, 2, out=x), lambda: B.nd_rows_to_samples(x, slots, 4),
                 lambda: B.nd_rows_to_samples(x, slots, 0), lambda: B.nd_rows_weight_grad(x, x, slots, 2),
                 lambda: B.nd_rows_weight_grad(x.half(), x, slots, 2),
                 lambda: B.nd_rows_group_sum(x, slots, start, 2, group_rows=slots),
                 lambda: B.nd_rows_group_sum(x, slots, start, 2, group_rows=slots[:0], num_rows=3),
                 lambda: B.nd_group_positions(slots, 6, out=slots[:5])):
        with pytest.raises(ValueError):
            call()
    for code, call in ((B.ND_ERR_BAD_ARGUMENT, lambda: B.nd_rows_by_transit(x, slots, 0)),
                       (B.ND_ERR_TOO_LARGE, lambda: B.nd_rows_by_transit(x, slots, 65537)),
                       (B.ND_ERR_TOO_LARGE, lambda: B.nd_rows_to_samples(torch.zeros(1, 8193, device=DEV), slots, 1)),
                       (B.ND_ERR_WORKSPACE, lambda: B.nd_rows_group_sum(x, slots, start, 2, workspace=slots))):
        with pytest.raises(B.NdError) as e:
            call()
        assert e.value.code == code
