"""The softmax loss over all vertices and its gradient against their formulas in 64 bits."""
import pytest
import torch

from paper_2009_06693_amd import binding as B

from rows_util import TYPES, U32, Loss, assert_within, half_step, rounded

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _inputs(n, V, d, k, dtype, seed, spread=2.0, empty=0.2):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(n, d, generator=g) * (spread / d ** 0.5)).to(dtype)
    w = torch.randn(V, d, generator=g).to(dtype)
    labels = torch.randint(0, V, (n, k), generator=g).int()
    labels[torch.rand(n, k, generator=g) < empty / 2] = -1
    labels[torch.rand(n, generator=g) < empty] = -1
    row_weight = (torch.rand(n, generator=g) + 0.5) / max(1, n)
    return x, w, labels, row_weight


def _run(x, w, labels, row_weight, grad=True):
    n, d = x.shape
    print(f"[loss] n={n} V={w.shape[0]} d={d} k={labels.shape[1]} {x.dtype} grad={grad}", flush=True)
    op = B.SoftmaxLoss(n, w.shape[0], d, labels.shape[1], x.dtype, grad=grad)
    op.workspace.fill_(0xFF)  # nothing is taken from what lies there
    for t in (op._loss, op._lse, op._dx, op._dw):
        if t is not None:
            t.fill_(float("nan"))
    out = op.grad(x, w, labels, row_weight) if grad else op.loss(x, w, labels)
    torch.cuda.synchronize()
    op.status()
    return out


SHAPES = [(1, 1, 1, 1), (1, 2, 3, 1), (3, 5, 8, 2), (1, 4096, 64, 1), (5, 57, 100, 3), (127, 129, 65, 2), (128, 128, 64, 1),
          (129, 1000, 128, 10), (300, 3001, 96, 4), (256, 5000, 256, 1), (33, 700, 257, 2), (40, 300, 1000, 1),
          (260, 2000, 512, 5), (2, 300, 8192, 1), (1000, 130, 40, 64), (700, 260, 192, 3), (17, 40000, 128, 1),
          (1500, 33, 16, 1)]


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("n,V,d,k", SHAPES)
def test_against_the_formulas(n, V, d, k, kind):
    x, w, labels, row_weight = _inputs(n, V, d, k, TYPES[kind], seed=n + V + d)
    want = Loss(x, w, labels, row_weight)
    args = [t.to(DEV) for t in (x, w, labels, row_weight)]
    want.check(*_run(*args), what="gradient call")
    want.check(*_run(*args, grad=False), what="forward call")


@pytest.mark.parametrize("kind", list(TYPES))
def test_vertices_in_several_pieces(kind):
    """More probabilities than lie in memory at a time."""
    n, V, d = 4100, 70000, 24
    x, w, labels, row_weight = (t.to(DEV) for t in _inputs(n, V, d, 2, TYPES[kind], seed=3))
    out = _run(x, w, labels, row_weight)
    Loss(x, w, labels, row_weight).check(*out)


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("d", [128, 300, 520])
def test_labels_are_not_rounded_with_the_vertices(kind, d):
    """Equal scores: every vertex weighs 1 / V and the label almost 1.  What is rounded to 16 bits before the products is a
    vertex's weight, off by u of itself, so that dx is off by u times the mean row's size next to its own rounding."""
    n, V, dtype = 70, 2500, TYPES[kind]
    g = torch.Generator().manual_seed(d)
    w = torch.randn(V, d, generator=g).to(dtype)
    labels = torch.randint(0, V, (n, 1), generator=g).int()
    row_weight = torch.rand(n, generator=g) + 0.1
    _, _, dx, _ = _run(torch.zeros(n, d, dtype=dtype, device=DEV), w.to(DEV), labels.to(DEV), row_weight.to(DEV))
    wd, gd = w.double(), row_weight.double()[:, None]
    want = gd * (wd.mean(0) - wd[labels[:, 0].long()])
    size = gd * wd.abs().mean(0)
    off = half_step(dtype) * size + (V + 16) * U32 * (size + want.abs())
    assert_within(dx, want, rounded(want, off, dtype), "dx")


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("n,V,d,k", [(4100, 70000, 260, 3), (1030, 50001, 520, 1), (1500, 40001, 33, 64), (127, 3001, 1030, 4)])
def test_scores_that_are_kept_and_made_again(n, V, d, k, kind):
    """Long rows: scores are kept between the two passes; shorter ones: made again, here in pieces."""
    x, w, labels, row_weight = (t.to(DEV) for t in _inputs(n, V, d, k, TYPES[kind], seed=d))
    out = _run(x, w, labels, row_weight)
    Loss(x, w, labels, row_weight).check(*out)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("d", [64, 72, 320])
def test_rows_at_strides_and_odd_addresses(kind, d):
    n, V, k = 150, 333, 2
    x, w, labels, row_weight = _inputs(n, V, d, k, TYPES[kind], seed=5)
    want = Loss(x, w, labels, row_weight)
    for pad, shift in ((8, 0), (1, 0), (16, 3)):
        def placed(rows):
            big = torch.full((rows.shape[0] * (d + pad) + shift,), float("nan"), dtype=rows.dtype, device=DEV)
            view = torch.as_strided(big, (rows.shape[0], d), (d + pad, 1), shift)
            view.copy_(rows)
            return big, view
        (_, xv), (_, wv) = placed(x), placed(w)
        (dxb, dx), (dwb, dw) = placed(torch.zeros_like(x)), placed(torch.zeros_like(w))
        loss, lse = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
        ws = torch.empty(B.nd_softmax_loss_workspace_bytes(n, V, d, k, x.dtype, True), dtype=torch.uint8, device=DEV)
        print(f"[loss] stride {d + pad} from {shift}, {kind}", flush=True)
        B.nd_softmax_loss_grad(xv, wv, labels.to(DEV), row_weight.to(DEV), loss, lse, dx, dw, ws)
        want.check(loss, lse, dx, dw, f"stride {d + pad} from {shift}")
        for big, rows in ((dxb, n), (dwb, V)):   # what lies between the rows is left alone
            gaps = torch.ones_like(big, dtype=torch.bool)
            torch.as_strided(gaps, (rows, d), (d + pad, 1), shift).fill_(False)
            assert bool(big[gaps].isnan().all())


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("d", [128, 300])
def test_rows_without_labels_are_left_out(kind, d):
    """Infinities and NaN in them reach nothing, and their outputs are zero."""
    n, V, k = 200, 500, 3
    x, w, labels, row_weight = _inputs(n, V, d, k, TYPES[kind], seed=7)
    dead = torch.arange(n) % 3 == 0
    labels[dead] = -1
    labels[~dead, 0] = 4
    labels[6] = torch.tensor([-5, -(2 ** 31), -1])  # any negative number is NULL
    x[0], x[3], x[6] = float("nan"), float("inf"), torch.finfo(x.dtype).min
    row_weight[0] = float("nan")
    clean = x.clone()
    clean[dead] = 0
    rw = torch.where(dead, 0.0, row_weight)
    out = _run(x.to(DEV), w.to(DEV), labels.to(DEV), row_weight.to(DEV))
    Loss(clean, w, labels, rw).check(*out)
    assert not out[0][dead].any() and not out[1][dead].any() and not out[2][dead].any()
    # none at all
    labels[:] = -1
    out = _run(x.to(DEV), w.to(DEV), labels.to(DEV), row_weight.to(DEV))
    assert not any(bool(t.any()) for t in out)


@pytest.mark.parametrize("kind", list(TYPES))
def test_no_rows(kind):
    w = torch.randn(300, 64, device=DEV).to(TYPES[kind])
    out = _run(w[:0], w, torch.empty((0, 2), dtype=torch.int32, device=DEV), None)
    assert out[0].numel() == 0 and out[3].shape == (300, 64) and not bool(out[3].any())


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("spread", [0.0, 40.0, 300.0])
def test_flat_and_peaked_distributions(kind, spread):
    """All products alike, and products whose exponentials leave fp32 on both sides."""
    x, w, labels, row_weight = _inputs(140, 900, 128, 2, TYPES[kind], seed=11, spread=spread)
    Loss(x, w, labels, row_weight).check(*_run(*(t.to(DEV) for t in (x, w, labels, row_weight))))


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
def test_infinities_and_nan_stay_in_their_rows(kind, value):
    """A row that counts and holds one has no finite loss; the other rows' outputs are as without it."""
    n, V, d = 70, 400, 128
    x, w, labels, row_weight = _inputs(n, V, d, 1, TYPES[kind], seed=13, empty=0.0)
    x[5, 3] = value
    loss, lse, dx, _ = _run(*(t.to(DEV) for t in (x, w, labels, row_weight)))
    assert not bool(loss[5].isfinite())
    keep = torch.arange(n) != 5
    want = Loss(x[keep], w, labels[keep], row_weight[keep])
    want.check(loss[keep], lse[keep], dx[keep])


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("value", [float("inf"), float("nan")])
def test_infinities_and_nan_of_long_rows_stay_there(kind, value):
    for d in (300, 520):
        x, w, labels, row_weight = _inputs(140, 400, d, 1, TYPES[kind], seed=d, empty=0.0)
        x[5, 3] = value
        loss, lse, dx, _ = _run(*(t.to(DEV) for t in (x, w, labels, row_weight)))
        assert not bool(loss[5].isfinite())
        keep = torch.arange(140) != 5
        Loss(x[keep], w, labels[keep], row_weight[keep]).check(loss[keep], lse[keep], dx[keep])


def test_weights_of_rows():
    """None counts as one; zeros give zero gradients; very different ones keep the small rows' gradients."""
    for kind, dtype in TYPES.items():
        x, w, labels, row_weight = _inputs(90, 300, 128, 2, dtype, seed=17)
        args = [t.to(DEV) for t in (x, w, labels)]
        Loss(x, w, labels).check(*_run(*args, None), what=f"{kind} none")
        out = _run(*args, torch.zeros(90, device=DEV))
        assert not bool(out[2].any()) and not bool(out[3].any())
        row_weight[::2] *= -1000
        Loss(x, w, labels, row_weight).check(*_run(*args, row_weight.to(DEV)), what=f"{kind} mixed")


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("d", [64, 300])
@pytest.mark.parametrize("n", [60, 300])
@pytest.mark.parametrize("value", [float("inf"), float("nan")])
def test_a_weight_that_is_not_finite_leaves_other_rows_alone(kind, d, n, value):
    x, w, labels, row_weight = (t.to(DEV) for t in _inputs(n, 700, d, 2, TYPES[kind], seed=n))
    labels[5, 0] = 3
    row_weight[:] = 1e-4
    want = _run(x, w, labels, row_weight)[2].clone()
    row_weight[5] = value
    got = _run(x, w, labels, row_weight)[2]
    others = torch.arange(n, device=DEV) != 5
    assert torch.equal(got[others], want[others])
    assert not bool(got[5].isfinite().any())


def test_only_the_gradients_that_are_asked_for():
    x, w, labels, row_weight = (t.to(DEV) for t in _inputs(200, 700, 128, 2, torch.bfloat16, seed=19))
    loss, lse, dx, dw = _run(x, w, labels, row_weight)
    ws = torch.empty(B.nd_softmax_loss_workspace_bytes(200, 700, 128, 2, x.dtype, True), dtype=torch.uint8, device=DEV)
    for a, b in ((torch.empty_like(dx), None), (None, torch.empty_like(dw)), (None, None)):
        l2, e2 = torch.empty_like(loss), torch.empty_like(lse)
        B.nd_softmax_loss_grad(x, w, labels, row_weight, l2, e2, a, b, ws)
        assert torch.equal(l2, loss) and torch.equal(e2, lse)
        assert (a is None or torch.equal(a, dx)) and (b is None or torch.equal(b, dw))


def test_labels_that_are_no_vertices_are_null_and_reported():
    x, w, labels, row_weight = _inputs(150, 256, 128, 3, torch.bfloat16, seed=23)
    labels[7, 1], labels[149, 2], labels[20] = 256, 2 ** 31 - 1, 300
    op = B.SoftmaxLoss(150, 256, 128, 3, torch.bfloat16, grad=True)
    out = op.grad(*(t.to(DEV) for t in (x, w, labels, row_weight)))
    Loss(x, w, labels, row_weight).check(*out)
    with pytest.raises(B.NdError) as e:
        op.status()
    assert e.value.code == B.ND_ERR_BAD_ROOT
    op.grad(*(t.to(DEV) for t in (x, w, labels.clamp(max=255), row_weight)))
    op.status()  # of the last call


@pytest.mark.parametrize("kind", list(TYPES))
def test_equal_inputs_give_equal_bits(kind):
    args = [t.to(DEV) for t in _inputs(3000, 5000, 128, 4, TYPES[kind], seed=29)]
    first = [t.clone() for t in _run(*args)]
    for a, b in zip(first, _run(*args)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("kind,d", [("bf16", 128), ("f16", 400), ("f32", 64)])
def test_replays_of_a_graph_and_two_streams(kind, d):
    args = [t.to(DEV) for t in _inputs(500, 3000, d, 2, TYPES[kind], seed=31)]
    n, V = 500, 3000
    a, b = (B.SoftmaxLoss(n, V, d, 2, TYPES[kind], grad=True) for _ in range(2))
    want = [t.clone() for t in a.grad(*args)]
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        got = a.grad(*args)
    other = [t.to(DEV) for t in _inputs(500, 3000, d, 2, TYPES[kind], seed=37)]
    for _ in range(3):
        for t in got:
            t.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want))
        b.grad(*other)
        torch.cuda.synchronize()
    want_b = [t.clone() for t in b.grad(*other)]
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        a.grad(*args, stream=s1)
        b.grad(*other, stream=s2)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(a.grad(*args), want))
    assert all(torch.equal(x, y) for x, y in zip(b.grad(*other), want_b))


@pytest.mark.parametrize("kind,n,d,grad", [("f16", 300, 520, True), ("f32", 300, 128, True), ("bf16", 3, 100, False),
                                           ("f32", 40, 60, False)])
def test_replays_over_long_and_few_rows(kind, n, d, grad):
    V = 3000
    args = [t.to(DEV) for t in _inputs(n, V, d, 2, TYPES[kind], seed=41)]
    op = B.SoftmaxLoss(n, V, d, 2, TYPES[kind], grad=grad)
    call = (lambda: op.grad(*args)) if grad else (lambda: op.loss(*args[:3]))
    want = [t.clone() for t in call()]
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        got = call()
    for _ in range(3):
        op.workspace.fill_(0xFF)
        for t in got:
            t.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want))
        assert all(torch.equal(x, y) for x, y in zip(call(), want))


def test_gradient_against_differences():
    """Directional derivatives of the weighted sum of losses, by differences of the formula in 64 bits."""
    x, w, labels, row_weight = _inputs(60, 200, 96, 3, torch.float32, seed=41)
    _, _, dx, dw = _run(*(t.to(DEV) for t in (x, w, labels, row_weight)))
    g = torch.Generator().manual_seed(1)

    def total(xd, wd):
        s = xd @ wd.T
        live = labels >= 0
        met = torch.where(live, s.gather(1, labels.clamp(min=0).long()), 0.0).sum(1)
        return float((row_weight.double() * (live.sum(1) * torch.logsumexp(s, 1) - met)).sum())

    h = 1e-4
    for which, grad in ((0, dx), (1, dw)):
        t = (x, w)[which].double()
        step = torch.randn(t.shape, generator=g, dtype=torch.float64)
        up, down = ((t + s * h * step) for s in (1, -1))
        slope = (total(up, w.double()) - total(down, w.double())) / (2 * h) if which == 0 else \
            (total(x.double(), up) - total(x.double(), down)) / (2 * h)
        got = float((grad.cpu().double() * step).sum())
        # the third derivative along a step of products' size 10 is below 10^3: h^2 / 6 of it; fp32 gradients
        assert abs(got - slope) <= 1e3 * h * h + 1e-4 * abs(slope) + 1e-6


def test_step_arrays_of_walks_are_labels():
    """The loss of next vertices along PPR walks, straight from nd_sample's arrays: ended walks are NULL."""
    from paper_2009_06693_amd import inputs
    g = inputs.small_graph(10, 12000, seed=11)
    dg = B.nd_graph_create(g.row_offsets, g.col_indices)
    roots = torch.arange(g.V, dtype=torch.int32, device=DEV)
    s = B.Sampler(dg, B.ND_PPR, B.nd_params_init(num_steps=6, term_prob=0.2), g.V)
    steps = s.run(roots, 9)
    table = (torch.randn(g.V, 64, generator=torch.Generator().manual_seed(2)) * 0.4).to(DEV)
    rows = B.nd_rows_to_samples(table, steps[2], 1)
    op = B.SoftmaxLoss(g.V, g.V, 64, 1, torch.float32, grad=True)
    out = op.grad(rows, table, steps[3])
    torch.cuda.synchronize()
    op.status()
    assert bool((steps[3] < 0).any())
    Loss(rows.cpu(), table.cpu(), steps[3].cpu()).check(*out)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("n", [1, 2, 3, 4, 5, 8, 9])
@pytest.mark.parametrize("V,d", [(1, 128), (63, 5), (4097, 128), (1000, 8), (70000, 60), (3000, 1024), (257, 1001), (100, 7)])
def test_few_rows_forward(n, V, d, kind):
    """Serving: one centre or a handful, over any number of vertices."""
    x, w, labels, _ = _inputs(n, V, d, 3, TYPES[kind], seed=n + V, empty=0.0)
    if n > 2:
        labels[1] = -1
        x[1] = float("nan")
    out = _run(x.to(DEV), w.to(DEV), labels.to(DEV), None, grad=False)
    Loss(x, w, labels).check(*out)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("d", [128, 300])
@pytest.mark.parametrize("n", [3, 200])
def test_vertices_that_scores_rule_out(n, d, kind):
    """Scores of the type's lowest values, or of minus infinity (forward), as programs mask vertices with: as if they were
    not there."""
    V = 700
    x, w, labels, row_weight = _inputs(n, V, d, 2, TYPES[kind], seed=43)
    x[:, 0] = 1.0
    out_of_it = torch.zeros(V, dtype=torch.bool)
    out_of_it[:300] = True
    labels = torch.where(labels >= 0, labels % 400 + 300, labels)
    kept = Loss(x, w[~out_of_it], torch.where(labels >= 0, labels - 300, labels), row_weight)
    low = torch.finfo(w.dtype).min if kind != "f16" else -30000.0
    for value, grad in ((low, True), (low, False), (float("-inf"), False)):
        masked = w.clone()
        masked[out_of_it] = 0
        masked[out_of_it, 0] = value
        out = _run(x.to(DEV), masked.to(DEV), labels.to(DEV), row_weight.to(DEV), grad)
        kept.check(*out[:2], what=f"{value}")
        if grad:
            kept.check(*out[:2], out[2], out[3][~out_of_it.to(DEV)], what=f"{value}")
            assert not bool(out[3][out_of_it.to(DEV)].any())


def test_refusals():
    x, w = torch.zeros(4, 8, device=DEV), torch.zeros(9, 8, device=DEV)
    labels, f = torch.zeros(4, 2, dtype=torch.int32, device=DEV), torch.zeros(4, device=DEV)
    ws = torch.empty(B.nd_softmax_loss_workspace_bytes(4, 9, 8, 2, torch.float32, True), dtype=torch.uint8, device=DEV)

    def call(x=x, w=w, labels=labels, loss=f, lse=f.clone(), ws=ws):
        B.nd_softmax_loss(x, w, labels, loss, lse, ws)
    call()
    for bad in (dict(x=x.cpu()), dict(x=x.double()), dict(x=x[0]), dict(labels=labels.long()), dict(labels=labels.cpu()),
                dict(loss=f.double()), dict(labels=labels.t().contiguous().t())):
        with pytest.raises(TypeError):
            call(**bad)
    for bad in (dict(w=w.half()), dict(w=torch.zeros(9, 7, device=DEV)), dict(x=torch.zeros(8, 4, device=DEV).t()),
                dict(x=x[:1].expand(4, 8)), dict(labels=labels[:3]), dict(loss=f[:3])):
        with pytest.raises(ValueError):
            call(**bad)
    with pytest.raises(B.NdError) as e:
        call(ws=ws[:300])
    assert e.value.code == B.ND_ERR_WORKSPACE
    with pytest.raises(B.NdError) as e:
        call(labels=torch.zeros(4, 65, dtype=torch.int32, device=DEV))
    assert e.value.code == B.ND_ERR_TOO_LARGE
