"""Cases of the operators that carry samples into training: the softmax loss over all vertices with its gradient, rows put
into the order of the transit groups and back with weights, and sums of rows per group.

`own` chooses between the plain form (elementary torch operations in 32 bits) and the library's calls.  A case is a dict
of plain values; `prepare` makes its inputs from a seed, `run` is one pass, `exact` the same outputs from the definitions
in 64 bits.
"""
import math

import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_BYTES = {"f32": 4, "bf16": 2, "f16": 2}
_DEVICE = "cuda:0"


# ----------------------------------------------------------------------------------------------------------- cases
# loss, loss_grad: n centre rows of d numbers against V vertices, k labels (contexts) per row, `ended` the share of rows
#   whose walk has ended (all labels NULL) and of labels that are NULL in the others.
# regroup, regroup_grad: n rows with m slots each under one of V keys, to the order of the groups and back with weights.
# neighbours, neighbours_grad: n rows, each the weighted sum of m sampled vertices' rows out of a table of V rows.
def listed():
    return [
        # one centre against a small graph's vertices: the smallest call, all latency (4,096 vertices: the R-MAT graph of scale 12)
        {"name": "loss_one_row", "op": "loss", "n": 1, "V": 4096, "d": 64, "k": 1, "type": "f32", "ended": 0.0},
        # the score of a handful of walk positions against 57,000 vertices, as in ranking the next vertex of a walk
        {"name": "loss_few_rows", "op": "loss", "n": 5, "V": 57000, "d": 128, "k": 1, "type": "bf16", "ended": 0.0},
        # evaluation of one step of every fourth walk, PPR walks of which a part has ended
        {"name": "loss_eval", "op": "loss", "n": 14250, "V": 57000, "d": 128, "k": 1, "type": "f16", "ended": 0.3},
        # an embedding in 32 bits of the small graph: all vertices are centres, windows of five to both sides
        {"name": "grad_small_f32", "op": "loss_grad", "n": 4096, "V": 4096, "d": 128, "k": 10, "type": "f32", "ended": 0.0},
        # the ordinary step: 8,192 centres of walks over 57,000 vertices
        {"name": "grad_walks", "op": "loss_grad", "n": 8192, "V": 57000, "d": 128, "k": 10, "type": "bf16", "ended": 0.1},
        # wide rows, as a model in front of the softmax gives them, and an odd number of them
        {"name": "grad_wide", "op": "loss_grad", "n": 2049, "V": 57000, "d": 1000, "k": 1, "type": "f16", "ended": 0.0},
        # the largest: 233,000 vertices
        {"name": "grad_large", "op": "loss_grad", "n": 8192, "V": 233000, "d": 256, "k": 10, "type": "bf16", "ended": 0.0},
        # one batch of rows for a few relation types, answered, not trained: the smallest of its kind
        {"name": "regroup_small", "op": "regroup", "n": 64, "V": 8, "d": 128, "m": 2, "type": "bf16", "ended": 0.0},
        # a training pass over wide rows under 64 keys, some slots without a key
        {"name": "regroup_train", "op": "regroup_grad", "n": 16385, "V": 64, "d": 1024, "m": 4, "type": "bf16", "ended": 0.05},
        # second hop of a k-hop [25,10] batch of 1,024 roots: ten neighbours' rows per parent, forward only
        {"name": "neighbours_batch", "op": "neighbours", "n": 25600, "V": 233000, "d": 100, "m": 10, "type": "f32", "ended": 0.02},
        # the same in training
        {"name": "neighbours_train", "op": "neighbours_grad", "n": 25600, "V": 233000, "d": 256, "m": 10, "type": "bf16", "ended": 0.02},
        # first hop with every vertex a root: 5.8 M rows are read
        {"name": "neighbours_all", "op": "neighbours_grad", "n": 233000, "V": 233000, "d": 128, "m": 25, "type": "bf16", "ended": 0.0},
    ]


def _spread(rng, low, high):
    """A whole number between low and high, spread over its logarithm."""
    return max(low, min(high, round(math.exp(rng.uniform(math.log(low), math.log(high))))))


def draw(rng):
    op = rng.choice(["loss", "loss_grad", "loss_grad", "regroup", "regroup_grad", "neighbours", "neighbours_grad"])
    case = {"op": op, "type": rng.choice(["f32", "bf16", "f16"]), "ended": rng.choice([0.0, 0.02, 0.3])}
    if op.startswith("loss"):
        case["k"] = rng.choice([1, 1, 4, 10])
        case["d"] = rng.choice([64, 128, 256, _spread(rng, 16, 1024)])
        case["V"] = _spread(rng, 256, 233000)
        # 32-bit products run at a fraction of the 16-bit rate: the same bound on their time
        room = (3.5e11 if case["type"] != "f32" else 3e10) / (case["V"] * case["d"])
        case["n"] = _spread(rng, 1, max(1, min(16384, int(room))))
    elif op.startswith("regroup"):
        case["m"] = rng.choice([1, 2, 4, 8])
        case["V"] = _spread(rng, 4, 4096)
        case["d"] = rng.choice([128, 1024, _spread(rng, 16, 2048)])
        case["n"] = _spread(rng, 16, max(16, int(6.6e7 / (case["m"] * case["d"]))))
    else:
        case["m"] = rng.choice([5, 10, 25, _spread(rng, 2, 40)])
        case["V"] = _spread(rng, 1000, 233000)
        case["d"] = rng.choice([64, 128, 256, _spread(rng, 16, 512)])
        case["n"] = _spread(rng, 64, max(64, int(1.5e8 / (case["m"] * case["d"]))))
    return case


def _dead_rows(case):
    return int(case["n"] * case["ended"])


def work(case):
    n, V, d, b = case["n"], case["V"], case["d"], _BYTES[case["type"]]
    op = case["op"]
    if op.startswith("loss"):
        live = n - _dead_rows(case)
        read = (live + V) * d * b + 4 * n * case["k"]
        if op == "loss":
            return {"bytes": read + 8 * n, "flops": 2.0 * live * V * d}
        return {"bytes": read + 4 * n + 8 * n + (n + V) * d * b, "flops": 8.0 * live * V * d}
    slots = n * case["m"]
    if op.startswith("regroup"):
        pairs = slots - _dead_slots(case)
        # rows in, pairs out; pairs in, rows out; order and places; weights
        once = (n + pairs) * d * b + 8 * pairs
        if op == "regroup":
            return {"bytes": 2 * once + 4 * slots, "flops": 2.0 * pairs * d}
        # gradients: the same two ways back, products of the incoming gradient with the pairs' rows for the weights
        return {"bytes": 4 * once + 8 * slots, "flops": 6.0 * pairs * d}
    pairs = slots - _dead_slots(case)
    touched = min(V, pairs)
    if op == "neighbours":
        return {"bytes": (touched + n) * d * b + 8 * slots, "flops": 2.0 * pairs * d}
    # table once forward and once for the weights' gradient; incoming gradient in, the table's gradient out
    return {"bytes": (touched + 2 * n + V) * d * b + 16 * slots + 4 * pairs, "flops": 6.0 * pairs * d}


def _dead_slots(case):
    return int(case["n"] * case["m"] * case["ended"])


# ---------------------------------------------------------------------------------------------------------- inputs
def _vertices(g, count, V):
    """Vertices as walks and hops meet them: few are met often (low ids here), most seldom."""
    u = torch.rand(count, generator=g, device=_DEVICE, dtype=torch.float64)
    return (u.pow(2.5) * V).to(torch.int64).clamp_(max=V - 1).to(torch.int32)


def _dropped(g, values, count):
    """The values with -1 in `count` places."""
    if count:
        values[torch.randperm(values.numel(), generator=g, device=_DEVICE)[:count]] = -1
    return values


def _groups(keys):
    """What nd_group_by_transit gives for these keys: pairs by key, slots of equal keys ascending; its plan for the calls."""
    order = torch.sort(keys.to(torch.int64), stable=True)
    live = int((keys >= 0).sum())
    first = keys.numel() - live
    sorted_keys, slots = order.values[first:], order.indices[first:]
    ids, sizes = torch.unique_consecutive(sorted_keys, return_counts=True)
    start = torch.zeros(ids.numel() + 1, dtype=torch.int64, device=keys.device)
    start[1:] = torch.cumsum(sizes, 0)
    return slots.to(torch.int32), ids.to(torch.int32), start.to(torch.int32)


def prepare(case, seed):
    g = torch.Generator(device=_DEVICE)
    g.manual_seed(seed)
    n, V, d, dtype = case["n"], case["V"], case["d"], _TYPES[case["type"]]
    state = {"case": dict(case)}

    def rows(count, scale=1.0):
        return (torch.randn(count, d, generator=g, device=_DEVICE) * scale).to(dtype)

    op = case["op"]
    if op.startswith("loss"):
        k = case["k"]
        # products with a spread of about 2: rows of a model under way
        state["x"], state["w"] = rows(n, 2.0 / math.sqrt(d)), rows(V)
        labels = _vertices(g, n * k, V)
        if k > 1:
            labels = _dropped(g, labels, int(n * k * case["ended"]))
        labels = labels.view(n, k)
        dead = torch.randperm(n, generator=g, device=_DEVICE)[:_dead_rows(case)]
        labels[dead] = -1
        # rows of a walk before its end have a label
        empty = (labels < 0).all(dim=1)
        empty[dead] = False
        labels[:, 0] = torch.where(empty, torch.zeros_like(labels[:, 0]), labels[:, 0])
        state["labels"] = labels.contiguous()
        if op == "loss_grad":
            # the mean over all pairs, weighted a little differently from row to row; gradients in fp16 want a loss scale
            spread = 0.5 + torch.rand(n, generator=g, device=_DEVICE)
            state["row_weight"] = spread * ((1024.0 if case["type"] == "f16" else 1.0) / (n * k))
        if own:
            from paper_2009_06693_amd import binding
            state["plan"] = binding.SoftmaxLoss(n, V, d, k, dtype, grad=op == "loss_grad", device=_DEVICE)
        return state

    m = case["m"]
    state["weights"] = torch.rand(n * m, generator=g, device=_DEVICE) * (2.0 / m)
    if op.startswith("regroup"):
        keys = _dropped(g, _vertices(g, n * m, V), _dead_slots(case))
        state["x"] = rows(n)
        state["slots"], state["ids"], state["start"] = _groups(keys)
        pairs = state["slots"].numel()
        state["z"] = rows(pairs)
        if op == "regroup_grad":
            state["dy"], state["dxs"] = rows(n), rows(pairs)
        return state

    vertices = _dropped(g, _vertices(g, n * m, V), _dead_slots(case))
    state["vertices"], state["table"] = vertices, rows(V)
    if op == "neighbours_grad":
        state["dy"] = rows(n)
        state["slots"], state["ids"], state["start"] = _groups(vertices)
    return state


# ------------------------------------------------------------------------------------------------------ plain form
def _plain_loss(x, w, labels, row_weight, grad):
    n, V = x.shape[0], w.shape[0]
    dtype, x, w = x.dtype, x.float(), w.float()
    live, places = labels >= 0, labels.clamp(min=0).long()
    count = live.sum(dim=1).float()
    loss, lse = torch.empty(n, device=x.device), torch.empty(n, device=x.device)
    if grad:
        dx, dw = torch.empty_like(x), torch.zeros_like(w)
    piece = max(1, (1 << 28) // V)
    for a in range(0, n, piece):
        b = min(n, a + piece)
        s = x[a:b] @ w.t()
        top = s.max(dim=1).values
        lse[a:b] = (top + (s - top[:, None]).exp().sum(dim=1).log()) * (count[a:b] > 0)
        met = torch.where(live[a:b], s.gather(1, places[a:b]), 0.0).sum(dim=1)
        loss[a:b] = count[a:b] * lse[a:b] - met
        if not grad:
            continue
        p = (s - lse[a:b, None]).exp() * count[a:b, None]
        p = torch.where(count[a:b, None] > 0, p, 0.0)
        p.scatter_add_(1, places[a:b], -live[a:b].float())
        p *= row_weight[a:b, None]
        dx[a:b] = p @ w
        dw += p.t() @ x[a:b]
    return (loss, lse, dx.to(dtype), dw.to(dtype)) if grad else (loss, lse)


def _plain_weighted(z, index, weights, n, m):
    """Sums over a row's slots of weight times row; slots without a place count nothing."""
    live = index >= 0
    out = torch.zeros(n, z.shape[1], device=z.device)
    for j in range(m):
        at, take = index.view(n, m)[:, j].clamp(min=0).long(), live.view(n, m)[:, j, None]
        part = z[at].float()
        if weights is not None:
            part = part * weights.view(n, m)[:, j, None]
        out += torch.where(take, part, 0.0)
    return out.to(z.dtype)


def _plain_dots(dy, z, index, n, m):
    out = torch.empty(n, m, device=dy.device)
    for j in range(m):
        at = index.view(n, m)[:, j]
        dots = (dy.float() * z[at.clamp(min=0).long()].float()).sum(dim=1)
        out[:, j] = torch.where(at >= 0, dots, 0.0)
    return out.view(-1)


def _plain_pairs(x, slots, weights, m):
    q = slots.long()
    out = x[q // m].float()
    if weights is not None:
        out = out * weights[q, None]
    return out.to(x.dtype)


def _plain_positions(slots, count):
    out = torch.full((count,), -1, dtype=torch.int32, device=slots.device)
    out[slots.long()] = torch.arange(slots.numel(), dtype=torch.int32, device=slots.device)
    return out


def _plain_group_sum(dy, slots, ids, start, weights, m, V):
    q = slots.long()
    out = torch.zeros(V, dy.shape[1], device=dy.device)
    rows = torch.repeat_interleave(ids.long(), (start[1:] - start[:-1]).long(), output_size=q.numel())
    piece = 1 << 21
    for a in range(0, q.numel(), piece):
        part = dy[q[a:a + piece] // m].float() * weights[q[a:a + piece], None]
        out.index_add_(0, rows[a:a + piece], part)
    return out.to(dy.dtype)


# ------------------------------------------------------------------------------------------------------------- run
def run(state):
    case = state["case"]
    op, n = case["op"], case["n"]
    if own:
        return _run_own(state, case, op, n)
    if op.startswith("loss"):
        return _plain_loss(state["x"], state["w"], state["labels"], state.get("row_weight"), op == "loss_grad")
    m, weights = case["m"], state["weights"]
    if op.startswith("regroup"):
        places = _plain_positions(state["slots"], n * m)
        out = [_plain_pairs(state["x"], state["slots"], None, m), _plain_weighted(state["z"], places, weights, n, m)]
        if op == "regroup_grad":
            out += [_plain_pairs(state["dy"], state["slots"], weights, m),
                    _plain_dots(state["dy"], state["z"], places, n, m),
                    _plain_weighted(state["dxs"], places, None, n, m)]
        return out
    out = [_plain_weighted(state["table"], state["vertices"], weights, n, m)]
    if op == "neighbours_grad":
        out += [_plain_group_sum(state["dy"], state["slots"], state["ids"], state["start"], weights, m, case["V"]),
                _plain_dots(state["dy"], state["table"], state["vertices"], n, m)]
    return out


def _run_own(state, case, op, n):
    from paper_2009_06693_amd import binding as B
    if op == "loss":
        return state["plan"].loss(state["x"], state["w"], state["labels"])
    if op == "loss_grad":
        return state["plan"].grad(state["x"], state["w"], state["labels"], state["row_weight"])
    m, weights = case["m"], state["weights"]
    if op.startswith("regroup"):
        slots = state["slots"]
        places = B.nd_group_positions(slots, n * m)
        out = [B.nd_rows_by_transit(state["x"], slots, m), B.nd_rows_to_samples(state["z"], places, m, weights)]
        if op == "regroup_grad":
            out += [B.nd_rows_by_transit(state["dy"], slots, m, weights),
                    B.nd_rows_weight_grad(state["dy"], state["z"], places, m),
                    B.nd_rows_to_samples(state["dxs"], places, m)]
        return out
    out = [B.nd_rows_to_samples(state["table"], state["vertices"], m, weights)]
    if op == "neighbours_grad":
        # the whole table's gradient: rows that no slot holds are zero
        out += [B.nd_rows_group_sum(state["dy"], state["slots"], state["start"], m, weights, group_rows=state["ids"],
                                    num_rows=case["V"]),
                B.nd_rows_weight_grad(state["dy"], state["table"], state["vertices"], m)]
    return out


# ----------------------------------------------------------------------------------------------------------- exact
def _exact_loss(state, grad):
    """By vertices: one-hot counts as a matrix, softmax by torch's definition of it in 64 bits."""
    x, w, labels = state["x"].double(), state["w"].double(), state["labels"].long()
    n, V = x.shape[0], w.shape[0]
    losses, norms, dxs = [], [], []
    dw = torch.zeros_like(w)
    step = max(1, (1 << 27) // V)
    for a in range(0, n, step):
        xa, la = x[a:a + step], labels[a:a + step]
        held = torch.zeros(xa.shape[0], V + 1, dtype=torch.float64, device=x.device)
        at = torch.where(la < 0, torch.full_like(la, V), la)
        held.scatter_add_(1, at, torch.ones_like(at, dtype=torch.float64))
        held = held[:, :V]
        count = held.sum(1)
        s = torch.matmul(xa, w.transpose(0, 1).contiguous())
        norm = torch.logsumexp(s, 1)
        norms.append(torch.where(count > 0, norm, torch.zeros_like(norm)))
        losses.append(torch.where(count > 0, count * norm - (held * s).sum(1), torch.zeros_like(norm)))
        if grad:
            rate = (count[:, None] * torch.softmax(s, 1) - held) * state["row_weight"][a:a + step, None].double()
            dxs.append(torch.matmul(rate, w))
            dw += torch.matmul(rate.transpose(0, 1).contiguous(), xa)
    out = (torch.cat(losses), torch.cat(norms))
    return out + (torch.cat(dxs), dw) if grad else out


def _exact_sums(values, factors, source, target, rows):
    """out[target] += factors * values[source], in 64 bits."""
    out = torch.zeros(rows, values.shape[1], dtype=torch.float64, device=values.device)
    piece = 1 << 20
    for a in range(0, source.numel(), piece):
        cut = slice(a, a + piece)
        part = values[source[cut]].double()
        out.index_add_(0, target[cut], part if factors is None else part * factors[cut].double()[:, None])
    return out


def _exact_products(a, b, of_a, of_b):
    out = torch.empty(of_a.numel(), dtype=torch.float64, device=a.device)
    piece = 1 << 20
    for c in range(0, of_a.numel(), piece):
        cut = slice(c, c + piece)
        out[cut] = (a[of_a[cut]].double() * b[of_b[cut]].double()).sum(1)
    return out


def exact(case, seed):
    state = prepare(case, seed)
    op, n = case["op"], case["n"]
    if op.startswith("loss"):
        return _exact_loss(state, op == "loss_grad")
    m, weights = case["m"], state["weights"]
    if op.startswith("regroup"):
        q = state["slots"].long()
        p = torch.arange(q.numel(), device=q.device)
        parents, factors = torch.div(q, m, rounding_mode="floor"), weights[q]
        out = [state["x"][parents].double(), _exact_sums(state["z"], factors, p, parents, n)]
        if op == "regroup_grad":
            dots = torch.zeros(n * m, dtype=torch.float64, device=q.device)
            dots[q] = _exact_products(state["dy"], state["z"], parents, p)
            out += [state["dy"][parents].double() * factors.double()[:, None], dots,
                    _exact_sums(state["dxs"], None, p, parents, n)]
        return out
    held = state["vertices"].long()
    q = torch.nonzero(held >= 0).view(-1)
    parents, met, factors = torch.div(q, m, rounding_mode="floor"), held[q], weights[q]
    out = [_exact_sums(state["table"], factors, met, parents, n)]
    if op == "neighbours_grad":
        dots = torch.zeros(n * m, dtype=torch.float64, device=q.device)
        dots[q] = _exact_products(state["dy"], state["table"], parents, met)
        out += [_exact_sums(state["dy"], factors, parents, met, case["V"]), dots]
    return out
