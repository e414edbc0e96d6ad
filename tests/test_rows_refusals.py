"""What the calls on rows and the softmax loss refuse, before anything is launched (no GPU; the addresses are made up)."""
import pytest

from paper_2009_06693_amd import binding as B

P = 4096  # an address that no call may touch


def _loss(grad, x=P, xs=8, w=P, ws=8, dtype=0, n=4, V=9, d=8, labels=P, k=2, loss=P, lse=P, dx=P, dxs=8, dw=P, dws=8,
          work=P, size=1 << 40):
    if grad:
        return B.lib().nd_softmax_loss_grad(x, xs, w, ws, dtype, n, V, d, labels, k, None, loss, lse, dx, dxs, dw, dws, work,
                                            size, None)
    return B.lib().nd_softmax_loss(x, xs, w, ws, dtype, n, V, d, labels, k, loss, lse, work, size, None)


@pytest.mark.parametrize("grad", [False, True])
@pytest.mark.parametrize("bad,code", [
    (dict(x=None), B.ND_ERR_NULL_POINTER), (dict(w=None), B.ND_ERR_NULL_POINTER), (dict(labels=None), B.ND_ERR_NULL_POINTER),
    (dict(loss=None), B.ND_ERR_NULL_POINTER), (dict(lse=None), B.ND_ERR_NULL_POINTER), (dict(work=None), B.ND_ERR_NULL_POINTER),
    (dict(dtype=3), B.ND_ERR_BAD_ARGUMENT), (dict(dtype=-1), B.ND_ERR_BAD_ARGUMENT), (dict(n=-1), B.ND_ERR_BAD_ARGUMENT),
    (dict(V=0), B.ND_ERR_BAD_ARGUMENT), (dict(k=0), B.ND_ERR_BAD_ARGUMENT), (dict(d=0), B.ND_ERR_BAD_ARGUMENT),
    (dict(xs=7), B.ND_ERR_BAD_ARGUMENT), (dict(ws=7), B.ND_ERR_BAD_ARGUMENT), (dict(xs=-8), B.ND_ERR_BAD_ARGUMENT),
    (dict(x=P + 2), B.ND_ERR_BAD_ARGUMENT), (dict(w=P + 1), B.ND_ERR_BAD_ARGUMENT),
    (dict(d=8193, xs=9000, ws=9000, dxs=9000, dws=9000), B.ND_ERR_TOO_LARGE), (dict(k=65), B.ND_ERR_TOO_LARGE),
    (dict(n=1 << 30), B.ND_ERR_TOO_LARGE), (dict(V=1 << 31), B.ND_ERR_TOO_LARGE), (dict(n=1 << 29, k=4), B.ND_ERR_TOO_LARGE),
    (dict(ws=1 << 61), B.ND_ERR_TOO_LARGE), (dict(size=100), B.ND_ERR_WORKSPACE), (dict(work=P + 128), B.ND_ERR_WORKSPACE),
])
def test_the_loss(grad, bad, code):
    assert _loss(grad, **bad) == code
    assert B.lib().nd_last_error()


@pytest.mark.parametrize("bad", [dict(dxs=7), dict(dws=3), dict(dx=P + 1), dict(dw=P + 2)])
def test_the_gradients_rows(bad):
    assert _loss(True, **bad) == B.ND_ERR_BAD_ARGUMENT


def test_sizes_of_the_loss():
    import torch
    size = B.nd_softmax_loss_workspace_bytes
    assert size(0, 1, 1, 1, torch.float32, False) > 0
    assert size(100, 1000, 64, 1, torch.bfloat16, True) > size(100, 1000, 64, 1, torch.bfloat16, False)
    for bad in ((-1, 9, 8, 1), (4, 0, 8, 1), (4, 9, 0, 1), (4, 9, 8193, 1), (4, 9, 8, 0), (4, 9, 8, 65)):
        with pytest.raises(B.NdError):
            size(*bad, torch.float16, True)
    with pytest.raises(B.NdError):
        size(4, 9, 8, 1, torch.float64, True)
    assert B.lib().nd_softmax_loss_status(None, None) == B.ND_ERR_NULL_POINTER


def _positions(slots=P, pairs=4, n=8, out=P):
    return B.lib().nd_group_positions(slots, pairs, None, n, out, None)


def _by_transit(x=P, xs=8, dtype=0, n=4, d=8, slots=P, pairs=4, m=2, out=P, outs=8):
    return B.lib().nd_rows_by_transit(x, xs, dtype, n, d, slots, pairs, None, m, None, out, outs, None)


def _to_samples(x=P, xs=8, dtype=0, pairs=4, d=8, slots=P, n=4, m=2, out=P, outs=8):
    return B.lib().nd_rows_to_samples(x, xs, dtype, pairs, d, slots, n, m, None, out, outs, None)


def _weight_grad(x=P, xs=8, dtype=0, pairs=4, d=8, slots=P, n=4, m=2, out=P, outs=8):
    return B.lib().nd_rows_weight_grad(x, xs, P, outs, dtype, pairs, d, slots, n, m, out, None)


def _group_sum(x=P, xs=8, dtype=0, n=4, d=8, slots=P, pairs=4, m=2, out=P, outs=8, start=P, groups=3, rows=None, out_rows=3,
               work=P, size=1 << 40):
    return B.lib().nd_rows_group_sum(x, xs, dtype, n, d, slots, pairs, start, groups, None, m, None, rows, out, outs, out_rows,
                                     work, size, None)


@pytest.mark.parametrize("call", [_by_transit, _to_samples, _weight_grad, _group_sum])
@pytest.mark.parametrize("bad,code", [
    (dict(x=None), B.ND_ERR_NULL_POINTER), (dict(slots=None), B.ND_ERR_NULL_POINTER), (dict(out=None), B.ND_ERR_NULL_POINTER),
    (dict(dtype=3), B.ND_ERR_BAD_ARGUMENT), (dict(n=-1), B.ND_ERR_BAD_ARGUMENT), (dict(pairs=-1), B.ND_ERR_BAD_ARGUMENT),
    (dict(m=0), B.ND_ERR_BAD_ARGUMENT), (dict(d=0), B.ND_ERR_BAD_ARGUMENT), (dict(xs=7), B.ND_ERR_BAD_ARGUMENT),
    (dict(outs=7), B.ND_ERR_BAD_ARGUMENT), (dict(x=P + 2), B.ND_ERR_BAD_ARGUMENT),
    (dict(d=8193, xs=9000, outs=9000), B.ND_ERR_TOO_LARGE), (dict(m=65537), B.ND_ERR_TOO_LARGE),
    (dict(n=1 << 30, m=2), B.ND_ERR_TOO_LARGE), (dict(pairs=1 << 31), B.ND_ERR_TOO_LARGE),
])
def test_calls_on_rows(call, bad, code):
    assert call(**bad) == code
    assert B.lib().nd_last_error()


@pytest.mark.parametrize("bad,code", [
    (dict(start=None), B.ND_ERR_NULL_POINTER), (dict(work=None), B.ND_ERR_NULL_POINTER),
    (dict(groups=-1), B.ND_ERR_BAD_ARGUMENT), (dict(out_rows=-1), B.ND_ERR_BAD_ARGUMENT), (dict(out_rows=2), B.ND_ERR_BAD_ARGUMENT),
    (dict(rows=P, out_rows=1 << 31), B.ND_ERR_TOO_LARGE), (dict(groups=1 << 31, out_rows=1 << 31), B.ND_ERR_TOO_LARGE),
    (dict(size=10), B.ND_ERR_WORKSPACE), (dict(work=P + 4), B.ND_ERR_WORKSPACE),
])
def test_sums_per_group(bad, code):
    assert _group_sum(**bad) == code


@pytest.mark.parametrize("bad,code", [
    (dict(slots=None), B.ND_ERR_NULL_POINTER), (dict(out=None), B.ND_ERR_NULL_POINTER), (dict(pairs=-1), B.ND_ERR_BAD_ARGUMENT),
    (dict(n=-1), B.ND_ERR_BAD_ARGUMENT), (dict(n=1 << 31), B.ND_ERR_TOO_LARGE), (dict(pairs=1 << 31), B.ND_ERR_TOO_LARGE),
])
def test_positions(bad, code):
    assert _positions(**bad) == code


def test_sizes_of_sums_per_group():
    size = B.nd_rows_group_sum_workspace_bytes
    assert size(0, 8) > 0 and size(1000, 128) < size(100000, 128)
    assert size(-1, 8) == size(4, 0) == size(4, 8193) == size(1 << 31, 8) == 0
