"""Dispatch, combine and their gradients against the float64 oracle; rows of no pair stay as they
were, and nothing of a pair without a row is read."""
import pytest
import torch

from group_bounds import HALF, within
from helpers import DEV, say
from oracle import groups as OG

pytestmark = pytest.mark.gpu
NAN = float("nan")


def _case(T, k, d, dtype, seed, live=0.7, shift=0, pad=0):
    """Tokens, rows, weights and an order of `live` of the pairs.  shift: elements that a matrix
    starts past an allocation's; pad: elements between its rows."""
    g = torch.Generator().manual_seed(seed)

    def matrix(rows, fill=None):
        buf = torch.full((shift + max(rows, 1) * (d + pad),), NAN, dtype=dtype, device=DEV)
        m = buf[shift:shift + rows * (d + pad)].view(rows, d + pad)[:, :d]
        m.copy_(torch.randn(rows, d, generator=g) if fill is None else torch.full((rows, d), fill))
        return m

    P = T * k
    has = torch.rand(P, generator=g) < live
    perm = torch.randperm(int(has.sum()), generator=g)
    at = torch.full((P,), -1, dtype=torch.long)
    at[has] = perm
    rows = at.view(T, k).to(torch.int32).to(DEV)
    w = torch.randn(T, k, generator=g)
    w[at.view(T, k) < 0] = NAN
    return matrix, rows, w.to(DEV), dict(rows=rows)


CASES = [(1, 1, 1), (1, 8, 7168), (5, 2, 7), (7, 3, 1367), (64, 8, 512), (33, 32, 136), (3, 5, 2049),
         (300, 4, 72)]


@pytest.mark.parametrize("T,k,d", CASES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("shift,pad", [(0, 0), (1, 3)])
def test_moves(T, k, d, dtype, shift, pad):
    from paper_2602_07265_amd import xshare as X
    say(f"moves case T={T} k={k} d={d} {dtype} shift={shift} pad={pad}")
    matrix, rows, w, order = _case(T, k, d, dtype, T + d, shift=shift, pad=pad)
    x, src, dy, moved, dsrc = matrix(T), matrix(T * k), matrix(T), matrix(T * k, 5.0), \
        matrix(T * k, 5.0)
    used = torch.zeros(T * k, dtype=torch.bool, device=DEV)
    used[rows[rows >= 0].long()] = True
    src[~used] = NAN                                      # rows of no pair are not read
    X.dispatch(x, order, out=moved)
    y = X.combine(src, w, order)
    dx = X.dispatch_backward(src, order)
    g = X.combine_backward(dy, src, w, order, out=dict(drows=dsrc))
    torch.cuda.synchronize()
    five = torch.full((T * k, d), 5.0, dtype=torch.float64, device=DEV)
    assert torch.equal(moved.double(), OG.dispatch(x, rows, five.clone()))
    # k multiply-adds in fp32, each at most half a step of what it gives
    ref, mag = OG.combine(src, w, rows)
    within(y, ref, mag, (k + 1) * 2.0 ** -24, "y")
    ref, mag = OG.combine(src, None, rows)
    within(dx, ref, mag, (k + 1) * 2.0 ** -24, "dx")
    dref, dw, dmag = OG.combine_backward(dy, src, w, rows, five)
    # one fp32 product, then the rounding
    within(dsrc, dref, dref.abs(), 2.0 ** -24, "dsrc")
    vec = 16 // dtype.itemsize
    # a lane's multiply-adds, six sums of lanes
    within(g["dw"], dw, dmag, (-(-d // (64 * vec)) * vec + 6) * 2.0 ** -24, "dw")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_gradient_in_place_of_the_rows(dtype):
    from paper_2602_07265_amd import xshare as X
    matrix, rows, w, order = _case(40, 4, 1000, dtype, 3)
    src, dy = matrix(160), matrix(40)
    want = X.combine_backward(dy, src, w, order, out=dict(drows=torch.zeros_like(src)))
    ref = src.clone()
    keep = torch.ones(160, dtype=torch.bool, device=DEV)
    keep[rows[rows >= 0].long()] = False
    got = X.combine_backward(dy, src, w, order, out=dict(drows=src))
    torch.cuda.synchronize()
    assert torch.equal(got["dw"], want["dw"]) and torch.equal(src[~keep], want["drows"][~keep])
    assert torch.equal(src[keep], ref[keep])


def test_no_tokens_and_no_rows():
    from paper_2602_07265_amd import xshare as X
    for T, live in ((0, 1.0), (9, 0.0)):
        matrix, rows, w, order = _case(T, 2, 40, torch.bfloat16, 1, live=live)
        x, src = matrix(T), matrix(2 * T, NAN)
        moved = X.dispatch(x, order, out=matrix(2 * T, 5.0))
        y = X.combine(src, w, order)
        g = X.combine_backward(x, src, w, order)
        torch.cuda.synchronize()
        assert (moved == 5.0).all() and (y == 0).all() and (g["dw"] == 0).all()
        assert X.dispatch_backward(src, order).shape == (T, 40)


def test_rows_that_are_no_rows():
    """Indexes past the buffer are no rows: nothing is read or written there."""
    from paper_2602_07265_amd import xshare as X
    rows = torch.tensor([[0, 4], [-7, 2 ** 31 - 1]], dtype=torch.int32, device=DEV)
    x = torch.ones(2, 24, device=DEV)
    out = X.dispatch(x, dict(rows=rows), out=torch.zeros(4, 24, device=DEV))
    y = X.dispatch_backward(torch.full((4, 24), 2.0, device=DEV), dict(rows=rows))
    torch.cuda.synchronize()
    assert (out[0] == 1).all() and (out[1:] == 0).all() and (y[0] == 2).all() and (y[1] == 0).all()


def test_infinities_and_nan_go_through():
    from paper_2602_07265_amd import xshare as X
    rows = torch.tensor([[0, 1]], dtype=torch.int32, device=DEV)
    for dtype in (torch.bfloat16, torch.float32):
        v = torch.tensor([[float("inf"), 1.0, NAN, -float("inf")], [1.0, 2.0, 3.0, 4.0]]).to(DEV, dtype)
        y = X.combine(v, torch.ones(1, 2, device=DEV), dict(rows=rows))
        torch.cuda.synchronize()
        assert y[0, 0] == float("inf") and y[0, 1] == 3.0 and y[0, 2].isnan() and y[0, 3] == -float("inf")
    assert HALF[torch.bfloat16] == 2.0 ** -8
