"""Matrices whose rows lie as far apart as they may, in one buffer of more than 2^32 elements, each beside
the others: every call gives the bits that it gives for the same rows close together."""
import pytest
import torch

from helpers import DEV, say
from test_gpu_adapters import _case as _adapters
from test_gpu_grouped import _case as _groups

pytestmark = pytest.mark.gpu
LD, ROWS = 1 << 22, 1100


@pytest.fixture(scope="module")
def columns():
    buf = torch.empty((ROWS, LD), dtype=torch.bfloat16, device=DEV)
    used = [0]

    def take(rows, cols, of=None):
        """rows of cols values of the buffer, its columns after the last taken ones; `of` copied."""
        if rows == 0:
            used[0] = 0
            return None
        m = buf[:rows, used[0]:used[0] + cols]
        used[0] += cols
        assert used[0] <= LD and m.stride() == (LD, 1)
        return m if of is None else m.copy_(of)
    yield take
    del buf


@pytest.mark.parametrize("counts,n,k", [([3, 0, 1096], 2056, 1096), ([1100], 136, 72),
                                        ([17] * 64 + [12], 264, 520)])
def test_products(columns, counts, n, k):
    from paper_2602_07265_amd import xshare as X
    say(f"products of far rows: {counts} n={n} k={k}")
    P, _, offsets, x, dy, w = _groups(counts, n, k, 5)
    columns(0, 0)
    fx, fdy, fy, fdx = columns(P, k, x), columns(P, n, dy), columns(P, n), columns(P, k)
    want = (X.grouped_linear(x, w, offsets), X.grouped_linear_backward_x(dy, w, offsets),
            X.grouped_linear_backward_w(dy, x, offsets))
    got = (X.grouped_linear(fx, w, offsets, y=fy), X.grouped_linear_backward_x(fdy, w, offsets, out=fdx),
           X.grouped_linear_backward_w(fdy, fx, offsets))
    torch.cuda.synchronize()
    for name, a, b in zip(("y", "dx", "dw"), got, want):
        assert torch.equal(a, b), name


def test_moves(columns):
    from paper_2602_07265_amd import xshare as X
    T, k, d = 275, 4, 1001
    say("moves of far rows")
    g = torch.Generator(device=DEV).manual_seed(1)
    rn = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    ids = torch.randint(0, 9, (T, k), generator=g, device=DEV).to(torch.int32)
    o, w = X.expert_order(ids, 9), rn(T, k)
    x, src = rn(T, d).bfloat16(), rn(T * k, d).bfloat16()
    columns(0, 0)
    fx, fsrc = columns(T, d, x), columns(T * k, d, src)
    outs = [columns(r, d) for r in (T * k, T, T, T * k)]
    want = (X.dispatch(x, o), X.combine(src, w, o), X.dispatch_backward(src, o),
            X.combine_backward(x, src, w, o))
    got = (X.dispatch(fx, o, out=outs[0]), X.combine(fsrc, w, o, out=outs[1]),
           X.dispatch_backward(fsrc, o, out=outs[2]),
           X.combine_backward(fx, fsrc, w, o, out=dict(drows=outs[3])))
    torch.cuda.synchronize()
    for a, b in zip(got[:3], want[:3]):
        assert torch.equal(a, b)
    assert torch.equal(got[3]["drows"], want[3]["drows"]) and torch.equal(got[3]["dw"], want[3]["dw"])


@pytest.mark.parametrize("T,r", [(7, 16), (7, 64), (1100, 16), (1100, 32), (1100, 72)])
def test_adapters(columns, T, r):
    from paper_2602_07265_amd import xshare as X
    L, n, d = 3, 264, 520
    say(f"adapters of far rows: T={T} r={r}")
    c = _adapters(T, L, r, n, d, r)
    columns(0, 0)
    f = {name: columns(T, c[name].shape[1], c[name]) for name in ("x", "dy", "base", "base_dx")}
    out, dx, rest = columns(T, n), columns(T, d), (c["a"], c["b"], c["ids"])
    want = X.adapters(c["x"], *rest, scales=c["scales"], base=c["base"])
    back = X.adapters_backward(c["dy"], c["x"], *rest, scales=c["scales"], base=c["base_dx"])
    got = X.adapters(f["x"], *rest, scales=c["scales"], base=f["base"], out=out)
    fback = X.adapters_backward(f["dy"], f["x"], *rest, scales=c["scales"], base=f["base_dx"],
                                out=dict(dx=dx))
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    for name in ("dx", "da", "db"):
        assert torch.equal(fback[name], back[name]), name


def test_a_single_row_beside_the_rows_it_goes_to():
    """One token in the columns behind its experts' rows."""
    from paper_2602_07265_amd import xshare as X
    say("one token beside its rows")
    k, d = 4, 136
    buf = torch.zeros((k, 2 * d), dtype=torch.bfloat16, device=DEV)
    buf[2, d:] = torch.arange(d, device=DEV)
    o = X.expert_order(torch.tensor([[3, 1, 0, 2]], dtype=torch.int32, device=DEV), 4)
    X.dispatch(buf[2:3, d:], o, out=buf[:, :d])
    torch.cuda.synchronize()
    assert all(torch.equal(buf[i, :d], buf[2, d:]) for i in range(k))
    assert (buf[[0, 1, 3], d:] == 0).all()
