"""The float64 oracle of the expert order, moves, products of groups of rows and adapters: by hand,
and its gradients against differences."""
import pytest
import torch

from oracle import groups as OG


def test_order_by_hand():
    ids = torch.tensor([[2, 0], [-1, 2], [0, 0], [7, 1]])
    offsets, rows, pairs = OG.expert_order(ids, 3)
    assert offsets == [0, 3, 4, 6]
    assert pairs == [1, 4, 5, 7, 0, 3, -1, -1]
    assert rows == [4, 0, -1, 5, 1, 2, -1, 3]


def _setup(seed=0):
    g = torch.Generator().manual_seed(seed)
    return lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)


def _rows():
    return torch.tensor([[4, 0], [-1, 5], [1, 2], [-1, 3]])


def test_moves_by_hand():
    rn = _setup()
    x, src, w, rows = rn(4, 3), rn(8, 3), rn(4, 2), _rows()
    out = OG.dispatch(x, rows, torch.full((8, 3), 9.0, dtype=torch.float64))
    assert torch.equal(out[[4, 0, 5, 1, 2, 3]], x[[0, 0, 1, 2, 2, 3]]) and (out[6:] == 9).all()
    y, m = OG.combine(src, w, rows)
    assert torch.allclose(y[0], w[0, 0] * src[4] + w[0, 1] * src[0])
    assert torch.allclose(y[1], w[1, 1] * src[5]) and torch.allclose(y[3], w[3, 1] * src[3])
    assert (m >= y.abs() - 1e-12).all()
    y1, _ = OG.combine(src, None, rows)
    assert torch.allclose(y1[2], src[1] + src[2])


def _against_differences(f, inputs, grads, names):
    """d f . v by central differences for a random direction in each input."""
    rn = _setup(5)
    for x, g, name in zip(inputs, grads, names):
        v = rn(*x.shape)
        keep, h = x.clone(), 1e-6
        x.copy_(keep + h * v)
        hi = f()
        x.copy_(keep - h * v)
        lo = f()
        x.copy_(keep)
        assert abs((hi - lo) / (2 * h) - float((g * v).sum())) <= 1e-6 * (1 + float((g * v).abs().sum())), \
            name


def test_gradients_of_moves():
    rn = _setup(1)
    src, w, dy, rows = rn(8, 5), rn(4, 2), rn(4, 5), _rows()
    dsrc, dw, _ = OG.combine_backward(dy, src, w, rows, torch.zeros(8, 5, dtype=torch.float64))
    _against_differences(lambda: float((OG.combine(src, w, rows)[0] * dy).sum()), (src, w),
                         (dsrc, dw), ("src", "w"))
    x, dr = rn(4, 5), rn(8, 5)
    dx = OG.combine(dr, None, rows)[0]
    _against_differences(
        lambda: float((OG.dispatch(x, rows, torch.zeros(8, 5, dtype=torch.float64)) * dr).sum()),
        (x,), (dx,), ("x",))


def test_products_and_their_gradients():
    rn = _setup(2)
    offsets, x, w, dy = [1, 3, 3, 7], rn(8, 5), rn(3, 4, 5), rn(8, 4)
    z = lambda n: torch.zeros(8, n, dtype=torch.float64)  # noqa: E731
    y, _ = OG.grouped_linear(x, w, offsets, z(4))
    assert (y[0] == 0).all() and (y[7] == 0).all()
    assert torch.allclose(y[2], w[0] @ x[2]) and torch.allclose(y[5], w[2] @ x[5])
    dx, _ = OG.grouped_linear_backward_x(dy, w, offsets, z(5))
    dw, _ = OG.grouped_linear_backward_w(dy, x, offsets)
    assert (dw[1] == 0).all()
    _against_differences(lambda: float((OG.grouped_linear(x, w, offsets, z(4))[0] * dy).sum()),
                         (x, w), (dx, dw), ("x", "w"))


@pytest.mark.parametrize("scaled,based", [(True, True), (False, False)])
def test_adapters_and_their_gradients(scaled, based):
    rn = _setup(3)
    ids = torch.tensor([1, -1, 0, 1, 5, 0])
    x, a, b, dy = rn(6, 7), rn(3, 2, 7), rn(3, 4, 2), rn(6, 4)
    s = rn(3) if scaled else None
    base, base_dx = (rn(6, 4), rn(6, 7)) if based else (None, None)
    y, _ = OG.adapters(x, a, b, ids, s, base)
    t = 3
    want = (s[1] if scaled else 1.0) * (b[1] @ (a[1] @ x[t])) + (base[t] if based else 0.0)
    assert torch.allclose(y[t], want)
    assert torch.equal(y[4], base[4] if based else torch.zeros(4, dtype=torch.float64))
    g, _ = OG.adapters_backward(dy, x, a, b, ids, s, base_dx)
    dx = g["dx"] - (base_dx if based else 0.0)
    assert (g["da"][2] == 0).all() and (g["db"][2] == 0).all()
    _against_differences(lambda: float((OG.adapters(x, a, b, ids, s, base)[0] * dy).sum()),
                         (x, a, b), (dx, g["da"], g["db"]), ("x", "a", "b"))
