"""The oracle's gradient of the routing by scores where a sigmoid nears 0 or 1, against its slope
s (1 - s) = e / (1 + e)^2, e = exp(-|h|), which keeps its bits there."""
import numpy as np

from oracle import gate as OG


def slope(h):
    e = np.exp(-np.abs(h.astype(np.float64)))
    return e / (1 + e) ** 2


def test_oracle_gradient_of_saturated_sigmoids():
    h = np.linspace(-80, 80, 33)[None]
    ids = np.arange(33)[None]
    d = OG.gradient(h, ids, np.ones((1, 33)), "sigmoid", False, 1.0)
    assert (np.abs(d - slope(h)) <= 1e-14 * slope(h)).all()
