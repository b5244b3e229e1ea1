"""The float64 oracle of the block-scaled FP8 products."""
import numpy as np
import pytest

from oracle import blocks as OB
from oracle.ffn import decode_e4m3


def test_rounding_is_to_the_nearest_value_ties_to_even():
    finite = np.unique(OB.VALUES[np.isfinite(OB.VALUES)])
    assert len(finite) == 253 and finite[-1] == 448.0
    rng = np.random.default_rng(0)
    v = np.concatenate([rng.uniform(-448, 448, 2000), rng.normal(0, 0.01, 2000),
                        (finite[:-1] + finite[1:]) / 2, finite])
    got = OB.round_e4m3(v)
    mantissa = {decode_e4m3(np.uint8(c)).item(): c & 1 for c in range(128) if c != 127}
    for x, r in zip(v, got):
        d = np.abs(finite - x)
        near = finite[d == d.min()]
        assert r in near
        if len(near) == 2:
            assert mantissa[abs(float(r))] == 0


@pytest.mark.parametrize("block_rows,rows,cols", [(1, 3, 272), (128, 130, 144), (128, 5, 16)])
def test_quantised_values(block_rows, rows, cols):
    rng = np.random.default_rng(1)
    x = rng.normal(0, 1, (rows, cols))
    x[0] = 0.0
    q, s = OB.quantize(x, block_rows)
    assert s.shape == (-(-rows // block_rows), -(-cols // 128))
    back = q * OB.spread(s, rows, cols, block_rows)
    a = 448.0 * OB.spread(s, rows, cols, block_rows)
    # half a step of E4M3: 2^-4 of the value, or of the least normal 2^-6 448 / a
    assert (np.abs(back - x) <= np.maximum(np.abs(x) * 2.0 ** -4, a / 448 * 2.0 ** -10)).all()
    assert (back[0] == 0).all()
    for r in range(s.shape[0]):
        for c in range(s.shape[1]):
            part = x[r * block_rows:(r + 1) * block_rows, c * 128:(c + 1) * 128]
            assert s[r, c] == max(np.abs(part).max(), OB.TINY) / 448.0


def test_experts_are_the_sum_over_pairs():
    rng = np.random.default_rng(2)
    T, E, d, f = 4, 3, 32, 48
    x = rng.normal(0, 1, (T, d))
    mats = [tuple(rng.normal(0, 0.1, s) for s in ((f, d), (f, d), (d, f))) for _ in range(E)]
    ids = np.array([[0, 2], [1, -1], [-1, -1], [2, 7]])
    w = rng.uniform(0, 1, (T, 2))
    y, term = OB.experts(x, ids, w, lambda e: mats[e] if 0 <= e < E else None)
    assert (y[2] == 0).all() and (term[2] == 0).all()
    xr = OB.rounded(x)
    for t in (0, 1, 3):
        ref = np.zeros(d)
        for r in range(2):
            if 0 <= ids[t, r] < E:
                w1, w3, w2 = mats[ids[t, r]]
                a, b = w1 @ xr[t], w3 @ xr[t]
                ref += w[t, r] * (w2 @ OB.rounded((a / (1 + np.exp(-a)) * b)[None])[0])
        assert np.allclose(y[t], ref, rtol=1e-12, atol=1e-15)
