"""What the bounds of test_gpu_block_error see: results with the final rounding alone pass, small
mistakes anywhere in the experts do not.  Float64 on the CPU."""
import numpy as np
import pytest

import block_error
from oracle import blocks as OB
from oracle.ffn import silu


def _layer(T=24, E=4, k=2, d=288, f=272):
    rng = np.random.default_rng(1)
    mats = [tuple(OB.rounded(rng.normal(0, 0.05, s)) for s in ((f, d), (f, d), (d, f)))
            for _ in range(E)]
    x = rng.normal(0, 1, (T, d))
    ids = np.stack([rng.permutation(E)[:k] for _ in range(T)])
    return x, ids, rng.uniform(0.2, 1, (T, k)), mats


def _experts(x, ids, w, mats, hidden=OB.rounded, act=silu, mix=lambda w: w):
    y = np.zeros_like(x)
    xr = OB.rounded(x)
    for t in range(len(x)):
        for r in range(ids.shape[1]):
            w1, w3, w2 = mats[ids[t, r]]
            h = act(w1 @ xr[t]) * (w3 @ xr[t])
            y[t] += mix(w[t, r]) * (w2 @ hidden(h[None])[0])
    return y


def _to_bf16(v):
    b = v.astype(np.float32).view(np.uint32).astype(np.uint64)
    b = (b + 0x7FFF + ((b >> 16) & 1)) & 0xFFFF0000
    return b.astype(np.uint32).view(np.float32).astype(np.float64)


def _wrong_scale(h):
    q, s = OB.quantize(h)
    s[:, 0] *= 1.05
    return q * OB.spread(s, *q.shape, block_rows=1)


def test_the_final_rounding_passes():
    ref = _experts(*_layer())
    assert np.allclose(ref, OB.experts(*_layer()[:3], lambda e: _layer()[3][e])[0], rtol=1e-12)
    block_error.check(_to_bf16(ref), ref, block_error.ROUNDING)


MISTAKES = {"1 % too large": lambda ref: 1.01 * ref, "1 % too small": lambda ref: 0.99 * ref,
            "0.2 % too large": lambda ref: 1.002 * ref,
            "hidden rows not quantised": lambda ref: _experts(*_layer(), hidden=lambda h: h),
            "a hidden scale 5 % off": lambda ref: _experts(*_layer(), hidden=_wrong_scale),
            "weights in 8 bits": lambda ref: _experts(
                *_layer(), mix=lambda w: float(OB.round_e4m3(w))),
            "silu of 1 % less": lambda ref: _experts(*_layer(), act=lambda a: silu(0.99 * a))}


@pytest.mark.parametrize("mistake", list(MISTAKES))
def test_small_mistakes_do_not(mistake):
    ref = _experts(*_layer())
    with pytest.raises(AssertionError):
        block_error.check(_to_bf16(MISTAKES[mistake](ref)), ref, block_error.FP8)
