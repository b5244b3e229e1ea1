"""FP8 products with a scale for each block of 128 (oracle side), in float64.

Quantisation of a block (1 x 128 or 128 x 128): a = max |x|, at least 448 * 2^-126; scale =
a / 448; a code is 448 x / a rounded to the nearest E4M3 value, ties to even.  A product is the
exact sum of decode(code) * scale over both operands; the experts are SwiGLU with the hidden
rows quantised again.
"""
from __future__ import annotations

import numpy as np

from .ffn import decode_e4m3, silu

TINY = 448.0 * 2.0 ** -126
VALUES = decode_e4m3(np.arange(256, dtype=np.uint8))


def round_e4m3(v):
    """The nearest E4M3 value (ties to even) of finite |v| <= 448."""
    v = np.asarray(v, np.float64)
    e = np.frexp(v)[1] - 1
    step = np.exp2(np.maximum(e, -6) - 3.0)
    return np.round(v / step) * step


def spread(s, rows, cols, block_rows=128):
    """Block scales as one for each element."""
    s = np.repeat(np.asarray(s, np.float64), 128, axis=-1)[..., :cols]
    return s if block_rows == 1 else np.repeat(s, block_rows, axis=-2)[..., :rows, :]


def quantize(x, block_rows=1):
    """(values of the codes, scales) of a finite matrix."""
    x = np.asarray(x, np.float64)
    rows, cols = x.shape
    nr, nc = -(-rows // block_rows), -(-cols // 128)
    pad = np.zeros((nr * block_rows, nc * 128))
    pad[:rows, :cols] = np.abs(x)
    a = np.maximum(pad.reshape(nr, block_rows, nc, 128).max(axis=(1, 3)), TINY)
    return round_e4m3(448.0 * x / spread(a, rows, cols, block_rows)), a / 448.0


def rounded(x):
    """x as its 1 x 128 blocks hold it."""
    q, s = quantize(x)
    return q * spread(s, *q.shape, block_rows=1)


def weight(codes, scales):
    codes = np.asarray(codes, np.uint8)
    return VALUES[codes] * spread(np.asarray(scales, np.float32), *codes.shape[-2:])


def product_bound(x, w):
    """A bound on the error of the fp32 sums of x w^T (x, w: what the codes and scales stand
    for).  The matrix instruction aligns the products of eight neighbouring inputs to the largest
    and drops what lies more than 13 bits below it: at most 8 * 2^-13 of the largest for each
    eight; the sums over blocks add (blocks + 2) 2^-23 of the sum of the products' sizes."""
    K = x.shape[1]
    pad = (-K) % 8
    ax, aw = (np.pad(np.abs(v), ((0, 0), (0, pad))) for v in (x, w))
    gx, gw = (v.reshape(v.shape[0], -1, 8).max(axis=2) for v in (ax, aw))
    return 8 * 2.0 ** -13 * (gx @ gw.T) + (-(-K // 128) + 2) * 2.0 ** -23 * (ax @ aw.T)


def experts(x, ids, w, weights):
    """y [T, d] and, for each pair, the largest term max_i |h_i W2_ji| of every output: a code
    of h that falls on the other side of its rounding boundary moves a term by an eighth of it at
    most.  weights(e): (W1, W3, W2) in float64."""
    x = np.asarray(x, np.float64)
    T, d = x.shape
    ids = np.asarray(ids)
    xr = rounded(x)
    y, term = np.zeros((T, d)), np.zeros((T, d))
    for e in np.unique(ids):
        mats = weights(int(e))
        if mats is None:
            continue
        w1, w3, w2 = mats
        t, r = np.nonzero(ids == e)
        h = rounded(silu(xr[t] @ w1.T) * (xr[t] @ w3.T))
        o = h @ w2.T
        for i in range(len(t)):
            wr = float(w[t[i], r[i]])
            y[t[i]] += wr * o[i]
            term[t[i]] += abs(wr) * np.abs(h[i][None, :] * w2).max(axis=1)
    return y, term
