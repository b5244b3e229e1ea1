"""What the calls on groups of rows may be off by, from their arithmetic.

HALF: the most that a rounding to a type changes a value by, relative to it.  A matrix instruction
sums 32 products into an fp32 accumulator: at most 32 roundings inside and one for each instruction,
each at most 2^-23 of the magnitudes summed (a truncating adder included)."""
import torch

HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def chain(n):
    """Relative to the terms' magnitudes: a sum of n products in matrix instructions."""
    return (-(-n // 32) + 32) * 2.0 ** -23


def within(got, ref, mag, rel, what=""):
    """|got - ref| <= HALF |ref| + rel mag (and rel of that rounded too), everywhere."""
    half = HALF[got.dtype]
    err = (got.double() - ref).abs()
    tol = half * ref.abs() + (1 + half) * rel * mag + 2.0 ** -133
    bad = ~(err <= tol)
    assert not bad.any(), (what, int(bad.sum()), float(err[bad].max()),
                           float((err / tol.clamp(min=1e-300)).nan_to_num(9e9).max()))


def adapter_rel(r, d):
    """y of adapters: two bf16 parts of h (2^-16), sums of d and then 2 r products."""
    return 2.0 ** -16 + chain(d) + chain(2 * r) + 2.0 ** -22


def factor_rel(T, long_side):
    """A factor's gradient: h or dh in three parts (2^-24), its own sum of `long_side` products, the
    sum of 3 T products, up to 768 parts of them."""
    return 2.0 ** -24 + chain(long_side) + chain(3 * T) + 2.0 ** -22
