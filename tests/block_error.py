"""Bounds of the experts' error over a whole output, beside the bounds of single elements.

ROUNDING: y is rounded to bf16 once, each element within half an ulp, 2^-8 of its power of two, and
evenly inside it: at most 2^-7 / sqrt(12) = 2.26e-3 of the elements' RMS.  Exact sums leave little
else (a relative error e of a hidden value h moves it by a whole step, 1/16 to 1/8 of it, with a
probability of about e / step: 1.3e-4 of the RMS for e = 3e-7): 2.4e-3 in all.
FP8: in FP8 instructions e is about 2e-5 of the hidden values' RMS, 0.9e-3 of the output's on average
over many values and more over few: 4e-3 in all.
SLOPE: neither rounding favours a side, so y is ref's size within the RMS bound / sqrt(values)."""
import numpy as np

ROUNDING, FP8, SLOPE = 2.4e-3, 4e-3, 1e-3


def error(y, ref):
    """(RMS of y - ref over ref's, how far y's size along ref is off)."""
    return (np.sqrt(((y - ref) ** 2).sum() / (ref ** 2).sum()),
            abs((y * ref).sum() / (ref ** 2).sum() - 1.0))


def check(y, ref, bound):
    rms, slope = error(y, ref)
    assert rms <= bound and slope <= SLOPE, (rms, slope)
