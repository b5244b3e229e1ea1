"""block_experts' error over whole outputs, in every form (block_error has the bounds).  Each case has
at least 8000 hidden values, so that no single one of them moves the error far."""
import numpy as np
import pytest
import torch

import block_error
from helpers import DEV, say
from oracle import blocks as OB
from test_gpu_blocks import _expert_weights, _f64, _oracle_weight, _routing, _run_experts, _x

pytestmark = pytest.mark.gpu


# gate/up / down: few rows, tiles of 32, 64 and 128 tokens; up to 32 rows an expert gate/up is in bf16
# instructions
@pytest.mark.parametrize("forms,T,E,k,d,f", [
    ("one token", 1, 64, 8, 2048, 1024), ("few / few", 6, 4, 2, 1040, 2320),
    ("few / 64", 16, 1, 1, 4096, 4096), ("few / 64", 60, 12, 3, 272, 528),
    ("few / 32", 130, 50, 4, 1040, 112), ("32 / 32", 60, 100, 4, 528, 272),
    ("32 / few", 16, 128, 8, 144, 784), ("32 / 32", 16, 128, 8, 2048, 768),
    ("128 / 64", 130, 12, 3, 272, 1040), ("128 / 128", 480, 100, 4, 528, 272),
    ("128 in FP8 / 64", 200, 12, 3, 272, 1040), ("128 in FP8 / 128", 1100, 24, 4, 1040, 272)])
def test_error_of_the_whole_output(forms, T, E, k, d, f):
    rng = np.random.default_rng(T + E + d)
    x, mats = _x(rng, T, d), _expert_weights(rng, E, d, f)
    ids, w = _routing(rng, T, E, k)
    say(f"experts error case {forms} T={T} E={E} k={k} d={d} f={f}")
    ref, _ = OB.experts(_f64(x), ids, w.astype(np.float32),
                        lambda e: tuple(_oracle_weight(q[e], s[e]) for q, s in mats))
    y = _f64(_run_experts(x, ids, w, mats))
    rms, slope = block_error.error(y, ref)
    say(f"  error {rms:.2e}, slope off by {slope:.1e}")
    block_error.check(y, ref, block_error.FP8 if "FP8" in forms else block_error.ROUNDING)
