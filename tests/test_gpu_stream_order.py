"""Calls on another stream than the current one, with workspaces and outputs of their own, while
the current stream allocates and overwrites memory: the results stay those of calls in order."""
import numpy as np
import pytest
import torch

from helpers import DEV, say
from test_gpu_blocks import _expert_weights, _routing, _weight, _x

pytestmark = pytest.mark.gpu


def _stream_of_memory(t):
    for seg in torch.cuda.memory_snapshot():
        if seg["address"] <= t.data_ptr() < seg["address"] + seg["total_size"]:
            return seg["stream"]
    raise AssertionError("not the caching allocator's memory")


def _calls(X):
    rng = np.random.default_rng(50)
    T, E, k, d, f = 40, 16, 4, 1024, 512
    x, mats = _x(rng, T, d).to(DEV), _expert_weights(rng, E, d, f)
    mats = [(q.to(DEV), s.to(DEV)) for q, s in mats]
    ids, w = _routing(rng, T, E, k)
    ids = torch.from_numpy(ids.astype(np.int32)).to(DEV)
    w = torch.from_numpy(w.astype(np.float32)).to(DEV)
    q, s = (t.to(DEV) for t in _weight(rng, 1003, d))
    wg = torch.from_numpy(rng.normal(0, 0.1, (E, d)).astype(np.float32)).to(DEV, torch.bfloat16)
    h = torch.from_numpy(rng.normal(0, 1.5, (T, E)).astype(np.float32)).to(DEV)
    dense = [torch.randn(sh, device=DEV).to(torch.bfloat16) * 0.05
             for sh in ((E, f, d), (E, f, d), (E, d, f))]
    qs, ss = [m[0] for m in mats], [m[1] for m in mats]
    return {
        "experts": lambda **kw: X.block_experts(x, ids, w, *qs, *ss, **kw),
        "linear": lambda **kw: X.block_linear(x, q, s, **kw),
        "quantize": lambda **kw: X.block_quantize(x, **kw)[0],
        "gate": lambda **kw: X.gate(h, k, **kw)["w"],
        "gate_backward": lambda **kw: X.gate_backward(h, ids, w, **kw),
        "router_logits": lambda **kw: X.router_logits(x, wg, **kw),
        "route": lambda **kw: X.route(h, k, 1, 8, **kw)["w"],
        "select_hier": lambda **kw: X.select_hier(h, [0, 10, T], k, 1, 4, 8, **kw)["w"],
        "moe_forward": lambda **kw: X.moe_forward(x, h, *dense, k, 1, 8, **kw)["y"],
        "moe_layer": lambda **kw: X.moe_layer(x, wg, *dense, k, 1, 8, **kw)["y"],
    }


def test_calls_on_a_stream_that_is_not_current():
    from paper_2602_07265_amd import xshare as X
    calls = _calls(X)
    ref = {name: call().clone() for name, call in calls.items()}
    torch.cuda.synchronize()
    side = [torch.cuda.Stream(), torch.cuda.Stream()]
    for name, call in calls.items():
        say(f"stream order case {name}")
        got = []
        for rep in range(6):
            got.append(call(stream=side[rep % 2]))
            assert _stream_of_memory(got[-1]) == side[rep % 2].cuda_stream, name
            for size in (1 << 12, 1 << 16, 1 << 19, 1 << 21):        # what the call has dropped
                torch.full((size,), 0xFF, dtype=torch.uint8, device=DEV)
        torch.cuda.synchronize()
        for y in got:
            assert torch.equal(y.view(torch.uint8), ref[name].view(torch.uint8)), name
