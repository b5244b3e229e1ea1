"""What holds for a call of adapters whatever way it goes, where its tokens are put in adapters' order
(test_adapter_paths checks that these sizes go so) and with one by one beside it: in place of the base, tokens
without an adapter, infinities, another stream; at every width of the rank's tiles."""
import pytest
import torch

from helpers import DEV, say
from test_gpu_adapters import NAN, _case
from test_gpu_groups_run import _stream_of_memory, _tuning

pytestmark = pytest.mark.gpu
L, N, D = 3, 136, 264
FEW, MANY = 8, 300                    # tokens: one by one, in order
RANKS = [16, 24, 40, 72, 128]
BOTH = [(T, r) for T in (FEW, MANY) for r in RANKS]
FACTORS = ("da", "db")


@pytest.mark.parametrize("T,r", BOTH)
def test_in_place_of_the_base(T, r):
    from paper_2602_07265_amd import xshare as X
    say(f"adapters in place of the base: T={T} r={r}")
    c = _case(T, L, r, N, D, 3 + r, pad=8)
    args = (c["x"], c["a"], c["b"], c["ids"])
    want = X.adapters(*args, scales=c["scales"], base=c["base"])
    got = X.adapters(*args, scales=c["scales"], base=c["base"], out=c["base"])
    g = X.adapters_backward(c["dy"], *args, base=c["base_dx"])
    h = X.adapters_backward(c["dy"], *args, base=c["base_dx"], out=dict(dx=c["base_dx"]))
    torch.cuda.synchronize()
    assert got is c["base"] and torch.equal(got, want)
    assert h["dx"] is c["base_dx"] and torch.equal(h["dx"], g["dx"])


@pytest.mark.parametrize("T,r", BOTH)
def test_tokens_without_an_adapter_have_no_part(T, r):
    from paper_2602_07265_amd import xshare as X
    say(f"adapters and tokens without one: T={T} r={r}")
    c = _case(T, L, r, N, D, 4 + r, none=0.5)
    c["ids"][0], c["ids"][1] = -1, 1
    off = (c["ids"] < 0) | (c["ids"] >= L)
    clean = {name: v.clone() for name, v in c.items()}
    c["x"][off], c["dy"][off] = NAN, float("inf")
    for s in (c, clean):
        s["y"] = X.adapters(s["x"], s["a"], s["b"], s["ids"], base=clean["base"])
        s["z"] = X.adapters(s["x"], s["a"], s["b"], s["ids"])
        s["g"] = X.adapters_backward(s["dy"], s["x"], s["a"], s["b"], s["ids"])
    torch.cuda.synchronize()
    assert torch.equal(c["y"], clean["y"]) and torch.equal(c["z"], clean["z"])
    assert torch.equal(c["y"][off], clean["base"][off]) and (c["z"][off] == 0).all()
    for name in ("dx", *FACTORS):
        assert torch.equal(c["g"][name], clean["g"][name]), name
    assert (c["g"]["dx"][off] == 0).all()


@pytest.mark.parametrize("T,r", BOTH)
def test_no_token_has_an_adapter(T, r):
    from paper_2602_07265_amd import xshare as X
    say(f"adapters of no token: T={T} r={r}")
    c = _case(T, L, r, N, D, 5 + r, none=1.0, pad=8)
    args = (c["x"], c["a"], c["b"], c["ids"])
    y, z = X.adapters(*args, base=c["base"]), X.adapters(*args)
    same = c["base"].clone()
    X.adapters(*args, base=same, out=same)
    g = X.adapters_backward(c["dy"], *args, base=c["base_dx"])
    torch.cuda.synchronize()
    assert torch.equal(y, c["base"]) and torch.equal(same, c["base"]) and (z == 0).all()
    assert torch.equal(g["dx"], c["base_dx"]) and (g["da"] == 0).all() and (g["db"] == 0).all()


@pytest.mark.parametrize("T,r", BOTH)
def test_an_infinity_stays_in_its_token(T, r):
    from paper_2602_07265_amd import xshare as X
    say(f"adapters and an infinity: T={T} r={r}")
    c = _case(T, L, r, N, D, 6 + r, none=0.0)
    ref = X.adapters(c["x"], c["a"], c["b"], c["ids"], base=c["base"])
    c["x"][3, 5] = float("inf")
    y = X.adapters(c["x"], c["a"], c["b"], c["ids"], base=c["base"])
    torch.cuda.synchronize()
    other = torch.arange(T, device=DEV) != 3
    assert torch.equal(y[other], ref[other]) and not y[3].isfinite().any()


@pytest.mark.parametrize("T,r", BOTH)
@pytest.mark.parametrize("where", ["x", "dy"])
def test_an_infinity_and_the_factors_gradients(T, r, where):
    """In a token's x: that column of its adapter's da, and by h all of its db.  In its dy: that row of db
    and, by dh, all of da and the token's dx.  Everything else keeps its bits."""
    from paper_2602_07265_amd import xshare as X
    say(f"adapters' gradients and an infinity in {where}: T={T} r={r}")
    c = _case(T, L, r, N, D, 7 + r, none=0.0)
    args = (c["x"], c["a"], c["b"], c["ids"])
    ref = X.adapters_backward(c["dy"], *args, base=c["base_dx"])
    c[where][3, 5] = float("inf")
    got = X.adapters_backward(c["dy"], *args, base=c["base_dx"])
    torch.cuda.synchronize()
    e = int(c["ids"][3])
    others = torch.arange(L, device=DEV) != e
    for name in FACTORS:
        assert torch.equal(got[name][others], ref[name][others]), name
    if where == "x":
        keep = torch.arange(D, device=DEV) != 5
        assert torch.equal(got["dx"], ref["dx"])
        assert torch.equal(got["da"][e][:, keep], ref["da"][e][:, keep])
        assert not got["da"][e][:, 5].isfinite().any() and not got["db"][e].isfinite().any()
    else:
        keep, rows = torch.arange(T, device=DEV) != 3, torch.arange(N, device=DEV) != 5
        assert torch.equal(got["dx"][keep], ref["dx"][keep]) and not got["dx"][3].isfinite().any()
        assert torch.equal(got["db"][e][rows], ref["db"][e][rows])
        assert not got["db"][e][5].isfinite().any() and not got["da"][e].isfinite().any()


TUNED = [300, 250, 9]                 # tokens of _tuning: the first in order


def test_calls_on_a_stream_that_is_not_current():
    from paper_2602_07265_amd import xshare as X
    for T in TUNED:
        t = _tuning(T)
        args = (t["x"], t["a"], t["b"], t["ids"])
        calls = (lambda **kw: X.adapters(*args, scales=t["scales"], **kw),
                 lambda **kw: X.adapters_backward(t["dy"], *args, scales=t["scales"], **kw)["db"])
        ref = [call().clone() for call in calls]
        torch.cuda.synchronize()
        side = [torch.cuda.Stream(), torch.cuda.Stream()]
        for i, call in enumerate(calls):
            say(f"adapters call {i} of {T} tokens on another stream")
            got = []
            for rep in range(6):
                got.append(call(stream=side[rep % 2]))
                assert _stream_of_memory(got[-1]) == side[rep % 2].cuda_stream
                for size in (1 << 12, 1 << 16, 1 << 19, 1 << 21):    # what the call has dropped
                    torch.full((size,), 0xFF, dtype=torch.uint8, device=DEV)
            torch.cuda.synchronize()
            for v in got:
                assert torch.equal(v, ref[i]), (T, i)
