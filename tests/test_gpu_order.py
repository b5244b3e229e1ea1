"""The pairs' expert order against a stable sort, bit for bit."""
import pytest
import torch

from helpers import DEV, say

pytestmark = pytest.mark.gpu


def _expected(ids, n):
    flat = ids.reshape(-1).long().cpu()
    key = torch.where((flat >= 0) & (flat < n), flat, torch.full_like(flat, n))
    pairs = torch.sort(key, stable=True).indices
    rows = torch.empty_like(pairs)
    rows[pairs] = torch.arange(pairs.numel())
    offsets = torch.cat([torch.zeros(1, dtype=torch.long),
                         torch.bincount(key, minlength=n + 1)[:n].cumsum(0)])
    return (offsets, rows.masked_fill(key == n, -1).view(ids.shape),
            pairs.masked_fill(key[pairs] == n, -1))


def _check(ids, n, **kw):
    from paper_2602_07265_amd import xshare as X
    got = X.expert_order(ids, n, **kw)
    torch.cuda.synchronize()
    for name, want in zip(("offsets", "rows", "pairs"), _expected(ids, n)):
        assert torch.equal(got[name].cpu().long(), want), name
    return got


def _ids(T, k, n, kind, seed=0):
    g = torch.Generator().manual_seed(seed)
    ids = torch.randint(0, n, (T, k), generator=g)
    if kind == "dropped":
        ids[torch.rand(T, k, generator=g) < 0.6] = -1
    elif kind == "none":
        ids[:] = torch.randint(n, n + 5, (T, k), generator=g)
    elif kind == "one":
        ids[:] = n - 1
    elif kind == "wild":
        ids = torch.randint(-2 ** 31, 2 ** 31 - 1, (T, k), generator=g)
        ids[::3] %= n
    elif kind == "sorted":
        ids = ids.reshape(-1).sort(descending=True).values.view(T, k)
    return ids.to(torch.int32).to(DEV)


# one workgroup and its last size, several and their parts' edges
@pytest.mark.parametrize("T,k,n", [(1, 1, 1), (1, 8, 256), (1, 32, 1024), (33, 2, 7), (129, 8, 1),
                                   (1024, 8, 256), (8192, 1, 1024), (8193, 1, 63), (2731, 3, 64),
                                   (4096, 5, 65), (16384, 8, 128), (512, 8, 1024), (4097, 1, 63),
                                   (8192, 8, 300), (65537, 1, 1024), (32768, 16, 9), (524289, 1, 33)])
@pytest.mark.parametrize("kind", ["random", "dropped", "none", "one", "wild", "sorted"])
def test_order(T, k, n, kind):
    say(f"order case T={T} k={k} n={n} {kind}")
    _check(_ids(T, k, n, kind), n)


def test_order_of_the_most_pairs():
    say("order case 2^20 pairs of 1024")
    _check(_ids(1 << 15, 32, 1024, "dropped"), 1024)


def test_order_without_tokens():
    from paper_2602_07265_amd import xshare as X
    r = X.expert_order(torch.empty((0, 4), dtype=torch.int32, device=DEV), 5)
    torch.cuda.synchronize()
    assert r["offsets"].tolist() == [0] * 6 and r["rows"].shape == (0, 4)


def test_order_into_given_buffers_and_workspace():
    from paper_2602_07265_amd import xshare as X
    ws = torch.empty(X.expert_order_workspace_bytes(9000, 2, 300), dtype=torch.uint8, device=DEV)
    for T in (9000, 4097, 20, 1):
        ids = _ids(T, 2, 300, "dropped", T)
        out = dict(offsets=torch.full((301,), 7, dtype=torch.int32, device=DEV),
                   pairs=torch.full((2 * T,), 7, dtype=torch.int32, device=DEV))
        got = _check(ids, 300, out=out, workspace=ws)
        assert got["offsets"] is out["offsets"] and got["pairs"] is out["pairs"]
