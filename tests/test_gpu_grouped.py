"""Products of groups of rows and their gradients against the float64 oracle, at the sizes where
tiles, blocks and groups end; rows of no group stay as they were and are not read."""
import pytest
import torch

from group_bounds import chain, within
from helpers import DEV, say
from oracle import groups as OG

pytestmark = pytest.mark.gpu
NAN = float("nan")


def _rand(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV).to(torch.bfloat16)


def _case(counts, n, k, seed, lead=0, tail=0, pad=0):
    """Groups of `counts` rows behind `lead` rows of none and before `tail`; values that are no group's
    are NaN.  pad: elements between rows."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    P = lead + sum(counts) + tail
    edge = [lead]
    for c in counts:
        edge.append(edge[-1] + c)

    def rows(cols):
        m = torch.full((P, cols + pad), NAN, dtype=torch.bfloat16, device=DEV)[:, :cols]
        m[lead:edge[-1]] = _rand(g, edge[-1] - lead, cols)
        return m

    w = _rand(g, len(counts), n, k)
    return P, edge, torch.tensor(edge, dtype=torch.int32, device=DEV), rows(k), rows(n), w


EDGES = [0, 1, 15, 16, 17, 31, 32, 33, 0, 63, 64, 65, 127, 128, 129]
CASES = [([1], 8, 8), ([1] * 8, 1536, 2048), ([0, 3, 0, 0, 1], 40, 72), ([24], 520, 64),
         (EDGES, 264, 136), (EDGES, 136, 520), ([255, 256, 257, 0, 1], 512, 192),
         ([700, 300, 513], 328, 1000), ([513], 8, 4096), ([2000], 1368, 8), ([300] * 3, 256, 256),
         ([40, 90, 0, 160], 384, 320)]


@pytest.mark.parametrize("case", range(len(CASES)))
@pytest.mark.parametrize("lead,tail,pad", [(0, 0, 0), (3, 130, 8)])
def test_products(case, lead, tail, pad):
    from paper_2602_07265_amd import xshare as X
    counts, n, k = CASES[case]
    say(f"products case {counts} n={n} k={k} lead={lead} tail={tail} pad={pad}")
    P, edge, offsets, x, dy, w = _case(counts, n, k, case, lead, tail, pad)
    y = torch.full((P, n + pad), 5.0, dtype=torch.bfloat16, device=DEV)
    dx = torch.full((P, k + pad), 5.0, dtype=torch.bfloat16, device=DEV)
    X.grouped_linear(x, w, offsets, y=y[:, :n])
    X.grouped_linear_backward_x(dy, w, offsets, out=dx[:, :k])
    dw = X.grouped_linear_backward_w(dy, x, offsets)
    dwb = X.grouped_linear_backward_w(dy, x, offsets,
                                      out=torch.empty(w.shape, dtype=torch.bfloat16, device=DEV))
    more = X.grouped_linear_backward_w(dy, x, offsets, out=torch.ones_like(dw), accumulate=True)
    torch.cuda.synchronize()
    assert (y[:, n:] == 5.0).all() and (dx[:, k:] == 5.0).all()
    ref, mag = OG.grouped_linear(x, w, edge, torch.full((P, n), 5.0, dtype=torch.float64, device=DEV))
    within(y[:, :n], ref, mag, chain(k), "y")
    ref, mag = OG.grouped_linear_backward_x(
        dy, w, edge, torch.full((P, k), 5.0, dtype=torch.float64, device=DEV))
    within(dx[:, :k], ref, mag, chain(n), "dx")
    ref, mag = OG.grouped_linear_backward_w(dy, x, edge)
    rel = chain(max(counts))
    within(dw, ref, mag, rel, "dw")
    within(dwb, ref, mag, rel, "dw bf16")
    within(more, ref + 1.0, mag, rel, "dw accumulated")


# Every form of the three products (test_group_launches checks that these are what the cases get): its
# tile, whether tiles are split, and groups that leave tiles nearly empty, nearly full and empty.
SKEW = [3000, 0, 1, 700, 4491]
HALVES = [2176, 127, 2177, 3712]    # of 256 rows' tiles, the last ones: 128, 127, 129 and 128
FORMS = [("linear", "64x32 x 2", [40, 0, 19, 1], 520, 2312), ("linear", "64x32 x 2", [1], 72, 10248),
         ("linear", "64x32", [700, 0, 300, 1], 520, 2312), ("linear", "64x64", [700, 0, 300, 1], 1032, 1096),
         ("linear", "128x64", [700, 0, 300, 1], 2312, 520), ("linear", "turns", SKEW, 2312, 520),
         ("linear", "turns", SKEW, 2048, 4104), ("linear", "turns", [8192], 4104, 264),
         ("linear", "turns", [5000, 3191], 2304, 1000),
         ("linear", "turns", HALVES, 2312, 520), ("linear", "turns", HALVES, 2048, 4104),
         ("x", "turns", HALVES, 2056, 4104), ("linear", "turns", [4096], 4096, 1032),
         ("x", "64x32 x 2", [700, 0, 300, 1], 2312, 520), ("x", "64x32 x 2", [0, 33], 10248, 72),
         ("x", "64x32", [700, 0, 300, 1], 520, 520), ("x", "64x64", [700, 0, 300, 1], 1032, 1096),
         ("x", "128x64", SKEW, 1032, 1096), ("x", "128x64", SKEW, 520, 2312),
         ("x", "turns", SKEW, 2056, 4104),
         ("x", "turns", [5000, 3191], 264, 4104),
         ("w", "128x64", [700, 0, 300, 1], 264, 520), ("w", "128x128", SKEW, 1032, 1096),
         ("w", "256x256", [900, 0, 1, 33, 511, 512, 1531, 512], 1016, 2040),
         ("w", "256x256", [900, 0, 1, 33, 511, 512, 1531, 512], 2048, 4104), ("w", "turns", [8192], 1032, 1096),
         ("w", "turns", [8191], 264, 520), ("w", "turns", [8191, 2], 2048, 4104)]


@pytest.mark.parametrize("case", range(len(FORMS)))
def test_forms(case):
    """In buffers between guards, the workspace too."""
    from paper_2602_07265_amd import xshare as X
    what, form, counts, n, k = FORMS[case]
    say(f"products form {form} of {what}: {counts} n={n} k={k}")
    P, edge, offsets, x, dy, w = _case(counts, n, k, case)
    need = X.grouped_linear_workspace_bytes(P, len(counts), n, k)
    ws = torch.full((need + 4096,), 0xA5, dtype=torch.uint8, device=DEV)
    if what == "w":
        buf = torch.full((len(counts) + 2, n, k), 5.0, device=DEV)
        X.grouped_linear_backward_w(dy, x, offsets, out=buf[1:-1], workspace=ws[:need])
        ref, mag = OG.grouped_linear_backward_w(dy, x, edge)
        # a split reduction is up to 256 sums' sum
        rel = chain(max(counts)) + 256 * 2.0 ** -24
    else:
        cols, red = (n, k) if what == "linear" else (k, n)
        buf = torch.full((P + 2, cols), 5.0, dtype=torch.bfloat16, device=DEV)
        call, ref = (X.grouped_linear, OG.grouped_linear) if what == "linear" else \
            (X.grouped_linear_backward_x, OG.grouped_linear_backward_x)
        out = dict(y=buf[1:-1]) if what == "linear" else dict(out=buf[1:-1])
        call(x if what == "linear" else dy, w, offsets, workspace=ws[:need], **out)
        ref, mag = ref(x if what == "linear" else dy, w, edge,
                       torch.zeros((P, cols), dtype=torch.float64, device=DEV))
        rel = chain(red) + 256 * 2.0 ** -24
    torch.cuda.synchronize()
    assert (ws[need:] == 0xA5).all() and (buf[0] == 5.0).all() and (buf[-1] == 5.0).all()
    within(buf[1:-1], ref, mag, rel, form)


@pytest.mark.parametrize("what,counts,n,k", [("linear", SKEW, 2048, 4104), ("x", SKEW, 2056, 4104),
                                             ("w", [8191, 2], 2048, 4104)])
def test_split_forms_again_and_with_infinities(what, counts, n, k):
    """The same bits again, and a row's infinity stays in its row (or group) where tiles are split."""
    from paper_2602_07265_amd import xshare as X
    P, edge, offsets, x, dy, w = _case(counts, n, k, 7)
    call = {"linear": lambda: X.grouped_linear(x, w, offsets),
            "x": lambda: X.grouped_linear_backward_x(dy, w, offsets),
            "w": lambda: X.grouped_linear_backward_w(dy, x, offsets)}[what]
    first = call()
    assert torch.equal(first, call()) and torch.equal(first, call())
    x[edge[1]], dy[edge[1]] = float("inf"), float("inf")
    got = call()
    torch.cuda.synchronize()
    if what == "w":
        assert torch.equal(got[0], first[0]) and not got[1].isfinite().any()
    else:
        at = edge[1]                                   # the second group has rows, or the next ones do
        keep = torch.arange(P, device=DEV) != at
        assert torch.equal(got[keep], first[keep]) and not got[at].isfinite().any()


def test_split_gradient_accumulates():
    from paper_2602_07265_amd import xshare as X
    counts, n, k = [8191], 264, 520
    P, edge, offsets, x, dy, w = _case(counts, n, k, 8)
    one = X.grouped_linear_backward_w(dy, x, offsets)
    two = X.grouped_linear_backward_w(dy, x, offsets, out=one.clone(), accumulate=True)
    half = X.grouped_linear_backward_w(dy, x, offsets,
                                       out=torch.empty_like(one, dtype=torch.bfloat16))
    torch.cuda.synchronize()
    assert torch.equal(two, one + one) and torch.equal(half, one.to(torch.bfloat16))


@pytest.mark.parametrize("E,P,n,k", [(1024, 700, 72, 136), (100, 5000, 264, 200), (65, 65, 128, 512)])
def test_many_groups(E, P, n, k):
    from paper_2602_07265_amd import xshare as X
    say(f"products case of {E} groups, {P} rows")
    g = torch.Generator().manual_seed(E)
    counts = torch.bincount(torch.randint(0, E, (P,), generator=g), minlength=E).tolist()
    P, edge, offsets, x, dy, w = _case(counts, n, k, E)
    y = X.grouped_linear(x, w, offsets)
    dx = X.grouped_linear_backward_x(dy, w, offsets)
    dw = X.grouped_linear_backward_w(dy, x, offsets)
    torch.cuda.synchronize()
    zeros = lambda c: torch.zeros((P, c), dtype=torch.float64, device=DEV)  # noqa: E731
    within(y, *OG.grouped_linear(x, w, edge, zeros(n)), chain(k), "y")
    within(dx, *OG.grouped_linear_backward_x(dy, w, edge, zeros(k)), chain(n), "dx")
    within(dw, *OG.grouped_linear_backward_w(dy, x, edge), chain(max(counts)), "dw")


def test_infinities_stay_in_their_rows_and_groups():
    """Values next to a group's edge and past the reduction's end have no part in it."""
    from paper_2602_07265_amd import xshare as X
    counts, n, k = [70, 1, 65, 30], 72, 104
    P, edge, offsets, x, dy, w = _case(counts, n, k, 9)
    x[edge[1]], dy[edge[1]] = float("inf"), float("inf")     # the whole second group
    y = X.grouped_linear(x, w, offsets)
    dx = X.grouped_linear_backward_x(dy, w, offsets)
    dw = X.grouped_linear_backward_w(dy, x, offsets)
    torch.cuda.synchronize()
    other = torch.ones(P, dtype=torch.bool, device=DEV)
    other[edge[1]] = False
    assert y[other].isfinite().all() and dx[other].isfinite().all()
    assert not y[~other].isfinite().any()
    assert dw[[0, 2, 3]].isfinite().all() and (dw[1].abs() == float("inf")).all()
    # one row's infinity in a group of many: the others' results are what they were
    x2 = x.clone()
    x2[edge[1]] = 1.0
    ref = X.grouped_linear(x2, w, offsets)
    torch.cuda.synchronize()
    assert torch.equal(y[other], ref[other])


def test_no_rows():
    from paper_2602_07265_amd import xshare as X
    P, edge, offsets, x, dy, w = _case([0, 0], 40, 72, 1)
    assert X.grouped_linear(x, w, offsets).shape == (0, 40)
    dw = X.grouped_linear_backward_w(dy, x, offsets, out=torch.ones((2, 40, 72), device=DEV))
    torch.cuda.synchronize()
    assert (dw == 0).all()
    dw = X.grouped_linear_backward_w(dy, x, offsets, out=torch.ones((2, 40, 72), device=DEV),
                                     accumulate=True)
    torch.cuda.synchronize()
    assert (dw == 1).all()


@pytest.mark.parametrize("bad", [[0, 50, 20, 60, 90], [-5, 10, 20, 30, 400], [90, 0, 90, 0, 90],
                                 [2 ** 31 - 1, -2 ** 31, 0, 2 ** 31 - 1, 5]])
def test_offsets_that_are_none_stay_inside_the_buffers(bad):
    """What they give is not said; nothing past the buffers is touched."""
    from paper_2602_07265_amd import xshare as X
    P, _, _, x, dy, w = _case([20, 20, 20, 30], 72, 72, 2)
    offsets = torch.tensor(bad, dtype=torch.int32, device=DEV)
    buf = torch.full((P + 2, 72), 5.0, dtype=torch.bfloat16, device=DEV)
    for call in (lambda o: X.grouped_linear(x, w, offsets, y=o),
                 lambda o: X.grouped_linear_backward_x(dy, w, offsets, out=o)):
        call(buf[1:P + 1])
        torch.cuda.synchronize()
        assert (buf[0] == 5.0).all() and (buf[P + 1] == 5.0).all()
    out = torch.full((6, 72, 72), 5.0, device=DEV)
    X.grouped_linear_backward_w(dy, x, offsets, out=out[1:5])
    torch.cuda.synchronize()
    assert (out[0] == 5.0).all() and (out[5] == 5.0).all()


def test_same_bits_again():
    from paper_2602_07265_amd import xshare as X
    P, edge, offsets, x, dy, w = _case([300, 20, 700, 1], 520, 264, 4)
    calls = (lambda: X.grouped_linear(x, w, offsets),
             lambda: X.grouped_linear_backward_x(dy, w, offsets),
             lambda: X.grouped_linear_backward_w(dy, x, offsets))
    first = [c() for c in calls]
    for _ in range(3):
        for a, c in zip(first, calls):
            assert torch.equal(a.view(torch.uint8), c().view(torch.uint8))
