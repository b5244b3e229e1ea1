"""The FP8 products with a scale for each block of 128 against the float64 oracle.

Codes must equal the oracle's exactly (bf16 inputs: the quotient is correctly rounded), scales
within one rounding.  block_linear: the bound of the matrix instruction's sums
(oracle.blocks.product_bound) and half an ulp of bf16.  block_experts: half an ulp of bf16, the
bounds of the two products (a relative 2^-10 of the terms' sizes covers both) and one code of
each hidden row on the other side of its rounding boundary, which moves that pair's largest term
by an eighth at most."""
import numpy as np
import pytest
import torch

from helpers import DEV, say
from oracle import blocks as OB
from test_gpu_guards import IN_FILL, OUT_FILL, Guarded

pytestmark = pytest.mark.gpu
HALF_ULP = 2.0 ** -8       # of bf16, relative to the value's power of two


def _x(rng, rows, cols, spread=1.0):
    v = rng.normal(0, spread, (rows, cols))
    v[:, rng.random(cols) < 0.02] *= 20
    return torch.from_numpy(v.astype(np.float32)).to(torch.bfloat16)


def _f64(t):
    return t.detach().cpu().double().numpy()


def _codes(rng, *shape):
    """Random finite codes, small values more often than large ones."""
    v = rng.normal(0, 90, shape).clip(-448, 448).astype(np.float32)
    return torch.from_numpy(v).to(torch.float8_e4m3fn).view(torch.uint8)


def _weight(rng, *shape):
    """Codes and scales (of no particular order from block to block)."""
    n = [-(-v // 128) for v in shape[-2:]]
    s = torch.from_numpy(rng.uniform(0.2, 2.0, (*shape[:-2], *n)).astype(np.float32) * 1e-3)
    return _codes(rng, *shape), s


def _oracle_weight(q, s):
    return OB.weight(q.numpy(), s.numpy())


# ------------------------------------------------------------------------- quantiser

def _check_quantize(x, block_rows, got):
    q, s = OB.quantize(_f64(x), block_rows)
    values = OB.VALUES[got[0].cpu().numpy()]
    assert np.array_equal(values, q)
    assert (np.abs(_f64(got[1]) - s) <= 2.0 ** -24 * s).all()


@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("rows,cols", [(1, 16), (1, 128), (2, 144), (3, 112), (16, 256),
                                       (127, 272), (128, 128), (129, 400), (300, 1040)])
def test_quantize(rows, cols, block_rows):
    from paper_2602_07265_amd import xshare as X
    rng = np.random.default_rng(rows + cols)
    x = _x(rng, rows, cols)
    say(f"quantize case {rows}x{cols} blocks of {block_rows}")
    _check_quantize(x, block_rows, X.block_quantize(x.to(DEV), block_rows))


def test_quantize_every_quotient_and_range():
    """Maxima of every mantissa against values of every mantissa, ties among them, from the least
    to the largest exponents of bf16; zero blocks."""
    from paper_2602_07265_amd import xshare as X
    rows = []
    mant = np.arange(128, dtype=np.uint32)
    for e in (0, 1, 2, 9, 60, 64, 65, 66, 127, 200, 227, 228, 254):
        for m in range(0, 128, 3):
            top = np.uint32((e << 7) | m)
            v = (np.maximum(int(top) - (rows.__len__() % 9) * 128 - mant.astype(np.int64), 0)
                 ).astype(np.uint32)
            v[0] = top
            v[1::2] |= 0x8000
            rows.append(v)
    rows.append(np.zeros(128, np.uint32))
    x = torch.from_numpy(np.stack(rows).astype(np.uint16).view(np.int16)).view(torch.bfloat16)
    say(f"quantize case ranges {tuple(x.shape)}")
    _check_quantize(x, 1, X.block_quantize(x.to(DEV)))


def test_quantize_not_finite():
    from paper_2602_07265_amd import xshare as X
    x = torch.ones((4, 272), dtype=torch.bfloat16)
    x[0, 3], x[1, 130], x[2, 0], x[2, 1] = float("inf"), float("nan"), float("-inf"), float("nan")
    q, s = X.block_quantize(x.to(DEV))
    v, s = OB.VALUES[q.cpu().numpy()], s.cpu().numpy()
    assert np.isinf(s[0, 0]) and np.isnan(s[1, 1]) and np.isnan(s[2, 0])
    assert np.isfinite(s).sum() == 9
    with np.errstate(invalid="ignore"):
        back = v * OB.spread(s, 4, 272, block_rows=1)
    bad = np.zeros((4, 272), bool)
    bad[0, :128] = bad[1, 128:256] = bad[2, :128] = True
    assert np.isnan(back[bad]).all() and (v[~bad] == 448).all()   # 1 is its block's maximum


def test_quantize_strided_guarded_and_empty():
    from paper_2602_07265_amd import xshare as X
    rng = np.random.default_rng(4)
    rows, cols, ld = 131, 176, 200
    x = _x(rng, rows, cols)
    for br in (1, 128):
        buf = Guarded(rows * ld * 2, IN_FILL)
        view = buf.view(torch.bfloat16, (rows, ld))[:, :cols]
        view.copy_(x.to(DEV))
        shape = (-(-rows // br), 2)
        gq, gs = Guarded(rows * cols, OUT_FILL), Guarded(shape[0] * 8, OUT_FILL)
        out = (gq.view(torch.uint8, (rows, cols)), gs.view(torch.float32, shape))
        say(f"quantize case strided blocks of {br}")
        X.block_quantize(view, br, out=out)
        torch.cuda.synchronize()
        _check_quantize(x, br, out)
        assert buf.intact() and gq.intact() and gs.intact()
    q, s = X.block_quantize(torch.empty((0, 32), dtype=torch.bfloat16, device=DEV))
    assert q.shape == (0, 32) and s.shape == (0, 1)
    with pytest.raises(X.XShareError):
        X.block_quantize(x.to(DEV)[:, 1:161])                  # not 16-byte aligned
    with pytest.raises(X.XShareError):
        X.block_quantize(x.to(DEV)[:, :24])
    with pytest.raises(ValueError):
        X.block_quantize(x.to(DEV).t())
    with pytest.raises(ValueError):
        X.block_quantize(x.to(DEV).float())


# ------------------------------------------------------------------------- linear

def _bf16_close(y, ref, slack):
    err = np.abs(_f64(y) - ref)
    tol = slack + HALF_ULP * (np.abs(ref) + slack)
    assert (err <= tol).all(), float((err / np.maximum(tol, 1e-300)).max())


def _check_linear(x, q, s, y):
    xr, w = OB.rounded(_f64(x)), _oracle_weight(q, s)
    _bf16_close(y, xr @ w.T, OB.product_bound(xr, w))


SIZES = [(1, 16), (7, 112), (16, 128), (64, 144), (65, 256), (130, 272), (257, 640), (513, 1040),
         (1367, 720), (96, 2720)]


@pytest.mark.parametrize("n,k", SIZES)
@pytest.mark.parametrize("T", [1, 2, 15, 16, 17, 33, 64, 65, 129, 300])
def test_linear(T, n, k):
    from paper_2602_07265_amd import xshare as X
    rng = np.random.default_rng(T * 7 + n + k)
    x, (q, s) = _x(rng, T, k), _weight(rng, n, k)
    say(f"linear case T={T} n={n} k={k}")
    y = X.block_linear(x.to(DEV), q.to(DEV), s.to(DEV))
    _check_linear(x, q, s, y)
    codes, scales = X.block_quantize(x.to(DEV))
    again = X.block_linear(codes, q.to(DEV), s.to(DEV), x_scale=scales)
    assert torch.equal(y.view(torch.int16), again.view(torch.int16))


# sizes at which each form of the product is the one that is chosen (weight rows x tokens of a
# workgroup), from codes, so that none of them quantises its rows itself
@pytest.mark.parametrize("form,T,n,k", [
    ("16x16", 16, 1001, 656), ("32x16", 13, 5003, 272), ("16x32", 30, 2049, 400),
    ("32x32", 31, 5003, 272), ("64x32", 29, 14337, 144), ("32x32", 150, 1003, 912),
    ("64x64", 600, 1367, 272), ("128x64", 290, 4100, 272), ("128x128", 160, 14339, 144),
    ("128x256", 270, 14339, 144), ("256x256", 700, 13001, 144), ("128x128", 515, 16385, 128)])
def test_linear_forms(form, T, n, k):
    from paper_2602_07265_amd import xshare as X
    rng = np.random.default_rng(T + n)
    x, (q, s) = _x(rng, T, k), _weight(rng, n, k)
    say(f"linear case form {form} T={T} n={n} k={k}")
    codes, scales = X.block_quantize(x.to(DEV))
    _check_linear(x, q, s, X.block_linear(codes, q.to(DEV), s.to(DEV), x_scale=scales))


# rows that every workgroup quantises for itself: both widths of the workgroups (on both sides of
# 4096 weight rows), the longest rows and one step past them, the most rows and one more
@pytest.mark.parametrize("T,n,k", [(1, 14347, 160), (3, 4095, 272), (3, 4096, 272), (16, 300, 1024),
                                   (1, 77, 16384), (1, 77, 16400), (17, 300, 656), (5, 200, 3264),
                                   (16, 4129, 1024), (5, 4097, 272), (1, 77, 32784)])
def test_linear_quantised_by_the_product(T, n, k):
    from paper_2602_07265_amd import xshare as X
    rng = np.random.default_rng(T + n + k)
    x, (q, s) = _x(rng, T, k), _weight(rng, n, k)
    say(f"linear case own quantisation T={T} n={n} k={k}")
    _check_linear(x, q, s, X.block_linear(x.to(DEV), q.to(DEV), s.to(DEV)))


@pytest.mark.parametrize("T,n,k", [(3, 100, 272), (40, 131, 400), (150, 264, 1040)])
def test_linear_strided_guarded(T, n, k):
    """Rows apart in x and y, NaN around everything that is read."""
    from paper_2602_07265_amd import xshare as X
    rng = np.random.default_rng(T)
    ldx, ldy = k + 24, n + 5
    x, (q, s) = _x(rng, T, k), _weight(rng, n, k)
    gx, gq = Guarded(T * ldx * 2, IN_FILL), Guarded(n * k, IN_FILL)
    gs, gy = Guarded(s.numel() * 4, IN_FILL), Guarded(T * ldy * 2, OUT_FILL)
    need = X.block_linear_workspace_bytes(T, n, k)
    gw = Guarded(need, OUT_FILL)
    xv = gx.view(torch.bfloat16, (T, ldx))[:, :k]
    xv.copy_(x.to(DEV))
    qv, sv = gq.view(torch.uint8, (n, k)), gs.view(torch.float32, s.shape)
    qv.copy_(q.to(DEV))
    sv.copy_(s.to(DEV))
    whole = gy.view(torch.bfloat16, (T, ldy))
    say(f"linear case strided T={T} n={n} k={k}")
    X.block_linear(xv, qv, sv, y=whole[:, :n], workspace=gw.view(torch.uint8, (need,)))
    torch.cuda.synchronize()
    _check_linear(x, q, s, whole[:, :n])
    assert (whole[:, n:].contiguous().view(torch.uint8) == OUT_FILL).all()
    for g in (gx, gq, gs, gy, gw):
        assert g.intact()


@pytest.mark.parametrize("T", [5, 70, 200])
def test_linear_not_finite(T):
    """A NaN or infinity in x or in a weight's code reaches its own row or column only."""
    from paper_2602_07265_amd import xshare as X
    rng = np.random.default_rng(6)
    n, k = 200, 272
    x, (q, s) = _x(rng, T, k), _weight(rng, n, k)
    clean = X.block_linear(x.to(DEV), q.to(DEV), s.to(DEV))
    x[1, 271], x[3, 0] = float("nan"), float("inf")
    q[7, 0] = 0x7F
    q[150, 271] = 0xFF
    y = X.block_linear(x.to(DEV), q.to(DEV), s.to(DEV))
    bad = torch.zeros((T, n), dtype=torch.bool, device=DEV)
    bad[[1, 3]] = True
    bad[:, [7, 150]] = True
    assert torch.isnan(y[bad]).all()
    assert torch.equal(y[~bad], clean[~bad])


@pytest.mark.parametrize("T,n,k", [(4, 144, 96), (50, 272, 208)])
def test_linear_input_gradient(T, n, k):
    """dx = dy W is the call on the transposed weight: against the formula, and against differences
    of sum(y dy) along random directions in float64 of the same dequantised weight."""
    from paper_2602_07265_amd import xshare as X
    rng = np.random.default_rng(8)
    q, s = _weight(rng, n, k)
    dy = _x(rng, T, n)
    qt, st = q.to(DEV).t().contiguous(), s.to(DEV).t().contiguous()
    say(f"linear gradient case T={T} n={n} k={k}")
    dx = X.block_linear(dy.to(DEV), qt, st)
    w = _oracle_weight(q, s)
    dyr = OB.rounded(_f64(dy))
    _bf16_close(dx, dyr @ w, OB.product_bound(dyr, w.T))
    for _ in range(3):
        x, v = rng.normal(0, 1, (T, k)), rng.normal(0, 1, (T, k))
        slope = (((x + 0.5 * v) @ w.T - (x - 0.5 * v) @ w.T) * dyr).sum()
        size = np.abs(_f64(dx) * v).sum()
        assert abs(slope - (_f64(dx) * v).sum()) <= 2 * HALF_ULP * size


def test_linear_offsets_past_32_bits():
    from paper_2602_07265_amd import xshare as X
    rng = np.random.default_rng(10)
    n, k = 131, 1 << 20                       # rows of 1 MiB
    n_all = 2100                              # 2.2 GB of codes; the last rows hold the data
    say("linear case offsets past 32 bits")
    q = torch.zeros((n_all, k), dtype=torch.uint8, device=DEV)
    part = _codes(rng, n, 4096)
    q[n_all - n:, k - 4096:] = part.to(DEV)
    s = torch.full((-(-n_all // 128), k // 128), 1e-3, device=DEV)
    x = torch.zeros((2, k), dtype=torch.bfloat16, device=DEV)
    tail = _x(rng, 2, 4096)
    x[:, k - 4096:] = tail.to(DEV)
    ld = (1 << 31) + 8                        # y's second row lies past 2^31 elements
    buf = torch.empty(ld + n_all, dtype=torch.bfloat16, device=DEV)
    y = buf.as_strided((2, n_all), (ld, 1))
    X.block_linear(x, q, s, y=y)
    torch.cuda.synchronize()
    xr, w = OB.rounded(_f64(tail)), OB.VALUES[part.numpy()] * float(np.float32(1e-3))
    assert (y[:, :n_all - n] == 0).all()
    _bf16_close(y[:, n_all - n:].contiguous(), xr @ w.T,
                OB.product_bound(xr, w) + 8192 * 2.0 ** -23 * (np.abs(xr) @ np.abs(w).T))
    del q, buf, y
    torch.cuda.empty_cache()


def test_linear_refusals_and_empty():
    from paper_2602_07265_amd import xshare as X
    q, s = (t.to(DEV) for t in _weight(np.random.default_rng(0), 40, 32))
    x = torch.zeros((3, 32), dtype=torch.bfloat16, device=DEV)
    assert X.block_linear(x[:0], q, s).shape == (0, 40)
    for call in (lambda: X.block_linear(x, q[:, :16], s), lambda: X.block_linear(x, q, s[:0]),
                 lambda: X.block_linear(x.float(), q, s), lambda: X.block_linear(x, q.int(), s),
                 lambda: X.block_linear(x, q, s, y=torch.empty((2, 40), dtype=torch.bfloat16,
                                                               device=DEV)),
                 lambda: X.block_linear(x.t(), q, s)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(X.XShareError) as e:
        X.block_linear(x, q, s, workspace=torch.empty(16, dtype=torch.uint8, device=DEV))
    assert e.value.status == X.EWORKSPACE


# ------------------------------------------------------------------------- experts

def _expert_weights(rng, E, d, f):
    return [_weight(rng, E, f, d), _weight(rng, E, f, d), _weight(rng, E, d, f)]


def _run_experts(x, ids, w, mats, **kw):
    from paper_2602_07265_amd import xshare as X
    qs, ss = [m[0].to(DEV) for m in mats], [m[1].to(DEV) for m in mats]
    return X.block_experts(x.to(DEV), torch.from_numpy(ids.astype(np.int32)).to(DEV),
                           torch.from_numpy(w.astype(np.float32)).to(DEV), *qs, *ss, **kw)


def _check_experts(x, ids, w, mats, y):
    E = mats[0][0].shape[0]
    ref, term = OB.experts(_f64(x), ids, w.astype(np.float32),
                           lambda e: tuple(_oracle_weight(q[e], s[e]) for q, s in mats)
                           if 0 <= e < E else None)
    f = mats[0][0].shape[1]
    _bf16_close(y, ref, term / 8 + 2.0 ** -10 * term * np.sqrt(f))


def _routing(rng, T, E, k, share=1):
    ids = np.stack([rng.permutation(E * share)[:k] for _ in range(T)])
    ids = np.where(ids < E, ids, -1)
    w = rng.uniform(0, 1, (T, k))
    return ids, w / w.sum(1, keepdims=True)


@pytest.mark.parametrize("E,k,d,f", [(1, 1, 16, 16), (4, 2, 144, 112), (8, 2, 256, 128),
                                     (5, 3, 400, 272), (40, 8, 272, 144), (3, 2, 1040, 640)])
@pytest.mark.parametrize("T", [1, 2, 17, 40, 130])
def test_experts(T, E, k, d, f):
    rng = np.random.default_rng(T + E + d)
    x, mats = _x(rng, T, d), _expert_weights(rng, E, d, f)
    ids, w = _routing(rng, T, E, k)
    say(f"experts case T={T} E={E} k={k} d={d} f={f}")
    _check_experts(x, ids, w, mats, _run_experts(x, ids, w, mats))


@pytest.mark.parametrize("E,k,d,f", [(3, 2, 16384, 64), (3, 2, 16400, 64), (5, 4, 96, 8192),
                                     (5, 4, 96, 8208), (40, 32, 64, 1024)])
def test_experts_one_token_limits(E, k, d, f):
    """One token at the largest rows that its own form keeps in LDS, and one step past them."""
    rng = np.random.default_rng(d + f)
    x, mats = _x(rng, 1, d), _expert_weights(rng, E, d, f)
    ids, w = _routing(rng, 1, E, k)
    say(f"experts case one token E={E} k={k} d={d} f={f}")
    _check_experts(x, ids, w, mats, _run_experts(x, ids, w, mats))


@pytest.mark.parametrize("T", [9, 150])
def test_experts_missing_pairs(T):
    """Ids outside [0, E), tokens without pairs, experts without tokens, one expert with all."""
    rng = np.random.default_rng(12)
    E, k, d, f = 6, 4, 272, 144
    x, mats = _x(rng, T, d), _expert_weights(rng, E, d, f)
    ids, w = _routing(rng, T, E, k, share=3)
    ids[2], ids[5, 1], ids[7, 3] = -1, 6, -(1 << 31)
    say(f"experts case missing pairs T={T}")
    y = _run_experts(x, ids, w, mats)
    _check_experts(x, ids, w, mats, y)
    assert (y[2] == 0).all()
    ids[:] = -1
    assert (_run_experts(x, ids, w, mats) == 0).all()
    ids[:, 0] = 4
    _check_experts(x, ids, w, mats, _run_experts(x, ids, w, mats))
    # a pair that is left out reads neither its weight nor x's other rows: NaN there stays out
    x[3] = float("nan")
    w[5, 1:] = float("nan")
    y = _run_experts(x, ids, w, mats)
    assert torch.isnan(y[3]).all() and torch.isfinite(y[4:]).all()


# both products in tiles of 32 and of 128 tokens; gate/up alone in tiles (experts of few down
# columns), down alone in tiles (experts of few hidden units); down in tiles of 64 tokens
@pytest.mark.parametrize("forms,T,E,k,d,f", [
    ("32 / 32", 60, 100, 4, 528, 272), ("32 / few", 9, 160, 8, 272, 144),
    ("128 / 128", 480, 100, 4, 528, 272), ("128 / 128", 160, 10, 8, 5136, 1296),
    ("32 / few", 25, 50, 4, 144, 272), ("few / 32", 30, 50, 4, 1040, 112),
    ("128 / 64", 130, 12, 3, 272, 1040), ("few / 64", 60, 12, 3, 272, 144)])
def test_experts_forms(forms, T, E, k, d, f):
    rng = np.random.default_rng(T + E + d)
    x, mats = _x(rng, T, d), _expert_weights(rng, E, d, f)
    ids, w = _routing(rng, T, E, k)
    ids[: T // 3, 0] = 1                       # one expert holds many rows, another none
    ids[ids == E - 1] = -1
    ids[: T // 3, 1:] = np.where(ids[: T // 3, 1:] == 1, 2, ids[: T // 3, 1:])
    say(f"experts case forms {forms} T={T} E={E} k={k} d={d} f={f}")
    _check_experts(x, ids, w, mats, _run_experts(x, ids, w, mats))


def test_experts_on_a_given_stream_and_output():
    from paper_2602_07265_amd import xshare as X
    rng = np.random.default_rng(31)
    T, E, k, d, f = 21, 6, 2, 272, 144
    x, mats = _x(rng, T, d), _expert_weights(rng, E, d, f)
    ids, w = _routing(rng, T, E, k)
    y = torch.empty((T, d), dtype=torch.bfloat16, device=DEV)
    ws = torch.empty(X.block_experts_workspace_bytes(T, k, E, d, f), dtype=torch.uint8,
                     device=DEV)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        got = _run_experts(x, ids, w, mats, y=y, workspace=ws, stream=side)
    side.synchronize()
    assert got is y
    _check_experts(x, ids, w, mats, y)


def test_experts_large_batch_of_small_experts():
    """Thousands of pairs: rows of every expert over several tiles, in any order of ids."""
    rng = np.random.default_rng(13)
    T, E, k, d, f = 1100, 24, 4, 144, 80
    x, mats = _x(rng, T, d), _expert_weights(rng, E, d, f)
    ids, w = _routing(rng, T, E, k)
    ids[:400, 0] = 3                                # one expert holds many
    ids[:400, 1:] = np.where(ids[:400, 1:] == 3, 4, ids[:400, 1:])
    say("experts case large batch")
    _check_experts(x, ids, w, mats, _run_experts(x, ids, w, mats))


@pytest.mark.parametrize("T", [7, 90])
def test_experts_strided_guarded(T):
    from paper_2602_07265_amd import xshare as X
    rng = np.random.default_rng(T)
    E, k, d, f = 5, 2, 272, 208
    x, mats = _x(rng, T, d), _expert_weights(rng, E, d, f)
    ids, w = _routing(rng, T, E, k, share=2)
    bufs = []

    def read(t, dtype):
        g = Guarded(t.numel() * t.element_size(), IN_FILL)
        v = g.view(dtype, t.shape)
        v.copy_(t.to(DEV))
        bufs.append(g)
        return v

    ldx, ldy = d + 16, d + 8
    gx, gy = Guarded(T * ldx * 2, IN_FILL), Guarded(T * ldy * 2, OUT_FILL)
    xv = gx.view(torch.bfloat16, (T, ldx))[:, :d]
    xv.copy_(x.to(DEV))
    whole = gy.view(torch.bfloat16, (T, ldy))
    need = X.block_experts_workspace_bytes(T, k, E, d, f)
    gw = Guarded(need, OUT_FILL)
    bufs += [gx, gy, gw]
    say(f"experts case strided T={T}")
    X.block_experts(xv, read(torch.from_numpy(ids.astype(np.int32)), torch.int32),
                    read(torch.from_numpy(w.astype(np.float32)), torch.float32),
                    *(read(m[0], torch.uint8) for m in mats),
                    *(read(m[1], torch.float32) for m in mats), y=whole[:, :d],
                    workspace=gw.view(torch.uint8, (need,)))
    torch.cuda.synchronize()
    _check_experts(x, ids, w, mats, whole[:, :d])
    assert (whole[:, d:].contiguous().view(torch.uint8) == OUT_FILL).all()
    for g in bufs:
        assert g.intact()


def test_experts_offsets_past_32_bits():
    """The last of 40 experts of 59 MB a matrix: its weights lie past 2^31 bytes."""
    from paper_2602_07265_amd import xshare as X
    rng = np.random.default_rng(15)
    E, d, f, T = 40, 7168, 8192, 3
    say("experts case offsets past 32 bits")
    qs = [torch.zeros((E, *shape), dtype=torch.uint8, device=DEV)
          for shape in ((f, d), (f, d), (d, f))]
    mats = [_weight(rng, 1, *shape) for shape in ((f, d), (f, d), (d, f))]
    ss = []
    for q, m in zip(qs, mats):
        q[E - 1] = m[0][0].to(DEV)
        s = torch.zeros((E, *m[1].shape[1:]), device=DEV)
        s[E - 1] = m[1][0].to(DEV)
        ss.append(s)
    x = _x(rng, T, d)
    ids, w = np.full((T, 1), E - 1), np.ones((T, 1))
    y = X.block_experts(x.to(DEV), torch.from_numpy(ids.astype(np.int32)).to(DEV),
                        torch.from_numpy(w.astype(np.float32)).to(DEV), *qs, *ss)
    _check_experts(x, ids - (E - 1), w, mats, y)
    del qs, ss
    torch.cuda.empty_cache()


def test_experts_refusals_and_empty():
    from paper_2602_07265_amd import xshare as X
    rng = np.random.default_rng(0)
    E, k, d, f, T = 3, 2, 32, 48, 4
    x = _x(rng, T, d)
    mats = _expert_weights(rng, E, d, f)
    ids, w = _routing(rng, T, E, k)
    assert _run_experts(x[:0], ids[:0], w[:0], mats).shape == (0, d)
    with pytest.raises(ValueError):
        _run_experts(x.float(), ids, w, mats)
    with pytest.raises(ValueError):
        _run_experts(x, ids, w[:, :1], mats)
    with pytest.raises(ValueError):
        _run_experts(x, ids, w, [mats[0], mats[1], mats[0]])
    with pytest.raises(X.XShareError) as e:
        _run_experts(x, ids, w, mats, workspace=torch.empty(256, dtype=torch.uint8, device=DEV))
    assert e.value.status == X.EWORKSPACE
    with pytest.raises(X.XShareError):
        _run_experts(x, ids, w, mats, y=torch.empty((T, d + 4), dtype=torch.bfloat16,
                                                    device=DEV)[:, :d])


# ------------------------------------------------------------------------- as programs run them

def _layer(X, x, wg, bias, mats, shared, ws=None):
    """The layer a program makes of the operators: router, gate, routed experts, and a shared
    expert as the experts' one-expert form."""
    logits = X.router_logits(x, wg)
    g = X.gate(logits, 4, score="sigmoid", bias=bias, n_groups=4, top_groups=2,
               group_score="top2", scale=2.5)
    y = X.block_experts(x, g["ids"], g["w"], *(m[0] for m in mats), *(m[1] for m in mats))
    one = torch.zeros((x.shape[0], 1), dtype=torch.int32, device=DEV)
    s = X.block_experts(x, one, torch.ones((x.shape[0], 1), device=DEV),
                        *(m[0] for m in shared), *(m[1] for m in shared))
    return y, s


def _layer_inputs(seed, T, N, d, f):
    rng = np.random.default_rng(seed)
    dev = lambda ms: [(q.to(DEV), s.to(DEV)) for q, s in ms]  # noqa: E731
    return (torch.from_numpy(rng.normal(0, 0.1, (N, d)).astype(np.float32)).to(
                DEV, torch.bfloat16),
            torch.from_numpy(rng.normal(0, 0.05, N).astype(np.float32)).to(DEV),
            dev(_expert_weights(rng, N, d, f)), dev(_expert_weights(rng, 1, d, f)),
            [_x(rng, T, d).to(DEV) for _ in range(3)])


@pytest.mark.parametrize("T", [1, 24, 200])
def test_graph_replays_and_streams_match_eager(T):
    """Only kernels on the caller's stream: a captured layer replays, and two layers in flight on
    two streams give the same bits as one after the other."""
    from paper_2602_07265_amd import xshare as X
    wg, bias, mats, shared, xs = _layer_inputs(1, T, 16, 256, 144)
    bits = lambda r: [t.view(torch.int16).clone() for t in r]  # noqa: E731
    ref = [bits(_layer(X, x, wg, bias, mats, shared)) for x in xs]
    torch.cuda.synchronize()
    buf = xs[0].clone()
    say(f"blocks graph case T={T}: capture")
    g = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _layer(X, buf, wg, bias, mats, shared)
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        out = _layer(X, buf, wg, bias, mats, shared)
    for rep in range(3):
        for i, x in enumerate(xs):
            buf.copy_(x)
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(bits(out), ref[i])), (rep, i)
            again = bits(_layer(X, x, wg, bias, mats, shared))
            assert all(torch.equal(a, b) for a, b in zip(again, ref[i]))
    say(f"blocks stream case T={T}")
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [None, None]
    torch.cuda.synchronize()
    for _ in range(3):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i] = _layer(X, xs[i], wg, bias, mats, shared)
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(a, b) for a, b in zip(bits(got[i]), ref[i]))


@pytest.mark.parametrize("T", [1, 33, 300])
def test_rows_do_not_depend_on_their_neighbours(T):
    """A token's result is the same bits wherever it stands in the batch."""
    from paper_2602_07265_amd import xshare as X
    wg, bias, mats, shared, xs = _layer_inputs(2, T, 16, 288, 160)
    x = xs[0]
    a = _layer(X, x, wg, bias, mats, shared)
    turn = torch.randperm(T, device=DEV)
    b = _layer(X, x[turn].contiguous(), wg, bias, mats, shared)
    for u, v in zip(a, b):
        assert torch.equal(u[turn].view(torch.int16), v.view(torch.int16))


def test_set_selection_feeds_the_experts():
    """The batch-level selection's ids and weights are the experts' input as they are."""
    from paper_2602_07265_amd import xshare as X
    rng = np.random.default_rng(21)
    T, N, k, d, f = 20, 16, 4, 272, 144
    x, mats = _x(rng, T, d), _expert_weights(rng, N, d, f)
    h = torch.from_numpy(rng.normal(0, 1.5, (T, N)).astype(np.float32)).to(DEV)
    r = X.route(h, k, 1, 6)
    y = X.block_experts(x.to(DEV), r["ids"], r["w"], *(m[0].to(DEV) for m in mats),
                        *(m[1].to(DEV) for m in mats))
    assert int(r["stats"][0]) == 6
    _check_experts(x, r["ids"].cpu().numpy(), r["w"].cpu().numpy(), mats, y)
