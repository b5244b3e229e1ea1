"""What the expert order, the moves, the products of groups of rows and the adapters refuse, on the
host: every call below fails its checks, so it returns before any HIP call.  Fake pointers are never
followed."""
import ctypes

import pytest
import torch

from paper_2602_07265_amd import xshare as X
from test_block_sizes import BIG as PAST
from test_block_sizes import OnGpu

FAKE = ctypes.c_void_p(1 << 20)
FAR = ctypes.c_void_p(1 << 30)
ODD = ctypes.c_void_p((1 << 20) + 1)
OFF8 = ctypes.c_void_p((1 << 20) + 8)
BIG = (1 << 20) + 8


def _order(ids=FAKE, T=8, k=2, E=16, offsets=FAKE, rows=FAKE, pairs=FAKE, ws=FAKE,
           ws_bytes=1 << 30):
    return X.lib().xshare_expert_order(ids, T, k, E, offsets, rows, pairs, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,status", [
    (dict(T=-1), X.EINVAL), (dict(k=0), X.EINVAL), (dict(E=0), X.EINVAL),
    (dict(T=BIG), X.EUNSUPPORTED), (dict(k=33), X.EUNSUPPORTED), (dict(E=1025), X.EUNSUPPORTED),
    (dict(T=1 << 19, k=3), X.EUNSUPPORTED), (dict(ids=None), X.EINVAL), (dict(ids=ODD), X.EINVAL),
    (dict(offsets=None), X.EINVAL), (dict(T=0, offsets=None), X.EINVAL), (dict(rows=None), X.EINVAL),
    (dict(pairs=None), X.EINVAL), (dict(pairs=ODD), X.EINVAL),
    (dict(T=8192, ws=None), X.EWORKSPACE), (dict(T=8192, ws_bytes=255), X.EWORKSPACE),
    (dict(T=8192, ws=OFF8), X.EINVAL)])
def test_order_refuses(kw, status):
    assert _order(**kw) == status


def _dispatch(x=FAKE, ldx=40, dtype=0, T=8, k=2, d=40, rows=FAKE, out=FAR, ld_out=40):
    return X.lib().xshare_dispatch(x, ldx, dtype, T, k, d, rows, out, ld_out, None)


def _combine(src=FAKE, ld=40, dtype=0, T=8, k=2, d=40, rows=FAKE, w=FAKE, y=FAR, ldy=40):
    return X.lib().xshare_combine(src, ld, dtype, T, k, d, rows, w, y, ldy, None)


def _backward(dy=FAKE, lddy=40, src=FAKE, ld=40, dtype=0, T=8, k=2, d=40, rows=FAKE, w=FAKE,
              dsrc=FAR, ldd=40, dw=FAKE):
    return X.lib().xshare_combine_backward(dy, lddy, src, ld, dtype, T, k, d, rows, w, dsrc, ldd, dw,
                                           None)


MOVES = [(dict(dtype=2), X.EINVAL), (dict(T=-1), X.EINVAL), (dict(k=0), X.EINVAL),
         (dict(d=0), X.EINVAL), (dict(T=BIG), X.EUNSUPPORTED), (dict(k=33), X.EUNSUPPORTED),
         (dict(d=BIG), X.EUNSUPPORTED), (dict(T=1 << 19, k=3), X.EUNSUPPORTED),
         (dict(rows=None), X.EINVAL), (dict(rows=ODD), X.EINVAL), (dict(d=41), X.EINVAL)]


@pytest.mark.parametrize("call", [_dispatch, _combine, _backward])
@pytest.mark.parametrize("kw,status", MOVES)
def test_moves_refuse(call, kw, status):
    assert call(**kw) == status
    assert call(T=0, rows=None) == X.OK


@pytest.mark.parametrize("call,kw,status", [
    (_dispatch, dict(x=None), X.EINVAL), (_dispatch, dict(x=ODD), X.EINVAL),
    (_dispatch, dict(x=ODD, dtype=1), X.EINVAL), (_dispatch, dict(ldx=39), X.EINVAL),
    (_dispatch, dict(out=None), X.EINVAL), (_dispatch, dict(ld_out=39), X.EINVAL),
    (_combine, dict(src=None), X.EINVAL), (_combine, dict(w=ODD), X.EINVAL),
    (_combine, dict(y=None), X.EINVAL), (_combine, dict(ldy=39), X.EINVAL),
    (_backward, dict(dy=None), X.EINVAL), (_backward, dict(src=None), X.EINVAL),
    (_backward, dict(dsrc=None), X.EINVAL), (_backward, dict(ldd=39), X.EINVAL),
    (_backward, dict(w=None), X.EINVAL), (_backward, dict(dw=None), X.EINVAL)])
def test_a_move_refuses(call, kw, status):
    assert call(**kw) == status


def _linear(x=FAKE, ldx=64, w=FAKE, offsets=FAKE, P=8, E=4, n=40, k=64, y=FAR, ldy=40, ws=FAKE,
            ws_bytes=1 << 30):
    return X.lib().xshare_grouped_linear(x, ldx, w, offsets, P, E, n, k, y, ldy, ws, ws_bytes, None)


def _linear_x(x=FAKE, ldx=64, w=FAKE, offsets=FAKE, P=8, E=4, n=64, k=40, y=FAR, ldy=40, ws=FAKE,
              ws_bytes=1 << 30):
    return X.lib().xshare_grouped_linear_backward_x(x, ldx, w, offsets, P, E, n, k, y, ldy, ws,
                                                    ws_bytes, None)


def _linear_w(dy=FAKE, lddy=40, x=FAKE, ldx=64, offsets=FAKE, P=8, E=4, n=40, k=64, dw=FAKE, dtype=0,
              accumulate=0, ws=FAKE, ws_bytes=1 << 30):
    return X.lib().xshare_grouped_linear_backward_w(dy, lddy, x, ldx, offsets, P, E, n, k, dw, dtype,
                                                    accumulate, ws, ws_bytes, None)


SIZES = [(dict(P=-1), X.EINVAL), (dict(E=0), X.EINVAL), (dict(n=0), X.EINVAL), (dict(k=0), X.EINVAL),
         (dict(n=36), X.EINVAL), (dict(k=60), X.EINVAL), (dict(P=BIG), X.EUNSUPPORTED),
         (dict(E=1025), X.EUNSUPPORTED), (dict(n=BIG), X.EUNSUPPORTED), (dict(k=BIG), X.EUNSUPPORTED),
         (dict(offsets=None), X.EINVAL), (dict(offsets=ODD), X.EINVAL), (dict(x=None), X.EINVAL),
         (dict(x=OFF8), X.EINVAL), (dict(ldx=32), X.EINVAL), (dict(ldx=68), X.EINVAL),
         (dict(P=256, ws=None), X.EWORKSPACE), (dict(P=256, ws_bytes=1 << 20), X.EWORKSPACE),
         (dict(P=256, ws=OFF8), X.EINVAL)]


@pytest.mark.parametrize("call", [_linear, _linear_x, _linear_w])
@pytest.mark.parametrize("kw,status", SIZES)
def test_products_refuse(call, kw, status):
    assert call(**kw) == status


@pytest.mark.parametrize("call,kw,status", [
    (_linear, dict(w=None), X.EINVAL), (_linear, dict(w=OFF8), X.EINVAL),
    (_linear, dict(y=OFF8), X.EINVAL), (_linear, dict(ldy=44), X.EINVAL),
    (_linear, dict(ldx=(1 << 22) + 8), X.EUNSUPPORTED), (_linear, dict(P=0, x=None), X.OK),
    (_linear_x, dict(w=OFF8), X.EINVAL), (_linear_x, dict(y=None), X.EINVAL),
    (_linear_x, dict(ldx=(1 << 22) + 8), X.EUNSUPPORTED), (_linear_x, dict(P=0, x=None), X.OK),
    (_linear_w, dict(dy=None), X.EINVAL), (_linear_w, dict(lddy=32), X.EINVAL),
    (_linear_w, dict(dw=None), X.EINVAL), (_linear_w, dict(dw=OFF8), X.EINVAL),
    (_linear_w, dict(ldx=(1 << 22) + 8), X.EUNSUPPORTED),
    (_linear_w, dict(lddy=(1 << 22) + 8), X.EUNSUPPORTED), (_linear_w, dict(dtype=2), X.EINVAL), (_linear_w, dict(dtype=1, accumulate=1), X.EUNSUPPORTED)])
def test_a_product_refuses(call, kw, status):
    assert call(**kw) == status


def _adapters(call, **kw):
    f = dict(struct_size=ctypes.sizeof(X.AdaptersArgs), T=8, n_adapters=4, rank=16, n=40, d=40,
             ldx=40, ld_base=40, ld_out=40, lddy=40, ws_bytes=1 << 30)
    for name in ("x", "a", "b", "ids", "scales", "base", "out", "dy", "da", "db", "ws"):
        f[name] = FAKE
    f["out"] = FAR
    f.update(kw)
    return getattr(X.lib(), call)(ctypes.byref(X.AdaptersArgs(**f)))


@pytest.mark.parametrize("call", ["xshare_adapters", "xshare_adapters_backward"])
@pytest.mark.parametrize("kw,status", [
    (dict(struct_size=8), X.EINVAL), (dict(T=-1), X.EINVAL), (dict(n_adapters=0), X.EINVAL),
    (dict(rank=0), X.EINVAL), (dict(rank=12), X.EINVAL), (dict(n=44), X.EINVAL),
    (dict(d=44), X.EINVAL), (dict(rank=136), X.EUNSUPPORTED), (dict(T=BIG), X.EUNSUPPORTED),
    (dict(n_adapters=1025), X.EUNSUPPORTED), (dict(n=BIG), X.EUNSUPPORTED),
    (dict(d=BIG), X.EUNSUPPORTED), (dict(x=None), X.EINVAL), (dict(x=OFF8), X.EINVAL),
    (dict(ldx=32), X.EINVAL), (dict(ldx=44), X.EINVAL), (dict(a=None), X.EINVAL),
    (dict(b=OFF8), X.EINVAL), (dict(ids=None), X.EINVAL), (dict(scales=ODD), X.EINVAL),
    (dict(base=OFF8), X.EINVAL), (dict(ld_base=32), X.EINVAL), (dict(base=FAR, ld_base=48), X.EINVAL),
    (dict(out=None), X.EINVAL), (dict(ld_out=32), X.EINVAL), (dict(ws=None), X.EWORKSPACE),
    (dict(ws_bytes=512), X.EWORKSPACE), (dict(ws=OFF8), X.EINVAL)])
def test_adapters_refuse(call, kw, status):
    assert _adapters(call, **kw) == status
    assert getattr(X.lib(), call)(None) == X.EINVAL


@pytest.mark.parametrize("kw", [dict(dy=None), dict(lddy=32), dict(da=None), dict(db=OFF8)])
def test_adapters_backward_refuses(kw):
    assert _adapters("xshare_adapters_backward", **kw) == X.EINVAL


def _past(elements, at=FAKE, size=2):
    return ctypes.c_void_p(at.value + elements * size)


@pytest.mark.parametrize("call", [
    lambda: _dispatch(out=FAKE, dtype=1), lambda: _dispatch(out=_past(8 * 40 - 1), dtype=1),
    lambda: _dispatch(x=_past(16 * 40 - 1, FAR, 4)), lambda: _combine(y=FAKE, k=1, dtype=1),
    lambda: _combine(src=_past(8 * 40 - 1, FAR, 4)), lambda: _backward(dy=FAR, dtype=1),
    lambda: _backward(dsrc=FAKE, src=FAR, dy=_past(16 * 40 - 1, FAKE, 4)),
    lambda: _backward(dsrc=FAKE, src=_past(40, FAKE, 4), dy=FAR),
    lambda: _backward(dsrc=FAKE, ldd=48, dy=FAR), lambda: _linear(y=FAKE, ldy=64),
    lambda: _linear(y=_past(7 * 64 + 56)), lambda: _linear(x=_past(32), ldx=104, y=FAKE, ldy=104),
    lambda: _linear(x=FAKE, ldx=104, y=_past(3 * 104 + 56), ldy=104),
    lambda: _linear_x(y=FAKE, ldy=64),
    lambda: _linear_x(y=_past(7 * 64 + 56)), lambda: _adapters("xshare_adapters", out=FAKE),
    lambda: _adapters("xshare_adapters", out=FAKE, base=FAR, x=_past(7 * 40 + 32)),
    lambda: _adapters("xshare_adapters", out=FAKE, base=_past(40), x=FAR),
    lambda: _adapters("xshare_adapters", out=FAKE, ld_base=48, x=FAR),
    lambda: _adapters("xshare_adapters_backward", x=FAR, dy=FAR, out=FAKE, base=_past(8)),
    lambda: _adapters("xshare_adapters_backward", x=FAR, base=None, out=FAKE),
    lambda: _adapters("xshare_adapters_backward", dy=FAR, base=None, out=FAKE)])
def test_outputs_over_inputs(call):
    assert call() == X.EINVAL


def test_workspaces_serve_smaller_batches():
    assert X.expert_order_workspace_bytes(512, 8, 300) == 0
    edges = [X.expert_order_workspace_bytes(T, 1, 300) for T in (4097, 65536, 65537, 524288, 1 << 20)]
    assert edges == sorted(edges) and edges[0] > 0
    a = [X.adapters_workspace_bytes(T, 5, 24, 400, 4096, True) for T in range(0, 9000, 37)]
    o = [X.expert_order_workspace_bytes(T, 8, 300) for T in range(0, 9000, 37)]
    p = [X.grouped_linear_workspace_bytes(P, 8, 40, 64) for P in range(0, 9000, 37)]
    assert p == sorted(p) and p[0] == 0 and p[-1] == 64 << 20
    assert X.grouped_linear_workspace_bytes(4096, 8, 40, 60) == 0
    assert X.grouped_linear_workspace_bytes(PAST, 8, 40, 64) == 0
    for sizes in (a, o):
        assert all(s % 256 == 0 for s in sizes) and sizes == sorted(sizes)
    assert a[0] > 0 and o[0] == 0 and o[-1] > 0
    # h and dh: three bf16 parts of 16, 32, 64 or 128 ranks a token
    for r, wide in ((8, 16), (24, 32), (40, 64), (72, 128), (104, 128)):
        T = 1 << 16
        big, small = (X.adapters_workspace_bytes(n, 1, r, 64, 64, True) for n in (T, T // 2))
        order = X.expert_order_workspace_bytes(T, 1, 1) - X.expert_order_workspace_bytes(T // 2, 1, 1)
        parts = [min(511 // 2, -(-n // 256)) for n in (T, T // 2)]
        assert big - small == 2 * 6 * (T // 2) * wide + 8 * (T // 2) + order \
            + 4 * r * 128 * (parts[0] - parts[1])
    assert X.adapters_workspace_bytes(8, 5, 12, 400, 4096) == 0
    assert X.expert_order_workspace_bytes(8, 33, 300) == 0
    assert X.adapters_workspace_bytes(PAST, 5, 16, 400, 4096) == 0
    assert X.expert_order_workspace_bytes(8, 2, PAST) == 0


def _t(dtype, *shape, grad=False):
    return torch.empty(shape, dtype=dtype, device="meta").as_subclass(OnGpu).requires_grad_(grad)


BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32


def _order_of(T, k):
    return dict(rows=_t(I32, T, k))


@pytest.mark.parametrize("call,name", [
    (lambda: X.dispatch(_t(BF, 4, 16, grad=True), _order_of(4, 2)), "x"),
    (lambda: X.combine(_t(BF, 8, 16, grad=True), _t(F32, 4, 2), _order_of(4, 2)), "rows"),
    (lambda: X.combine(_t(BF, 8, 16), _t(F32, 4, 2, grad=True), _order_of(4, 2)), "w"),
    (lambda: X.grouped_linear(_t(BF, 4, 16, grad=True), _t(BF, 2, 8, 16), _t(I32, 3)), "x"),
    (lambda: X.grouped_linear(_t(BF, 4, 16), _t(BF, 2, 8, 16, grad=True), _t(I32, 3)), "w"),
    (lambda: X.adapters(_t(BF, 4, 16), _t(BF, 2, 8, 16, grad=True), _t(BF, 2, 8, 8), _t(I32, 4)),
     "a"),
    (lambda: X.adapters(_t(BF, 4, 16), _t(BF, 2, 8, 16), _t(BF, 2, 8, 8), _t(I32, 4),
                        scales=_t(F32, 2, grad=True)), "scales")])
def test_a_gradient_is_not_dropped_without_a_word(call, name):
    with pytest.raises(ValueError, match=f"{name} requires a gradient"):
        call()


@pytest.mark.parametrize("call", [
    lambda: X.expert_order(_t(I32, 4, 2), PAST),
    lambda: X.dispatch(_t(BF, PAST, 16), _order_of(PAST, 2)),
    lambda: X.dispatch_backward(_t(BF, 8, PAST), _order_of(4, 2)),
    lambda: X.grouped_linear(_t(BF, PAST, 16), _t(BF, 2, 8, 16), _t(I32, 3)),
    lambda: X.grouped_linear_backward_w(_t(BF, 4, 8), _t(BF, 4, 16), _t(I32, PAST)),
    lambda: X.adapters(_t(BF, PAST, 16), _t(BF, 2, 8, 16), _t(BF, 2, 8, 8), _t(I32, PAST))])
def test_sizes_past_32_bits(call):
    with pytest.raises(X.XShareError) as e:
        call()
    assert e.value.status == X.EUNSUPPORTED


@pytest.mark.parametrize("call,match", [
    (lambda: X.dispatch(_t(BF, 5, 16), _order_of(4, 2)), "4 rows"),
    (lambda: X.dispatch(_t(torch.float16, 4, 16), _order_of(4, 2)), "float32 or bfloat16"),
    (lambda: X.dispatch(_t(BF, 4, 16), _order_of(4, 2), out=_t(F32, 8, 16)), "bfloat16"),
    (lambda: X.combine(_t(BF, 7, 16), _t(F32, 4, 2), _order_of(4, 2)), "8 rows"),
    (lambda: X.combine(_t(BF, 8, 16), _t(F32, 4, 3), _order_of(4, 2)), "shape"),
    (lambda: X.combine(_t(BF, 8, 16), None, _order_of(4, 2)), "w must be"),
    (lambda: X.combine_backward(_t(BF, 4, 16), _t(F32, 8, 16), _t(F32, 4, 2), _order_of(4, 2)),
     "bfloat16"),
    (lambda: X.grouped_linear(_t(BF, 4, 24), _t(BF, 2, 8, 16), _t(I32, 3)), "16 columns"),
    (lambda: X.grouped_linear(_t(BF, 4, 16), _t(BF, 2, 8, 16), _t(I32, 4)), "shape"),
    (lambda: X.grouped_linear(_t(F32, 4, 16), _t(BF, 2, 8, 16), _t(I32, 3)), "bfloat16"),
    (lambda: X.grouped_linear_backward_w(_t(BF, 4, 8), _t(BF, 5, 16), _t(I32, 3)), "4 rows"),
    (lambda: X.grouped_linear_backward_w(_t(BF, 4, 8), _t(BF, 4, 16), _t(I32, 3), accumulate=True),
     "accumulate"),
    (lambda: X.adapters(_t(BF, 4, 16), _t(BF, 2, 8, 16), _t(BF, 2, 8, 16), _t(I32, 4)), "shape"),
    (lambda: X.adapters(_t(BF, 4, 16), _t(BF, 2, 8, 16), _t(BF, 2, 8, 8), _t(I32, 4),
                        base=_t(BF, 3, 8)), "4 rows")])
def test_binding_refuses(call, match):
    with pytest.raises(ValueError, match=match):
        call()


def test_binding_refuses_host_tensors():
    x, ids = torch.zeros((4, 16), dtype=BF), torch.zeros((4, 2), dtype=I32)
    w, off = torch.zeros((2, 8, 16), dtype=BF), torch.zeros(3, dtype=I32)
    order = dict(rows=ids)
    for call in (lambda: X.expert_order(ids, 2), lambda: X.dispatch(x, order),
                 lambda: X.dispatch_backward(x, order),
                 lambda: X.combine(x, torch.zeros((4, 2)), order),
                 lambda: X.combine_backward(x, x, torch.zeros((4, 2)), order),
                 lambda: X.grouped_linear(x, w, off),
                 lambda: X.grouped_linear_backward_x(x, w, off),
                 lambda: X.grouped_linear_backward_w(x, x, off),
                 lambda: X.adapters(x, w, w, ids[:, 0].contiguous()),
                 lambda: X.adapters_backward(x, x, w, w, ids[:, 0].contiguous())):
        with pytest.raises(ValueError):
            call()
