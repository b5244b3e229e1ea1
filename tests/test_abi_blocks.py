"""What the routing by scores and the block-scaled FP8 products refuse, on the host: every call
below fails its checks, so it returns before any HIP call.  Fake pointers are never followed."""
import ctypes

import pytest
import torch

from paper_2602_07265_amd import xshare as X

FAKE = ctypes.c_void_p(1 << 20)
ODD = ctypes.c_void_p((1 << 20) + 2)
BIG = (1 << 20) + 16


def _gate(call="gate", dtype=0, T=8, ld=None, logits=FAKE, ids=FAKE, out=FAKE, **kw):
    f = dict(n_experts=64, top_k=4, score=1, n_groups=8, top_groups=4, group_score=1,
             renormalize=1, scale=2.5)
    f.update(kw)
    p = X.GateParams(**f)
    ld = p.n_experts if ld is None else ld
    if call == "gate":
        return X.lib().xshare_gate(logits, dtype, T, ld, None, ctypes.byref(p), ids, out, None)
    return X.lib().xshare_gate_backward(logits, dtype, T, ld, ctypes.byref(p), ids, FAKE, out,
                                        None)


BOTH = [(dict(T=-1), X.EINVAL), (dict(n_experts=0), X.EINVAL), (dict(top_k=0), X.EINVAL),
        (dict(top_k=65), X.EINVAL), (dict(score=2), X.EINVAL), (dict(dtype=2), X.EINVAL),
        (dict(ld=63), X.EINVAL), (dict(scale=float("nan")), X.EINVAL),
        (dict(scale=float("inf")), X.EINVAL), (dict(T=BIG), X.EUNSUPPORTED),
        (dict(n_experts=1032), X.EUNSUPPORTED),
        (dict(n_experts=256, top_k=33, top_groups=8), X.EUNSUPPORTED),
        (dict(logits=None), X.EINVAL), (dict(ids=None), X.EINVAL), (dict(out=None), X.EINVAL)]
CHOICE = [(dict(n_groups=0), X.EINVAL), (dict(n_groups=7), X.EINVAL),
          (dict(top_groups=0), X.EINVAL), (dict(top_groups=9), X.EINVAL),
          (dict(group_score=2), X.EINVAL), (dict(top_groups=1, top_k=9), X.EINVAL),
          (dict(n_groups=64, top_groups=8), X.EINVAL),        # two best of one expert
          (dict(n_experts=256, n_groups=128, top_groups=8), X.EUNSUPPORTED)]


@pytest.mark.parametrize("kw,status", BOTH + CHOICE)
def test_gate_refuses(kw, status):
    assert _gate(**kw) == status


@pytest.mark.parametrize("kw,status", BOTH)
def test_gate_backward_refuses(kw, status):
    assert _gate("backward", **kw) == status


def test_gate_without_tokens_or_parameters():
    assert _gate(T=0, logits=None, ids=None, out=None) == X.OK
    assert _gate("backward", T=0, logits=None, ids=None, out=None) == X.OK
    assert X.lib().xshare_gate(FAKE, 0, 1, 8, None, None, FAKE, FAKE, None) == X.EINVAL


def _quant(x=FAKE, rows=8, cols=256, ld=256, block_rows=1, q=FAKE, s=FAKE):
    return X.lib().xshare_block_quantize(x, rows, cols, ld, block_rows, q, s, None)


@pytest.mark.parametrize("kw,status", [
    (dict(x=None), X.EINVAL), (dict(q=None), X.EINVAL), (dict(s=None), X.EINVAL),
    (dict(x=ODD), X.EINVAL), (dict(q=ODD), X.EINVAL), (dict(s=ODD), X.EINVAL),
    (dict(rows=-1), X.EINVAL), (dict(cols=0), X.EINVAL), (dict(cols=248), X.EINVAL),
    (dict(ld=255), X.EINVAL), (dict(ld=260), X.EINVAL), (dict(block_rows=0), X.EINVAL),
    (dict(block_rows=64), X.EINVAL), (dict(rows=BIG), X.EUNSUPPORTED),
    (dict(cols=BIG, ld=BIG), X.EUNSUPPORTED), (dict(rows=0, x=None), X.OK)])
def test_quantize_refuses(kw, status):
    assert _quant(**kw) == status


def _linear(x=FAKE, ldx=256, xq=None, xs=None, T=8, n=100, k=256, wq=FAKE, s=FAKE, y=FAKE,
            ldy=100, ws=FAKE, ws_bytes=1 << 30):
    return X.lib().xshare_block_linear(x, ldx, xq, xs, T, n, k, wq, s, y, ldy, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,status", [
    (dict(x=None), X.EINVAL), (dict(x=None, xq=FAKE), X.EINVAL),
    (dict(x=None, xs=FAKE), X.EINVAL), (dict(xq=FAKE, xs=FAKE), X.EINVAL),
    (dict(x=None, xq=ODD, xs=FAKE), X.EINVAL), (dict(x=ODD), X.EINVAL),
    (dict(ldx=250), X.EINVAL), (dict(ldx=264 - 4), X.EINVAL), (dict(T=-1), X.EINVAL),
    (dict(n=0), X.EINVAL), (dict(k=0), X.EINVAL), (dict(k=24), X.EINVAL),
    (dict(wq=None), X.EINVAL), (dict(wq=ODD), X.EINVAL), (dict(s=None), X.EINVAL),
    (dict(y=None), X.EINVAL), (dict(ldy=99), X.EINVAL), (dict(T=BIG), X.EUNSUPPORTED),
    (dict(n=BIG, ldy=BIG), X.EUNSUPPORTED), (dict(k=BIG, ldx=BIG), X.EUNSUPPORTED),
    (dict(ws=None), X.EWORKSPACE), (dict(ws_bytes=100), X.EWORKSPACE),
    (dict(T=0, x=None, wq=None), X.OK)])
def test_linear_refuses(kw, status):
    assert _linear(**kw) == status


def _experts(**kw):
    f = dict(struct_size=ctypes.sizeof(X.BlockExpertsArgs), T=8, top_k=2, n_experts=4, d=256,
             f=128, ldx=256, ldy=256, ws_bytes=1 << 30)
    for name in ("x", "ids", "w", "w1", "w3", "w2", "w1_scale", "w3_scale", "w2_scale", "y",
                 "ws"):
        f[name] = FAKE
    f.update(kw)
    return X.lib().xshare_block_experts(ctypes.byref(X.BlockExpertsArgs(**f)))


@pytest.mark.parametrize("kw,status", [
    (dict(struct_size=8), X.EINVAL), (dict(T=-1), X.EINVAL), (dict(top_k=0), X.EINVAL),
    (dict(n_experts=0), X.EINVAL), (dict(d=0), X.EINVAL), (dict(f=0), X.EINVAL),
    (dict(d=248), X.EINVAL), (dict(f=120), X.EINVAL), (dict(ldx=255), X.EINVAL),
    (dict(ldy=255), X.EINVAL), (dict(ldy=260), X.EINVAL), (dict(x=ODD), X.EINVAL),
    (dict(y=ODD), X.EINVAL), (dict(w1=ODD), X.EINVAL), (dict(w3=ODD), X.EINVAL),
    (dict(w2=ODD), X.EINVAL), (dict(n_experts=1025), X.EUNSUPPORTED),
    (dict(top_k=33), X.EUNSUPPORTED), (dict(T=BIG), X.EUNSUPPORTED),
    (dict(T=1 << 19, top_k=4), X.EUNSUPPORTED), (dict(f=BIG), X.EUNSUPPORTED),
    (dict(d=BIG, ldx=BIG, ldy=BIG), X.EUNSUPPORTED), (dict(ws=None), X.EWORKSPACE),
    (dict(ws_bytes=1000), X.EWORKSPACE), (dict(T=0, x=None, ws=None), X.OK)]
    + [({n: None}, X.EINVAL) for n in ("x", "ids", "w", "w1", "w3", "w2", "w1_scale",
                                       "w3_scale", "w2_scale", "y")])
def test_experts_refuse(kw, status):
    assert _experts(**kw) == status
    assert X.lib().xshare_block_experts(None) == X.EINVAL


def test_workspace_sizes():
    a = X.block_linear_workspace_bytes(7, 100, 272)
    assert a % 256 == 0 and a >= 7 * 272 + 7 * 3 * 4
    assert X.block_linear_workspace_bytes(7, 0, 272) == 0
    assert X.block_linear_workspace_bytes(7, 100, 24) == 0
    b = X.block_experts_workspace_bytes(7, 2, 4, 256, 128)
    assert b % 256 == 0 and b >= 7 * 256 + 14 * (128 + 4 * 256)
    assert X.block_experts_workspace_bytes(7, 2, 4, 250, 128) == 0
    assert X.block_experts_workspace_bytes(7, 33, 64, 256, 128) == 0


def test_binding_refuses_host_tensors():
    cpu = torch.zeros((4, 32), dtype=torch.float32)
    x = torch.zeros((4, 32), dtype=torch.bfloat16)
    codes, scales = torch.zeros((32, 32), dtype=torch.uint8), torch.zeros((1, 1))
    for call in (lambda: X.gate(cpu, 2), lambda: X.gate(cpu.double(), 2),
                 lambda: X.gate_backward(cpu, torch.zeros((4, 2), dtype=torch.int32),
                                         torch.zeros((4, 2))),
                 lambda: X.block_quantize(x), lambda: X.block_linear(x, codes, scales),
                 lambda: X.block_experts(x, torch.zeros((4, 2), dtype=torch.int32),
                                         torch.zeros((4, 2)), codes[None], codes[None],
                                         codes[None], scales[None], scales[None],
                                         scales[None])):
        with pytest.raises(ValueError):
            call()
