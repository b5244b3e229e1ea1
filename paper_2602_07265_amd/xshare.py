"""Python binding of libxshare.so (argument marshalling only).

Every computation runs in the HIP kernels behind the C ABI of include/xshare.h; this module
checks tensor devices/dtypes/shapes, carves nothing itself except the workspace tensor it
allocates when none is passed, and forwards raw device pointers plus the current HIP stream.
There is no fallback: if the library is not built or no GPU is present, calls raise.

A call with ``stream=`` works on that stream, and what it allocates (workspace, outputs) comes from
that stream's memory.  It does not wait for the current stream; tensors given to it must live
until ``stream`` has passed the call (``Tensor.record_stream``), as for torch's own operations.
"""
from __future__ import annotations

import ctypes
import functools
import inspect
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libxshare.so")
# the profiling build (block timeline of the expert GEMMs, xshare_block_times)
TIMELINE_LIB_PATH = os.path.join(_HERE, "libxshare_timeline.so")
TIME_BLOCKS, TIME_SEQ_BLOCKS, TIME_SEQ_STRIDE = 16384, 1024, 33   # XSHARE_TIME_*

OK, EINVAL, EUNSUPPORTED, EWORKSPACE, EHIP = 0, 1, 2, 3, 4
BUDGET = {"total": 0, "extra": 1, "per_group": 2, "threshold": 3}
SCORE = {"topk": 0, "dense": 1}
N_STAGE_EVENTS = 5
NOALLOC_SCRATCH_BYTES = 64 << 20     # XSHARE_NOALLOC_SCRATCH_BYTES
STAGES = ("route", "gate_up", "down", "combine")


def _placed(call):
    """``call``, run where it belongs.

    The device of its first argument is made current for it: a kernel goes to the current device,
    whatever its arguments' device is.  ``stream``, where it is another one than that device's current
    stream, is made current too: what the call allocates or copies itself belongs to the stream
    that works on it, so that no later allocation of the caller's stream gets memory that is
    still in use there.  What it returns may be used and dropped on the caller's stream (after
    waiting for ``stream``)."""
    names = list(inspect.signature(call).parameters)
    first, at = names[0], names.index("stream")

    def on_device(i, *args, **kw):
        if i < 0 or i == torch._C._cuda_getDevice():
            return call(*args, **kw)
        with torch.cuda.device(i):
            return call(*args, **kw)

    @functools.wraps(call)
    def placed(*args, **kw):
        stream = args[at] if len(args) > at else kw.get("stream")
        try:
            i = (args[0] if args else kw[first]).get_device()
        except (AttributeError, KeyError):
            i = -1                                        # not a GPU tensor: not for here to say
        if stream is None:
            if i < 0 or i == torch._C._cuda_getDevice():  # (nearly always, and at once)
                return call(*args, **kw)
            return on_device(i, *args, **kw)
        if not isinstance(stream, torch.cuda.Stream):     # any object that holds a handle
            stream = torch.cuda.ExternalStream(stream.cuda_stream, None if i < 0 else i)
        if 0 <= i != stream.device.index:
            raise ValueError(f"{first} is on cuda:{i}, the stream on {stream.device}")
        own = torch.cuda.current_stream(stream.device)
        if own.cuda_stream == stream.cuda_stream:
            return on_device(i, *args, **kw)
        with torch.cuda.stream(stream):                   # (its device too)
            res = call(*args, **kw)
        for t in res.values() if isinstance(res, dict) else \
                res if isinstance(res, tuple) else (res,):
            if isinstance(t, torch.Tensor) and t.is_cuda:
                t.record_stream(own)
        return res
    return placed


class RouteParams(ctypes.Structure):
    _fields_ = [
        ("n_experts", ctypes.c_int32),
        ("top_k", ctypes.c_int32),
        ("warmup_k0", ctypes.c_int32),
        ("budget", ctypes.c_int32),
        ("budget_mode", ctypes.c_int32),
        ("score_mode", ctypes.c_int32),
        ("per_request_budget", ctypes.c_int32),
        ("threshold", ctypes.c_float),
        ("ledger", ctypes.c_void_p),
    ]


class EpLayout(ctypes.Structure):
    _fields_ = [
        ("n_groups", ctypes.c_int32),
        ("local_group", ctypes.c_int32),
        ("expert_group", ctypes.c_void_p),
        ("host_expert_group", ctypes.c_void_p),
    ]


class SharedExperts(ctypes.Structure):
    _fields_ = [
        ("n_shared", ctypes.c_int32),
        ("w1", ctypes.c_void_p),
        ("w3", ctypes.c_void_p),
        ("w2", ctypes.c_void_p),
    ]


class LayerArgs(ctypes.Structure):
    """xshare_layer_args (include/xshare.h), the argument struct of xshare_moe_forward_v2."""
    _fields_ = [
        ("struct_size", ctypes.c_size_t),
        ("T", ctypes.c_int32), ("d", ctypes.c_int32), ("f", ctypes.c_int32),
        ("x", ctypes.c_void_p), ("logits", ctypes.c_void_p), ("w_gate", ctypes.c_void_p),
        ("weight_format", ctypes.c_int32),
        ("w1", ctypes.c_void_p), ("w3", ctypes.c_void_p), ("w2", ctypes.c_void_p),
        ("w1_scale", ctypes.c_void_p), ("w3_scale", ctypes.c_void_p),
        ("w2_scale", ctypes.c_void_p),
        ("params", ctypes.POINTER(RouteParams)),
        ("req_offsets", ctypes.c_void_p), ("host_offsets", ctypes.c_void_p),
        ("R", ctypes.c_int32),
        ("ep", ctypes.POINTER(EpLayout)), ("shared", ctypes.POINTER(SharedExperts)),
        ("y", ctypes.c_void_p), ("logits_out", ctypes.c_void_p), ("sel_mask", ctypes.c_void_p),
        ("topk_ids", ctypes.c_void_p), ("topk_w", ctypes.c_void_p), ("stats", ctypes.c_void_p),
        ("ws", ctypes.c_void_p), ("ws_bytes", ctypes.c_size_t),
        ("stage_events", ctypes.c_void_p),
        ("stream", ctypes.c_void_p),
    ]


class GateParams(ctypes.Structure):
    """xshare_gate_params (include/xshare.h)."""
    _fields_ = [
        ("n_experts", ctypes.c_int32), ("top_k", ctypes.c_int32), ("score", ctypes.c_int32),
        ("n_groups", ctypes.c_int32), ("top_groups", ctypes.c_int32),
        ("group_score", ctypes.c_int32), ("renormalize", ctypes.c_int32),
        ("scale", ctypes.c_float),
    ]


class BlockExpertsArgs(ctypes.Structure):
    """xshare_block_experts_args (include/xshare.h)."""
    _fields_ = [
        ("struct_size", ctypes.c_size_t),
        ("T", ctypes.c_int32), ("top_k", ctypes.c_int32), ("n_experts", ctypes.c_int32),
        ("d", ctypes.c_int32), ("f", ctypes.c_int32),
        ("x", ctypes.c_void_p), ("ldx", ctypes.c_int64),
        ("ids", ctypes.c_void_p), ("w", ctypes.c_void_p),
        ("w1", ctypes.c_void_p), ("w3", ctypes.c_void_p), ("w2", ctypes.c_void_p),
        ("w1_scale", ctypes.c_void_p), ("w3_scale", ctypes.c_void_p),
        ("w2_scale", ctypes.c_void_p),
        ("y", ctypes.c_void_p), ("ldy", ctypes.c_int64),
        ("ws", ctypes.c_void_p), ("ws_bytes", ctypes.c_size_t),
        ("stream", ctypes.c_void_p),
    ]


WEIGHTS = {"bf16": 0, "fp8": 1, "mxfp4": 2}
_EXPERTS_ARGS_BYTES = ctypes.sizeof(BlockExpertsArgs)
GATE = {"softmax": 0, "sigmoid": 1}
GROUP = {"max": 0, "top2": 1}

STATS_FIELDS = ("n_selected", "n_active", "n_vanilla_union", "n_warmup", "n_start",
                "budget_eff", "max_group_load")


class XShareError(RuntimeError):
    def __init__(self, status: int, what: str):
        super().__init__(f"{what}: {status_string(status)} ({status})")
        self.status = status


_lib = None
_P = ctypes.c_void_p
_I32 = ctypes.c_int32
_I64 = ctypes.c_int64
_SZ = ctypes.c_size_t


def lib() -> ctypes.CDLL:
    """The loaded libxshare.so (raises if it was not built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                               "`python -m paper_2602_07265_amd.build` (hipcc, gfx950)")
        L = ctypes.CDLL(LIB_PATH)
        L.xshare_route_workspace_bytes.argtypes = [_I32, ctypes.POINTER(RouteParams)]
        L.xshare_route_workspace_bytes.restype = _SZ
        L.xshare_moe_workspace_bytes.argtypes = [_I32, _I32, _I32, ctypes.POINTER(RouteParams),
                                                 ctypes.POINTER(EpLayout),
                                                 ctypes.POINTER(SharedExperts)]
        L.xshare_moe_workspace_bytes.restype = _SZ
        L.xshare_layer_workspace_bytes.argtypes = [_I32, _I32, _I32, ctypes.POINTER(RouteParams),
                                                   ctypes.POINTER(EpLayout),
                                                   ctypes.POINTER(SharedExperts)]
        L.xshare_layer_workspace_bytes.restype = _SZ
        L.xshare_router_workspace_bytes.argtypes = [_I32, _I32, _I32]
        L.xshare_router_workspace_bytes.restype = _SZ
        L.xshare_router_logits.argtypes = [_P, _P, _I32, _I32, _I32, _P, _P, _SZ, _P]
        L.xshare_router_logits.restype = ctypes.c_int
        L.xshare_moe_layer.argtypes = [_P, _P, _I32, _I32, _I32, _P, _P, _P,
                                       ctypes.POINTER(SharedExperts), ctypes.POINTER(RouteParams),
                                       _P, _P, _I32, ctypes.POINTER(EpLayout), _P, _P, _P, _P, _P,
                                       _P, _P, _SZ, _P, _P]
        L.xshare_moe_layer.restype = ctypes.c_int
        L.xshare_moe_forward_fp8.argtypes = [_P, _P, _I32, _I32, _I32, _P, _P, _P, _P, _P, _P,
                                             ctypes.POINTER(RouteParams), _P, _P, _I32,
                                             ctypes.POINTER(EpLayout), _P, _P, _P, _P, _P, _P,
                                             _SZ, _P, _P]
        L.xshare_moe_forward_fp8.restype = ctypes.c_int
        L.xshare_moe_forward_mxfp4.argtypes = [_P, _P, _I32, _I32, _I32, _P, _P, _P, _P, _P, _P,
                                             ctypes.POINTER(RouteParams), _P, _P, _I32,
                                             ctypes.POINTER(EpLayout), _P, _P, _P, _P, _P, _P,
                                             _SZ, _P, _P]
        L.xshare_moe_forward_mxfp4.restype = ctypes.c_int
        L.xshare_mx_scales_tiled_bytes.argtypes = [_I32, _I32, _I32]
        L.xshare_mx_scales_tiled_bytes.restype = _SZ
        L.xshare_mx_scales_tile.argtypes = [_P, _P, _I32, _I32, _I32, _P]
        L.xshare_mx_scales_tile.restype = ctypes.c_int
        L.xshare_route.argtypes = [_P, _I32, ctypes.POINTER(RouteParams), _P, _P, _P, _P, _P, _SZ,
                                   _P]
        L.xshare_route.restype = ctypes.c_int
        L.xshare_select_hier.argtypes = [_P, _I32, _P, _P, _I32, ctypes.POINTER(RouteParams), _P,
                                         _P, _P, _P, _P, _SZ, _P]
        L.xshare_select_hier.restype = ctypes.c_int
        L.xshare_select_ep.argtypes = [_P, _I32, ctypes.POINTER(RouteParams),
                                       ctypes.POINTER(EpLayout), _P, _P, _P, _P, _P, _P, _SZ, _P]
        L.xshare_select_ep.restype = ctypes.c_int
        L.xshare_moe_forward.argtypes = [_P, _P, _I32, _I32, _I32, _P, _P, _P,
                                         ctypes.POINTER(RouteParams), _P, _P, _I32,
                                         ctypes.POINTER(EpLayout), ctypes.POINTER(SharedExperts),
                                         _P, _P, _P, _P, _P, _P, _SZ, _P, _P]
        L.xshare_moe_forward.restype = ctypes.c_int
        L.xshare_moe_forward_noalloc.argtypes = [_P, _P, _I32, _I32, _I32, _P, _P, _P,
                                                 ctypes.POINTER(RouteParams), _P, _P, _I32,
                                                 ctypes.POINTER(EpLayout),
                                                 ctypes.POINTER(SharedExperts), _P, _P, _P, _P,
                                                 _P, _P, _P]
        L.xshare_moe_forward_noalloc.restype = ctypes.c_int
        L.xshare_moe_forward_v2.argtypes = [ctypes.POINTER(LayerArgs)]
        L.xshare_moe_forward_v2.restype = ctypes.c_int
        L.xshare_moe_forward_v2_workspace_bytes.argtypes = [ctypes.POINTER(LayerArgs)]
        L.xshare_moe_forward_v2_workspace_bytes.restype = _SZ
        L.xshare_gate.argtypes = [_P, _I32, _I32, _I64, _P, ctypes.POINTER(GateParams), _P, _P,
                                  _P]
        L.xshare_gate.restype = ctypes.c_int
        L.xshare_gate_backward.argtypes = [_P, _I32, _I32, _I64, ctypes.POINTER(GateParams), _P,
                                           _P, _P, _P]
        L.xshare_gate_backward.restype = ctypes.c_int
        L.xshare_block_quantize.argtypes = [_P, _I32, _I32, _I64, _I32, _P, _P, _P]
        L.xshare_block_quantize.restype = ctypes.c_int
        L.xshare_block_linear_workspace_bytes.argtypes = [_I32, _I32, _I32]
        L.xshare_block_linear_workspace_bytes.restype = _SZ
        L.xshare_block_linear.argtypes = [_P, _I64, _P, _P, _I32, _I32, _I32, _P, _P, _P, _I64,
                                          _P, _SZ, _P]
        L.xshare_block_linear.restype = ctypes.c_int
        L.xshare_block_experts_workspace_bytes.argtypes = [_I32, _I32, _I32, _I32, _I32]
        L.xshare_block_experts_workspace_bytes.restype = _SZ
        L.xshare_block_experts.argtypes = [ctypes.POINTER(BlockExpertsArgs)]
        L.xshare_block_experts.restype = ctypes.c_int
        L.xshare_probe_stream_read.argtypes = [_P, _SZ, _I32, _I32, _P, _P]
        L.xshare_probe_stream_read.restype = ctypes.c_int
        L.xshare_block_times.argtypes = [_P, _P, _P, _I32, _P]
        L.xshare_block_times.restype = ctypes.c_int
        L.xshare_status_string.argtypes = [_I32]
        L.xshare_status_string.restype = ctypes.c_char_p
        L.xshare_version.argtypes = []
        L.xshare_version.restype = ctypes.c_char_p
        L.xshare_layer_budgets.argtypes = [_I32, _I32, _P]
        L.xshare_layer_budgets.restype = ctypes.c_int
        _lib = L
    return _lib


def status_string(status: int) -> str:
    return lib().xshare_status_string(int(status)).decode()


def version() -> str:
    return lib().xshare_version().decode()


def params(n_experts: int, top_k: int, warmup_k0: int, budget: int, budget_mode="total",
           score_mode="topk", per_request_budget: int = 0, threshold: float = 0.0,
           ledger=None) -> RouteParams:
    """``threshold`` is tau of the "threshold" budget mode (Algorithm 1's stopping rule);
    ``ledger`` an optional device int32 tensor of LEDGER_FIELDS' length that the call adds
    its counts to."""
    if ledger is not None:
        _dev(ledger, torch.int32, (len(LEDGER_FIELDS) + 2,), "ledger")
    return RouteParams(int(n_experts), int(top_k), int(warmup_k0), int(budget),
                       BUDGET[budget_mode] if isinstance(budget_mode, str) else int(budget_mode),
                       SCORE[score_mode] if isinstance(score_mode, str) else int(score_mode),
                       int(per_request_budget), float(threshold),
                       None if ledger is None else ledger.data_ptr())


LEDGER_FIELDS = ("layers", "selected", "active", "vanilla_union", "invalid", "max_selected")


def new_ledger(device="cuda") -> torch.Tensor:
    """A zeroed budget ledger (xshare_budget_ledger) in device memory."""
    return torch.zeros(len(LEDGER_FIELDS) + 2, dtype=torch.int32, device=device)


def ledger_dict(ledger: torch.Tensor) -> dict:
    return dict(zip(LEDGER_FIELDS, ledger.to("cpu").tolist()))


def layer_budgets(K: int, L: int) -> list:
    """Uniform per-layer budgets m_l for a global budget K over L layers (host call)."""
    m = (ctypes.c_int32 * max(int(L), 1))()
    _check(lib().xshare_layer_budgets(int(K), int(L), m), "xshare_layer_budgets")
    return [int(v) for v in m[:int(L)]]


def route_workspace_bytes(T: int, p: RouteParams) -> int:
    return int(lib().xshare_route_workspace_bytes(int(T), ctypes.byref(p)))


def moe_workspace_bytes(T: int, d: int, f: int, p: RouteParams, ep=None, shared=None) -> int:
    """``ep``: an EpLayout or None; ``shared``: a SharedExperts or None."""
    return int(lib().xshare_moe_workspace_bytes(int(T), int(d), int(f), ctypes.byref(p),
                                                None if ep is None else ctypes.byref(ep),
                                                None if shared is None else ctypes.byref(shared)))


def layer_workspace_bytes(T: int, d: int, f: int, p: RouteParams, ep=None, shared=None) -> int:
    return int(lib().xshare_layer_workspace_bytes(int(T), int(d), int(f), ctypes.byref(p),
                                                  None if ep is None else ctypes.byref(ep),
                                                  None if shared is None else ctypes.byref(shared)))


def _shared(shared, d, f, dev):
    """SharedExperts from a (w1 [N_s,f,d], w3 [N_s,f,d], w2 [N_s,d,f]) tuple of bf16 tensors."""
    if shared is None:
        return None
    w1, w3, w2 = shared
    ns = w1.shape[0]
    _dev(w1, torch.bfloat16, (ns, f, d), "shared w1")
    _dev(w3, torch.bfloat16, (ns, f, d), "shared w3")
    _dev(w2, torch.bfloat16, (ns, d, f), "shared w2")
    return SharedExperts(int(ns), w1.data_ptr(), w3.data_ptr(), w2.data_ptr())


@_placed
def router_logits(x: torch.Tensor, w_gate: torch.Tensor, *, out=None, workspace=None,
                  stream=None) -> torch.Tensor:
    """h = W_g x on the GPU (fp32 [T, N])."""
    T, d = x.shape
    N = w_gate.shape[0]
    _dev(x, torch.bfloat16, (T, d), "x")
    _dev(w_gate, torch.bfloat16, (N, d), "w_gate")
    out = torch.empty((T, N), dtype=torch.float32, device=x.device) if out is None else out
    _dev(out, torch.float32, (T, N), "logits")
    need = int(lib().xshare_router_workspace_bytes(T, d, N))
    if workspace is None:
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=x.device)
    st = lib().xshare_router_logits(_ptr(x), _ptr(w_gate), T, d, N, _ptr(out), _ptr(workspace),
                                    workspace.numel(), _stream(stream))
    _check(st, "xshare_router_logits")
    return out


class GroupMap:
    """GPU groups of the experts for expert parallelism: ``groups`` None (equal contiguous
    blocks of N / G) or a per-expert sequence / device int32 tensor of group ids."""

    def __init__(self, n_groups: int, groups=None, local_group: int = -1, device="cuda"):
        self.host = None
        self.dev = None
        if groups is not None:
            if isinstance(groups, torch.Tensor) and groups.is_cuda:
                self.dev = _dev(groups, torch.int32, (groups.numel(),), "expert_group")
            else:
                self.host = torch.as_tensor([int(v) for v in groups], dtype=torch.int32)
                self.dev = self.host.to(device)
        self.layout = EpLayout(int(n_groups), int(local_group),
                               None if self.dev is None else self.dev.data_ptr(),
                               None if self.host is None else self.host.data_ptr())

    def with_local(self, local_group: int) -> "GroupMap":
        g = GroupMap.__new__(GroupMap)
        g.host, g.dev = self.host, self.dev
        g.layout = EpLayout(self.layout.n_groups, int(local_group), self.layout.expert_group,
                            self.layout.host_expert_group)
        return g


# ----------------------------------------------------------------------------- helpers

def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _dev(t, dtype, shape, name):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t


def _stream(stream):
    s = torch.cuda.current_stream() if stream is None else stream
    return ctypes.c_void_p(s.cuda_stream)


def _check(status, what):
    if status != OK:
        raise XShareError(status, what)


def stats_dict(stats: torch.Tensor) -> dict:
    v = stats.to("cpu").tolist()
    return dict(zip(STATS_FIELDS, v))


def _offsets(req_offsets, device):
    """(device int32 tensor, host int32 array pointer holder) from a list/array/tensor."""
    if isinstance(req_offsets, torch.Tensor) and req_offsets.is_cuda:
        dev = _dev(req_offsets, torch.int32, (req_offsets.numel(),), "req_offsets")
        return dev, None
    host = torch.as_tensor(list(int(v) for v in req_offsets), dtype=torch.int32)
    return host.to(device), host


# ----------------------------------------------------------------------------- entry points

def _route_impl(logits, p, req_offsets, out, workspace, stream):
    T, N = logits.shape
    k = p.top_k
    dev = logits.device
    _dev(logits, torch.float32, (T, N), "logits")
    if N != p.n_experts:
        raise ValueError("logits width must equal n_experts")
    out = dict(out or {})
    sel = out.get("sel_mask") if out.get("sel_mask") is not None else torch.empty(N, dtype=torch.uint8, device=dev)
    ids = out.get("ids") if out.get("ids") is not None else torch.empty((T, k), dtype=torch.int32, device=dev)
    w = out.get("w") if out.get("w") is not None else torch.empty((T, k), dtype=torch.float32, device=dev)
    stats = out.get("stats") if out.get("stats") is not None else torch.empty(8, dtype=torch.int32, device=dev)
    _dev(sel, torch.uint8, (N,), "sel_mask")
    _dev(ids, torch.int32, (T, k), "ids")
    _dev(w, torch.float32, (T, k), "w")
    _dev(stats, torch.int32, (8,), "stats")
    need = route_workspace_bytes(T, p)
    if workspace is None:
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=dev)
    if req_offsets is None:
        st = lib().xshare_route(_ptr(logits), T, ctypes.byref(p), _ptr(sel), _ptr(ids), _ptr(w),
                                _ptr(stats), _ptr(workspace), workspace.numel(), _stream(stream))
        _check(st, "xshare_route")
    else:
        d_off, h_off = _offsets(req_offsets, dev)
        R = d_off.numel() - 1
        hp = None if h_off is None else ctypes.c_void_p(h_off.data_ptr())
        st = lib().xshare_select_hier(_ptr(logits), T, _ptr(d_off), hp, R, ctypes.byref(p),
                                      _ptr(sel), _ptr(ids), _ptr(w), _ptr(stats), _ptr(workspace),
                                      workspace.numel(), _stream(stream))
        _check(st, "xshare_select_hier")
    return dict(sel_mask=sel, ids=ids, w=w, stats=stats)


@_placed
def select_ep(logits: torch.Tensor, groups: GroupMap, top_k: int, warmup_k0: int,
              per_group_budget: int, score_mode="topk", *, ledger=None, out=None,
              workspace=None, stream=None) -> dict:
    """Algorithms 5-6 on the GPU: dict(sel_mask, ids, w, stats, group_load)."""
    T, N = logits.shape
    dev = logits.device
    _dev(logits, torch.float32, (T, N), "logits")
    p = params(N, top_k, warmup_k0, per_group_budget, "per_group", score_mode, ledger=ledger)
    G = groups.layout.n_groups
    out = dict(out or {})
    sel = out.get("sel_mask") if out.get("sel_mask") is not None else torch.empty(N, dtype=torch.uint8, device=dev)
    ids = out.get("ids") if out.get("ids") is not None else torch.empty((T, top_k), dtype=torch.int32, device=dev)
    w = out.get("w") if out.get("w") is not None else torch.empty((T, top_k), dtype=torch.float32, device=dev)
    stats = out.get("stats") if out.get("stats") is not None else torch.empty(8, dtype=torch.int32, device=dev)
    load = out.get("group_load") if out.get("group_load") is not None else torch.empty(max(G, 1), dtype=torch.int32, device=dev)
    _dev(sel, torch.uint8, (N,), "sel_mask")
    _dev(ids, torch.int32, (T, top_k), "ids")
    _dev(w, torch.float32, (T, top_k), "w")
    _dev(stats, torch.int32, (8,), "stats")
    need = route_workspace_bytes(T, p)
    if workspace is None:
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=dev)
    st = lib().xshare_select_ep(_ptr(logits), T, ctypes.byref(p), ctypes.byref(groups.layout),
                                _ptr(sel), _ptr(ids), _ptr(w), _ptr(load), _ptr(stats),
                                _ptr(workspace), workspace.numel(), _stream(stream))
    _check(st, "xshare_select_ep")
    return dict(sel_mask=sel, ids=ids, w=w, stats=stats, group_load=load)


@_placed
def route(logits: torch.Tensor, top_k: int, warmup_k0: int, budget: int, budget_mode="total",
          score_mode="topk", *, tau: float = 0.0, ledger=None, out=None, workspace=None,
          stream=None) -> dict:
    """Algorithm 2 on the GPU: returns dict(sel_mask, ids, w, stats) device tensors."""
    p = params(logits.shape[1], top_k, warmup_k0, budget, budget_mode, score_mode, 0, tau,
               ledger)
    return _route_impl(logits, p, None, out, workspace, stream)


@_placed
def select_hier(logits: torch.Tensor, req_offsets, top_k: int, warmup_k0: int,
                per_request_budget: int, budget: int, budget_mode="total", score_mode="topk", *,
                tau: float = 0.0, ledger=None, out=None, workspace=None, stream=None) -> dict:
    """Algorithms 3-4 on the GPU; req_offsets as a host sequence (validated) or device tensor."""
    p = params(logits.shape[1], top_k, warmup_k0, budget, budget_mode, score_mode,
               per_request_budget, tau, ledger)
    return _route_impl(logits, p, req_offsets, out, workspace, stream)


@_placed
def moe_forward(x: torch.Tensor, logits: torch.Tensor, w1: torch.Tensor, w3: torch.Tensor,
                w2: torch.Tensor, top_k: int, warmup_k0: int, budget: int, budget_mode="total",
                score_mode="topk", *, req_offsets=None, per_request_budget: int = 0,
                groups: GroupMap | None = None, tau: float = 0.0, shared=None, ledger=None,
                y=None, routing_out=True, workspace=None, stage_events=None,
                stream=None) -> dict:
    """The MoE layer: returns dict(y [T,d] bf16, and sel_mask/ids/w/stats if routing_out).

    With ``groups`` the selection is Algorithms 5-6 (``budget`` is m_g, budget_mode is
    ignored) and, if groups has a local group, y is that group's share of the layer."""
    T, d = x.shape
    N = logits.shape[1]
    f = w1.shape[1]
    dev = x.device
    _dev(x, torch.bfloat16, (T, d), "x")
    _dev(logits, torch.float32, (T, N), "logits")
    _dev(w1, torch.bfloat16, (N, f, d), "w1")
    _dev(w3, torch.bfloat16, (N, f, d), "w3")
    _dev(w2, torch.bfloat16, (N, d, f), "w2")
    if groups is not None:
        budget_mode = "per_group"
    p = params(N, top_k, warmup_k0, budget, budget_mode, score_mode, per_request_budget, tau,
               ledger)
    ep = None if groups is None else groups.layout
    sh = _shared(shared, d, f, dev)
    if y is None:
        y = torch.empty((T, d), dtype=torch.bfloat16, device=dev)
    _dev(y, torch.bfloat16, (T, d), "y")
    res = {"y": y}
    if routing_out:
        res.update(sel_mask=torch.empty(N, dtype=torch.uint8, device=dev),
                   ids=torch.empty((T, top_k), dtype=torch.int32, device=dev),
                   w=torch.empty((T, top_k), dtype=torch.float32, device=dev),
                   stats=torch.empty(8, dtype=torch.int32, device=dev))
    need = moe_workspace_bytes(T, d, f, p, ep, sh)
    if workspace is None:
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=dev)
    d_off = h_off = None
    R = 0
    if req_offsets is not None:
        d_off, h_off = _offsets(req_offsets, dev)
        R = d_off.numel() - 1
    ev = None
    if stage_events is not None:
        if len(stage_events) != N_STAGE_EVENTS:
            raise ValueError(f"stage_events needs {N_STAGE_EVENTS} events")
        ev = (ctypes.c_void_p * N_STAGE_EVENTS)(*[e.handle for e in stage_events])
    st = lib().xshare_moe_forward(
        _ptr(x), _ptr(logits), T, d, f, _ptr(w1), _ptr(w3), _ptr(w2), ctypes.byref(p),
        _ptr(d_off), None if h_off is None else ctypes.c_void_p(h_off.data_ptr()), R,
        None if ep is None else ctypes.byref(ep), None if sh is None else ctypes.byref(sh),
        _ptr(y),
        _ptr(res.get("sel_mask")), _ptr(res.get("ids")), _ptr(res.get("w")),
        _ptr(res.get("stats")), _ptr(workspace), workspace.numel(), ev, _stream(stream))
    _check(st, "xshare_moe_forward")
    return res


@_placed
def moe_forward_noalloc(x: torch.Tensor, logits: torch.Tensor, w1: torch.Tensor,
                        w3: torch.Tensor, w2: torch.Tensor, top_k: int, warmup_k0: int,
                        budget: int, budget_mode="total", score_mode="topk", *, y=None,
                        out=None, stage_events=None, stream=None) -> dict:
    """xshare_moe_forward_noalloc: the layer with the library's own fixed scratch array (no
    workspace).  ``y`` and ``out`` (a dict of sel_mask / ids / w / stats tensors) are
    preallocated outputs; with them the call allocates nothing here either.  Flat selection
    (Algorithm 2) only in this binding."""
    T, d = x.shape
    N = logits.shape[1]
    f = w1.shape[1]
    dev = x.device
    _dev(x, torch.bfloat16, (T, d), "x")
    _dev(logits, torch.float32, (T, N), "logits")
    _dev(w1, torch.bfloat16, (N, f, d), "w1")
    _dev(w3, torch.bfloat16, (N, f, d), "w3")
    _dev(w2, torch.bfloat16, (N, d, f), "w2")
    p = params(N, top_k, warmup_k0, budget, budget_mode, score_mode)
    if y is None:
        y = torch.empty((T, d), dtype=torch.bfloat16, device=dev)
    _dev(y, torch.bfloat16, (T, d), "y")
    res = {"y": y}
    if out is not None:
        res.update(out)
        _dev(res["sel_mask"], torch.uint8, (N,), "sel_mask")
        _dev(res["ids"], torch.int32, (T, top_k), "ids")
        _dev(res["w"], torch.float32, (T, top_k), "w")
        _dev(res["stats"], torch.int32, (8,), "stats")
    ev = None
    if stage_events is not None:
        if len(stage_events) != N_STAGE_EVENTS:
            raise ValueError(f"stage_events needs {N_STAGE_EVENTS} events")
        ev = (ctypes.c_void_p * N_STAGE_EVENTS)(*[e.handle for e in stage_events])
    st = lib().xshare_moe_forward_noalloc(
        _ptr(x), _ptr(logits), T, d, f, _ptr(w1), _ptr(w3), _ptr(w2), ctypes.byref(p), None,
        None, 0, None, None, _ptr(y), _ptr(res.get("sel_mask")), _ptr(res.get("ids")),
        _ptr(res.get("w")), _ptr(res.get("stats")), ev, _stream(stream))
    _check(st, "xshare_moe_forward_noalloc")
    return res


@_placed
def moe_forward_fp8(x: torch.Tensor, logits: torch.Tensor, q1: torch.Tensor, q3: torch.Tensor,
                    q2: torch.Tensor, s1: torch.Tensor, s3: torch.Tensor, s2: torch.Tensor,
                    top_k: int, warmup_k0: int, budget: int, budget_mode="total",
                    score_mode="topk", *, req_offsets=None, per_request_budget: int = 0,
                    groups: GroupMap | None = None, tau: float = 0.0, ledger=None, y=None,
                    routing_out=True, workspace=None, stage_events=None, stream=None) -> dict:
    """The MoE layer with FP8 E4M3FN expert weights (uint8 codes) and per-row fp32 scales."""
    T, d = x.shape
    N = logits.shape[1]
    f = q1.shape[1]
    dev = x.device
    _dev(x, torch.bfloat16, (T, d), "x")
    _dev(logits, torch.float32, (T, N), "logits")
    _dev(q1, torch.uint8, (N, f, d), "w1 codes")
    _dev(q3, torch.uint8, (N, f, d), "w3 codes")
    _dev(q2, torch.uint8, (N, d, f), "w2 codes")
    _dev(s1, torch.float32, (N, f), "w1 scales")
    _dev(s3, torch.float32, (N, f), "w3 scales")
    _dev(s2, torch.float32, (N, d), "w2 scales")
    if groups is not None:
        budget_mode = "per_group"
    p = params(N, top_k, warmup_k0, budget, budget_mode, score_mode, per_request_budget, tau,
               ledger)
    ep = None if groups is None else groups.layout
    if y is None:
        y = torch.empty((T, d), dtype=torch.bfloat16, device=dev)
    _dev(y, torch.bfloat16, (T, d), "y")
    res = {"y": y}
    if routing_out:
        res.update(sel_mask=torch.empty(N, dtype=torch.uint8, device=dev),
                   ids=torch.empty((T, top_k), dtype=torch.int32, device=dev),
                   w=torch.empty((T, top_k), dtype=torch.float32, device=dev),
                   stats=torch.empty(8, dtype=torch.int32, device=dev))
    need = moe_workspace_bytes(T, d, f, p, ep)
    if workspace is None:
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=dev)
    d_off = h_off = None
    R = 0
    if req_offsets is not None:
        d_off, h_off = _offsets(req_offsets, dev)
        R = d_off.numel() - 1
    ev = None
    if stage_events is not None:
        if len(stage_events) != N_STAGE_EVENTS:
            raise ValueError(f"stage_events needs {N_STAGE_EVENTS} events")
        ev = (ctypes.c_void_p * N_STAGE_EVENTS)(*[e.handle for e in stage_events])
    st = lib().xshare_moe_forward_fp8(
        _ptr(x), _ptr(logits), T, d, f, _ptr(q1), _ptr(q3), _ptr(q2), _ptr(s1), _ptr(s3),
        _ptr(s2), ctypes.byref(p), _ptr(d_off),
        None if h_off is None else ctypes.c_void_p(h_off.data_ptr()), R,
        None if ep is None else ctypes.byref(ep), _ptr(y), _ptr(res.get("sel_mask")),
        _ptr(res.get("ids")), _ptr(res.get("w")), _ptr(res.get("stats")), _ptr(workspace),
        workspace.numel(), ev, _stream(stream))
    _check(st, "xshare_moe_forward_fp8")
    return res


def mx_granules(k: int) -> int:
    """Granules of 8 scale blocks (256 inputs) per row in the tiled MXFP4 scale layout."""
    return (k + 255) // 256


@_placed
def tile_mx_scales(scales: torch.Tensor, stream=None) -> torch.Tensor:
    """xshare_mx_scales_tile: E8M0 scales [n, rows, k/32] (row-major) -> the tiled layout
    the MXFP4 GEMMs read, [n, rows/16, ceil(k/256), 16, 8] uint8 (a new tensor)."""
    n, rows, nb = scales.shape
    k = 32 * nb
    if scales.dtype != torch.uint8 or not scales.is_cuda:
        raise ValueError("scales: a uint8 device tensor [n, rows, k/32]")
    src = scales.contiguous()
    out = torch.empty((n, rows // 16, mx_granules(k), 16, 8), dtype=torch.uint8,
                      device=scales.device)
    assert out.numel() == lib().xshare_mx_scales_tiled_bytes(n, rows, k)
    _check(lib().xshare_mx_scales_tile(_ptr(src), _ptr(out), n, rows, k, _stream(stream)),
           "xshare_mx_scales_tile")
    return out


def mx_tiled(weights):
    """(q1, q3, q2, e1, e3, e2) with row-major scales -> the same with tiled scales."""
    q1, q3, q2, e1, e3, e2 = weights
    return q1, q3, q2, tile_mx_scales(e1), tile_mx_scales(e3), tile_mx_scales(e2)


@_placed
def moe_forward_mxfp4(x: torch.Tensor, logits: torch.Tensor, q1: torch.Tensor, q3: torch.Tensor,
                      q2: torch.Tensor, e1: torch.Tensor, e3: torch.Tensor, e2: torch.Tensor,
                      top_k: int, warmup_k0: int, budget: int, budget_mode="total",
                      score_mode="topk", *, req_offsets=None, per_request_budget: int = 0,
                      groups: GroupMap | None = None, tau: float = 0.0, ledger=None, y=None,
                      routing_out=True, workspace=None, stage_events=None, stream=None) -> dict:
    """The MoE layer with MXFP4 expert weights: packed E2M1 codes (uint8, two per byte) and
    one E8M0 scale byte per 32 inputs of a row, in the tiled layout (tile_mx_scales)."""
    T, d = x.shape
    N = logits.shape[1]
    f = q1.shape[1]
    dev = x.device
    _dev(x, torch.bfloat16, (T, d), "x")
    _dev(logits, torch.float32, (T, N), "logits")
    _dev(q1, torch.uint8, (N, f, d // 2), "w1 codes")
    _dev(q3, torch.uint8, (N, f, d // 2), "w3 codes")
    _dev(q2, torch.uint8, (N, d, f // 2), "w2 codes")
    _dev(e1, torch.uint8, (N, f // 16, mx_granules(d), 16, 8), "w1 tiled scales")
    _dev(e3, torch.uint8, (N, f // 16, mx_granules(d), 16, 8), "w3 tiled scales")
    _dev(e2, torch.uint8, (N, d // 16, mx_granules(f), 16, 8), "w2 tiled scales")
    if groups is not None:
        budget_mode = "per_group"
    p = params(N, top_k, warmup_k0, budget, budget_mode, score_mode, per_request_budget, tau,
               ledger)
    ep = None if groups is None else groups.layout
    if y is None:
        y = torch.empty((T, d), dtype=torch.bfloat16, device=dev)
    _dev(y, torch.bfloat16, (T, d), "y")
    res = {"y": y}
    if routing_out:
        res.update(sel_mask=torch.empty(N, dtype=torch.uint8, device=dev),
                   ids=torch.empty((T, top_k), dtype=torch.int32, device=dev),
                   w=torch.empty((T, top_k), dtype=torch.float32, device=dev),
                   stats=torch.empty(8, dtype=torch.int32, device=dev))
    need = moe_workspace_bytes(T, d, f, p, ep)
    if workspace is None:
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=dev)
    d_off = h_off = None
    R = 0
    if req_offsets is not None:
        d_off, h_off = _offsets(req_offsets, dev)
        R = d_off.numel() - 1
    ev = None
    if stage_events is not None:
        if len(stage_events) != N_STAGE_EVENTS:
            raise ValueError(f"stage_events needs {N_STAGE_EVENTS} events")
        ev = (ctypes.c_void_p * N_STAGE_EVENTS)(*[e.handle for e in stage_events])
    st = lib().xshare_moe_forward_mxfp4(
        _ptr(x), _ptr(logits), T, d, f, _ptr(q1), _ptr(q3), _ptr(q2), _ptr(e1), _ptr(e3),
        _ptr(e2), ctypes.byref(p), _ptr(d_off),
        None if h_off is None else ctypes.c_void_p(h_off.data_ptr()), R,
        None if ep is None else ctypes.byref(ep), _ptr(y), _ptr(res.get("sel_mask")),
        _ptr(res.get("ids")), _ptr(res.get("w")), _ptr(res.get("stats")), _ptr(workspace),
        workspace.numel(), ev, _stream(stream))
    _check(st, "xshare_moe_forward_mxfp4")
    return res


@_placed
def moe_layer(x: torch.Tensor, w_gate: torch.Tensor, w1: torch.Tensor, w3: torch.Tensor,
              w2: torch.Tensor, top_k: int, warmup_k0: int, budget: int, budget_mode="total",
              score_mode="topk", *, shared=None, req_offsets=None, per_request_budget: int = 0,
              groups: GroupMap | None = None, tau: float = 0.0, ledger=None, y=None,
              routing_out=True, logits_out=True, workspace=None, stage_events=None,
              stream=None) -> dict:
    """The whole layer from hidden states: router GEMM, selection, routed and shared experts.
    Returns dict(y, and logits/sel_mask/ids/w/stats as requested)."""
    T, d = x.shape
    N = w_gate.shape[0]
    f = w1.shape[1]
    dev = x.device
    _dev(x, torch.bfloat16, (T, d), "x")
    _dev(w_gate, torch.bfloat16, (N, d), "w_gate")
    _dev(w1, torch.bfloat16, (N, f, d), "w1")
    _dev(w3, torch.bfloat16, (N, f, d), "w3")
    _dev(w2, torch.bfloat16, (N, d, f), "w2")
    if groups is not None:
        budget_mode = "per_group"
    p = params(N, top_k, warmup_k0, budget, budget_mode, score_mode, per_request_budget, tau,
               ledger)
    ep = None if groups is None else groups.layout
    sh = _shared(shared, d, f, dev)
    if y is None:
        y = torch.empty((T, d), dtype=torch.bfloat16, device=dev)
    _dev(y, torch.bfloat16, (T, d), "y")
    res = {"y": y}
    if logits_out:
        res["logits"] = torch.empty((T, N), dtype=torch.float32, device=dev)
    if routing_out:
        res.update(sel_mask=torch.empty(N, dtype=torch.uint8, device=dev),
                   ids=torch.empty((T, top_k), dtype=torch.int32, device=dev),
                   w=torch.empty((T, top_k), dtype=torch.float32, device=dev),
                   stats=torch.empty(8, dtype=torch.int32, device=dev))
    need = layer_workspace_bytes(T, d, f, p, ep, sh)
    if workspace is None:
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=dev)
    d_off = h_off = None
    R = 0
    if req_offsets is not None:
        d_off, h_off = _offsets(req_offsets, dev)
        R = d_off.numel() - 1
    ev = None
    if stage_events is not None:
        if len(stage_events) != N_STAGE_EVENTS:
            raise ValueError(f"stage_events needs {N_STAGE_EVENTS} events")
        ev = (ctypes.c_void_p * N_STAGE_EVENTS)(*[e.handle for e in stage_events])
    st = lib().xshare_moe_layer(
        _ptr(x), _ptr(w_gate), T, d, f, _ptr(w1), _ptr(w3), _ptr(w2),
        None if sh is None else ctypes.byref(sh), ctypes.byref(p), _ptr(d_off),
        None if h_off is None else ctypes.c_void_p(h_off.data_ptr()), R,
        None if ep is None else ctypes.byref(ep), _ptr(y), _ptr(res.get("logits")),
        _ptr(res.get("sel_mask")), _ptr(res.get("ids")), _ptr(res.get("w")),
        _ptr(res.get("stats")), _ptr(workspace), workspace.numel(), ev, _stream(stream))
    _check(st, "xshare_moe_layer")
    return res


# ----------------------------------------------------------------------------- HIP events

class HipEvent:
    """A raw hipEvent_t (for the stage_events argument and kernel timing on any stream)."""
    _hip = None

    @classmethod
    def _rt(cls):
        if cls._hip is None:
            h = ctypes.CDLL("libamdhip64.so")
            h.hipEventCreate.argtypes = [ctypes.POINTER(ctypes.c_void_p)]
            h.hipEventCreateWithFlags.argtypes = [ctypes.POINTER(ctypes.c_void_p), ctypes.c_uint]
            h.hipEventRecord.argtypes = [ctypes.c_void_p, ctypes.c_void_p]
            h.hipEventSynchronize.argtypes = [ctypes.c_void_p]
            h.hipEventElapsedTime.argtypes = [ctypes.POINTER(ctypes.c_float), ctypes.c_void_p,
                                              ctypes.c_void_p]
            h.hipEventDestroy.argtypes = [ctypes.c_void_p]
            cls._hip = h
        return cls._hip

    def __init__(self, timing: bool = True):
        self.handle = ctypes.c_void_p()
        rt = self._rt()
        flags = 0 if timing else 2                 # hipEventDisableTiming
        if rt.hipEventCreateWithFlags(ctypes.byref(self.handle), flags) != 0:
            raise RuntimeError("hipEventCreateWithFlags failed")
        self.handle = self.handle.value

    def record(self, stream=None):
        s = torch.cuda.current_stream() if stream is None else stream
        if self._rt().hipEventRecord(self.handle, ctypes.c_void_p(s.cuda_stream)) != 0:
            raise RuntimeError("hipEventRecord failed")

    def synchronize(self):
        self._rt().hipEventSynchronize(self.handle)

    def elapsed_ms(self, later: "HipEvent") -> float:
        out = ctypes.c_float()
        if self._rt().hipEventElapsedTime(ctypes.byref(out), self.handle, later.handle) != 0:
            raise RuntimeError("hipEventElapsedTime failed")
        return float(out.value)

    def __del__(self):
        try:
            if self.handle and self._hip is not None:
                self._hip.hipEventDestroy(self.handle)
        except Exception:
            pass


@_placed
def moe_forward_v2(x: torch.Tensor, top_k: int, warmup_k0: int, budget: int,
                   budget_mode="total", score_mode="topk", *, logits=None, w_gate=None,
                   weights=(), scales=(None, None, None), weight_format="bf16",
                   req_offsets=None, per_request_budget: int = 0,
                   groups: GroupMap | None = None, tau: float = 0.0, shared=None, ledger=None,
                   y=None, routing_out=True, logits_out=False, workspace=None,
                   stage_events=None, stream=None) -> dict:
    """xshare_moe_forward_v2: the layer from one argument struct.  ``logits`` (fp32 [T, N]) or
    ``w_gate`` (bf16 [N, d], logits computed on the device); ``weights`` = (w1, w3, w2) in
    ``weight_format`` with ``scales`` for FP8 / MXFP4.  Shapes are checked by the library;
    this only marshals pointers."""
    T, d = x.shape
    w1, w3, w2 = weights
    N = (logits if logits is not None else w_gate).shape[0 if logits is None else 1]
    f = w1.shape[1]
    dev = x.device
    if groups is not None:
        budget_mode = "per_group"
    p = params(N, top_k, warmup_k0, budget, budget_mode, score_mode, per_request_budget, tau,
               ledger)
    ep = None if groups is None else groups.layout
    sh = _shared(shared, d, f, dev)
    if y is None:
        y = torch.empty((T, d), dtype=torch.bfloat16, device=dev)
    res = {"y": y}
    if logits_out:
        res["logits"] = torch.empty((T, N), dtype=torch.float32, device=dev)
    if routing_out:
        res.update(sel_mask=torch.empty(N, dtype=torch.uint8, device=dev),
                   ids=torch.empty((T, top_k), dtype=torch.int32, device=dev),
                   w=torch.empty((T, top_k), dtype=torch.float32, device=dev),
                   stats=torch.empty(8, dtype=torch.int32, device=dev))
    d_off = h_off = None
    R = 0
    if req_offsets is not None:
        d_off, h_off = _offsets(req_offsets, dev)
        R = d_off.numel() - 1
    ev = None
    if stage_events is not None:
        if len(stage_events) != N_STAGE_EVENTS:
            raise ValueError(f"stage_events needs {N_STAGE_EVENTS} events")
        ev = (ctypes.c_void_p * N_STAGE_EVENTS)(*[e.handle for e in stage_events])
    s1, s3, s2 = scales
    a = LayerArgs()
    a.struct_size = ctypes.sizeof(LayerArgs)
    a.T, a.d, a.f = T, d, f
    a.x = x.data_ptr()
    a.logits = None if logits is None else logits.data_ptr()
    a.w_gate = None if w_gate is None else w_gate.data_ptr()
    a.weight_format = WEIGHTS[weight_format]
    a.w1, a.w3, a.w2 = w1.data_ptr(), w3.data_ptr(), w2.data_ptr()
    a.w1_scale = None if s1 is None else s1.data_ptr()
    a.w3_scale = None if s3 is None else s3.data_ptr()
    a.w2_scale = None if s2 is None else s2.data_ptr()
    a.params = ctypes.pointer(p)
    a.req_offsets = None if d_off is None else d_off.data_ptr()
    a.host_offsets = None if h_off is None else h_off.data_ptr()
    a.R = R
    a.ep = None if ep is None else ctypes.pointer(ep)
    a.shared = None if sh is None else ctypes.pointer(sh)
    a.y = y.data_ptr()
    for field, key in (("logits_out", "logits"), ("sel_mask", "sel_mask"), ("topk_ids", "ids"),
                       ("topk_w", "w"), ("stats", "stats")):
        setattr(a, field, None if res.get(key) is None else res[key].data_ptr())
    a.stage_events = None if ev is None else ctypes.cast(ev, ctypes.c_void_p)
    a.stream = _stream(stream).value
    need = int(lib().xshare_moe_forward_v2_workspace_bytes(ctypes.byref(a)))
    if workspace is None:
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=dev)
    a.ws, a.ws_bytes = workspace.data_ptr(), workspace.numel()
    _check(lib().xshare_moe_forward_v2(ctypes.byref(a)), "xshare_moe_forward_v2")
    return res


# ------------------------------------------- routing by scores, FP8 products in blocks of 128

def _rows(t, dtype, name, cols=None):
    """A GPU matrix of dtype whose rows may lie apart (its columns do not); its row stride."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor")
    if t.dtype is not dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    shape = t.shape
    if len(shape) != 2 or (cols is not None and shape[1] != cols):
        raise ValueError(f"{name} must be a matrix" + ("" if cols is None else f" of {cols} columns")
                         + f", got {tuple(shape)}")
    if t.is_contiguous():
        return shape[1]
    ld, step = t.stride()
    if shape[1] > 1 and step != 1:
        raise ValueError(f"{name}: the elements of a row must be neighbours")
    return ld if shape[0] > 1 else shape[1]


def _fit(device, *wanted):
    """Checks (tensor, dtype, shape, name) against a call's device, in few lookups: the shortest
    calls take about as long as their checks."""
    for t, dtype, shape, name in wanted:
        if t.dtype is not dtype or t.shape != shape or t.device != device \
                or not t.is_contiguous():
            _dev(t, dtype, shape, name)
            raise ValueError(f"{name} is on {t.device}, not {device}")


def _past_32_bits(sizes):
    """Whether one of the sizes, or-ed together, is more than the library's 32 bits hold: it would
    arrive as another, smaller one.  (Negative ones arrive as they are, and are refused there.)"""
    return sizes >> 31 not in (0, -1)


def _sizes(sizes, call):
    if _past_32_bits(sizes):
        raise XShareError(EUNSUPPORTED, call)


def _on(device, t, name):
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, not {device}")


def _workspace(device, t):
    """The bytes of a given workspace, which have to be as many as its elements say."""
    _on(device, t, "workspace")
    if not t.is_contiguous():
        raise ValueError("workspace must be contiguous")
    return t.numel() * t.element_size()


def _no_gradient(t, name, instead):
    """Refuses a tensor whose gradient autograd would expect of this call, which records none."""
    if t.requires_grad and torch.is_grad_enabled():
        raise ValueError(f"{name} requires a gradient, which this call does not record: detach it or "
                         f"call under torch.no_grad(); {instead}")


def _stream_of(x, stream):
    """The handle of x's device's current stream, without a Stream object where torch gives it
    (3 us less a call, of about 10 that the shortest of these calls take)."""
    if stream is not None:
        return stream.cuda_stream
    try:
        return torch._C._cuda_getCurrentRawStream(x.get_device())
    except AttributeError:
        return torch.cuda.current_stream(x.device).cuda_stream


def _gate_params(N, top_k, score, n_groups, top_groups, group_score, renormalize, scale):
    return GateParams(N, int(top_k), GATE[score] if isinstance(score, str) else int(score),
                      n_groups, top_groups,
                      GROUP[group_score] if isinstance(group_score, str) else int(group_score),
                      int(bool(renormalize)), float(scale))


def _logits(logits):
    dtype = logits.dtype if isinstance(logits, torch.Tensor) else None
    if dtype is not torch.float32 and dtype is not torch.bfloat16:
        raise ValueError("logits must be a float32 or bfloat16 GPU tensor")
    return int(dtype is torch.bfloat16), _rows(logits, dtype, "logits")


@_placed
def gate(logits: torch.Tensor, top_k: int, *, score="softmax", bias=None, n_groups: int = 1,
         top_groups: int = 1, group_score="max", renormalize: bool = True, scale: float = 1.0,
         out=None, stream=None) -> dict:
    """A router's choice for each token of logits [T, N] (fp32 or bf16): dict(ids int32 [T, k],
    w fp32 [T, k]).  ``bias`` (fp32 [N]) enters the choice only; with ``n_groups`` the experts
    come from the ``top_groups`` best groups (group_score "max" or "top2").  Records no gradient
    (``gate_backward`` gives the logits')."""
    dtype, ld = _logits(logits)
    T, N = logits.shape
    k, n_groups, top_groups = int(top_k), int(n_groups), int(top_groups)
    if (T | N | k | n_groups | top_groups) >> 31:
        _sizes(T | N | k | n_groups | top_groups, "xshare_gate")
    if logits.requires_grad:
        _no_gradient(logits, "logits", "gate_backward gives it")
    if bias is not None:
        _fit(logits.device, (bias, torch.float32, (N,), "bias"))
    ids, w = (None, None) if out is None else (out.get("ids"), out.get("w"))
    if ids is None:
        ids = logits.new_empty((T, max(k, 0)), dtype=torch.int32)
    else:
        _fit(logits.device, (ids, torch.int32, (T, k), "ids"))
    if w is None:
        w = logits.new_empty((T, max(k, 0)), dtype=torch.float32)
    else:
        _fit(logits.device, (w, torch.float32, (T, k), "w"))
    p = _gate_params(N, k, score, n_groups, top_groups, group_score, renormalize, scale)
    st = lib().xshare_gate(logits.data_ptr(), dtype, T, ld,
                           None if bias is None else bias.data_ptr(), ctypes.byref(p),
                           ids.data_ptr(), w.data_ptr(), _stream_of(logits, stream))
    _check(st, "xshare_gate")
    return dict(ids=ids, w=w)


@_placed
def gate_backward(logits: torch.Tensor, ids: torch.Tensor, dw: torch.Tensor, *, score="softmax",
                  renormalize: bool = True, scale: float = 1.0, out=None,
                  stream=None) -> torch.Tensor:
    """The gradient of the logits (fp32 [T, N]) from dw, the gradient of ``gate``'s weights, for
    its choice ids; score, renormalize and scale as given to ``gate``."""
    dtype, ld = _logits(logits)
    T, N = logits.shape
    k = ids.shape[1] if ids.dim() == 2 else -1
    if (T | N | k) >> 31:
        _sizes(T | N | k, "xshare_gate_backward")
    _fit(logits.device, (ids, torch.int32, (T, k), "ids"), (dw, torch.float32, (T, k), "dw"))
    if out is None:
        out = logits.new_empty((T, N), dtype=torch.float32)
    else:
        _fit(logits.device, (out, torch.float32, (T, N), "out"))
    p = _gate_params(N, k, score, 1, 1, "max", renormalize, scale)
    st = lib().xshare_gate_backward(logits.data_ptr(), dtype, T, ld, ctypes.byref(p),
                                    ids.data_ptr(), dw.data_ptr(), out.data_ptr(),
                                    _stream_of(logits, stream))
    _check(st, "xshare_gate_backward")
    return out


def _blocks(n):
    return (n + 127) // 128


@_placed
def block_quantize(x: torch.Tensor, block_rows: int = 1, *, out=None, stream=None) -> tuple:
    """(codes uint8 [rows, cols], scales fp32) of a bf16 matrix: E4M3FN with one scale for each
    block of block_rows x 128 (1: activations, 128: weights).  ``out``: the two to write."""
    ld = _rows(x, torch.bfloat16, "x")
    rows, cols = x.shape
    block_rows = int(block_rows)
    if (rows | cols | block_rows) >> 31:
        _sizes(rows | cols | block_rows, "xshare_block_quantize")
    step = max(block_rows, 1)
    shape = (-(-rows // step), _blocks(cols))
    q, s = (None, None) if out is None else out
    if q is None:
        q = x.new_empty((rows, cols), dtype=torch.uint8)
    else:
        _fit(x.device, (q, torch.uint8, (rows, cols), "codes"))
    if s is None:
        s = x.new_empty(shape, dtype=torch.float32)
    else:
        _fit(x.device, (s, torch.float32, shape, "scales"))
    st = lib().xshare_block_quantize(x.data_ptr(), rows, cols, ld, block_rows, q.data_ptr(),
                                     s.data_ptr(), _stream_of(x, stream))
    _check(st, "xshare_block_quantize")
    return q, s


def block_linear_workspace_bytes(T: int, n: int, k: int) -> int:
    T, n, k = int(T), int(n), int(k)
    if _past_32_bits(T | n | k):
        return 0                                  # as for other invalid sizes
    return int(lib().xshare_block_linear_workspace_bytes(T, n, k))


@_placed
def block_linear(x: torch.Tensor, wq: torch.Tensor, ws: torch.Tensor, *, x_scale=None, y=None,
                 workspace=None, stream=None) -> torch.Tensor:
    """y = x W^T (bf16 [T, n]) with W as codes wq uint8 [n, k] and scales ws of its 128 x 128
    blocks.  x is bf16, quantized here in 1 x 128 blocks, or with ``x_scale`` its codes
    (``block_quantize``).  Records no gradient: the input's is this call on dy with
    ``wq.t().contiguous()`` and ``ws.t().contiguous()``."""
    if wq.dim() != 2:
        raise ValueError("wq must be a matrix of codes")
    n, k = wq.shape
    own = x_scale is None
    if own:
        ldx = _rows(x, torch.bfloat16, "x", k)
    else:
        ldx = k
        _dev(x, torch.uint8, (x.shape[0], k), "x codes")
        _fit(x.device, (x_scale, torch.float32, (x.shape[0], _blocks(k)), "x_scale"))
    dev, T, L = x.device, x.shape[0], lib()
    if (T | n | k) >> 31:
        _sizes(T | n | k, "xshare_block_linear")
    if own and x.requires_grad:
        _no_gradient(x, "x", "it is block_linear of y's on the transposed codes and scales")
    _fit(dev, (wq, torch.uint8, (n, k), "wq"),
         (ws, torch.float32, (_blocks(n), _blocks(k)), "ws"))
    if y is None:
        y, ldy = x.new_empty((T, n), dtype=torch.bfloat16), n
    else:
        ldy = _rows(y, torch.bfloat16, "y", n)
        _on(dev, y, "y")
        if y.shape[0] != T:
            raise ValueError(f"y must have {T} rows, got {y.shape[0]}")
    size = 0
    if workspace is not None:
        size = _workspace(dev, workspace)
    elif own:
        size = L.xshare_block_linear_workspace_bytes(T, n, k)
        workspace = x.new_empty(size, dtype=torch.uint8)
    px = x.data_ptr()
    st = L.xshare_block_linear(px if own else None, ldx, None if own else px,
                                   None if own else x_scale.data_ptr(), T, n, k, wq.data_ptr(),
                                   ws.data_ptr(), y.data_ptr(), ldy,
                                   None if workspace is None else workspace.data_ptr(), size,
                                   _stream_of(x, stream))
    _check(st, "xshare_block_linear")
    return y


def block_experts_workspace_bytes(T: int, top_k: int, n_experts: int, d: int, f: int) -> int:
    T, k, N, d, f = int(T), int(top_k), int(n_experts), int(d), int(f)
    if _past_32_bits(T | k | N | d | f):
        return 0
    return int(lib().xshare_block_experts_workspace_bytes(T, k, N, d, f))


@_placed
def block_experts(x: torch.Tensor, ids: torch.Tensor, w: torch.Tensor, q1: torch.Tensor,
                  q3: torch.Tensor, q2: torch.Tensor, s1: torch.Tensor, s3: torch.Tensor,
                  s2: torch.Tensor, *, y=None, workspace=None, stream=None) -> torch.Tensor:
    """The routed SwiGLU experts of given pairs: y_i = sum_r w_ir E_{ids_ir}(x_i) (bf16 [T, d]),
    FP8 weights (codes uint8 [N, f, d], [N, f, d], [N, d, f]) with a scale for each 128 x 128
    block, activations quantized in 1 x 128 blocks.  ids and w [T, k] as ``gate`` or the set
    selections return them; a pair whose id is not in [0, N) is left out.  Records no gradient."""
    ldx = _rows(x, torch.bfloat16, "x")
    T, d = x.shape
    if q1.dim() != 3 or ids.dim() != 2:
        raise ValueError("weights are [N, f, d], ids [T, k]")
    N, f = q1.shape[0], q1.shape[1]
    k = ids.shape[1]
    dev, L = x.device, lib()
    if (T | k | N | d | f) >> 31:
        _sizes(T | k | N | d | f, "xshare_block_experts")
    if x.requires_grad or w.requires_grad:
        _no_gradient(x, "x", "there is no backward call")
        _no_gradient(w, "w", "there is no backward call")
    up, down = (N, _blocks(f), _blocks(d)), (N, _blocks(d), _blocks(f))
    _fit(dev, (ids, torch.int32, (T, k), "ids"), (w, torch.float32, (T, k), "w"),
         (q1, torch.uint8, (N, f, d), "w1 codes"), (q3, torch.uint8, (N, f, d), "w3 codes"),
         (q2, torch.uint8, (N, d, f), "w2 codes"), (s1, torch.float32, up, "w1 scales"),
         (s3, torch.float32, up, "w3 scales"), (s2, torch.float32, down, "w2 scales"))
    if y is None:
        y, ldy = x.new_empty((T, d)), d
    else:
        ldy = _rows(y, torch.bfloat16, "y", d)
        _on(dev, y, "y")
        if y.shape[0] != T:
            raise ValueError(f"y must have {T} rows, got {y.shape[0]}")
    if workspace is None:
        size = L.xshare_block_experts_workspace_bytes(T, k, N, d, f)
        workspace = x.new_empty(size, dtype=torch.uint8)
    else:
        size = _workspace(dev, workspace)
    a = BlockExpertsArgs(_EXPERTS_ARGS_BYTES, T, k, N, d, f, x.data_ptr(), ldx,
                         ids.data_ptr(), w.data_ptr(), q1.data_ptr(), q3.data_ptr(),
                         q2.data_ptr(), s1.data_ptr(), s3.data_ptr(), s2.data_ptr(),
                         y.data_ptr(), ldy, workspace.data_ptr(), size,
                         _stream_of(x, stream))
    _check(L.xshare_block_experts(ctypes.byref(a)), "xshare_block_experts")
    return y


@_placed
def probe_stream_read(buf: torch.Tensor, blocks: int = 2048, mode: int = 0, sink=None,
                      stream=None):
    """Enqueues one streaming read of ``buf`` (a contiguous GPU tensor, 16-byte aligned,
    size a multiple of 16 bytes; ``mode`` as xshare_probe_stream_read); time it with
    HipEvents on the same stream."""
    if not buf.is_cuda or not buf.is_contiguous():
        raise ValueError("buf must be a contiguous GPU tensor")
    if sink is None:
        sink = torch.zeros(1, dtype=torch.int32, device=buf.device)
    _check(lib().xshare_probe_stream_read(_ptr(buf), buf.numel() * buf.element_size(),
                                          int(blocks), int(mode), _ptr(sink),
                                          _stream(stream)),
           "xshare_probe_stream_read")
    return sink


def use_timeline_library() -> None:
    """Makes this process load the profiling build (libxshare_timeline.so) instead of the
    product library; call before the first call into the library."""
    global LIB_PATH
    if _lib is not None:
        raise RuntimeError("the library is already loaded")
    LIB_PATH = TIMELINE_LIB_PATH


@_placed
def block_times(clear: bool = True, stream=None) -> dict:
    """The block timeline of the last expert-GEMM launches (xshare_block_times; the profiling
    build only): uint64 arrays of 100 MHz clock stamps, "gate_up" and "down" [blocks, 2]
    (start, end) and "down_units" [blocks, 33] (start, then unit ends); 0 = not stamped.
    ``clear`` zeroes the stamps afterwards, so the next read holds only later launches."""
    dev = torch.device("cuda", torch.cuda.current_device())
    gu = torch.zeros(2 * TIME_BLOCKS, dtype=torch.int64, device=dev)
    dn = torch.zeros(2 * TIME_BLOCKS, dtype=torch.int64, device=dev)
    units = torch.zeros(TIME_SEQ_BLOCKS * TIME_SEQ_STRIDE, dtype=torch.int64, device=dev)
    _check(lib().xshare_block_times(_ptr(gu), _ptr(dn), _ptr(units), int(bool(clear)),
                                    _stream(stream)),
           "xshare_block_times")
    (stream or torch.cuda.current_stream()).synchronize()
    return {"gate_up": gu.cpu().numpy().view("uint64").reshape(-1, 2),
            "down": dn.cpu().numpy().view("uint64").reshape(-1, 2),
            "down_units": units.cpu().numpy().view("uint64").reshape(-1, TIME_SEQ_STRIDE)}
