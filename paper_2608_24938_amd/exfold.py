"""ctypes binding of libexfold (the C-ABI in include/exfold.h).

Argument marshalling only: torch supplies device memory and the current
stream; every step of the layer runs in the library's HIP kernels.  The
library is loaded on first use; a missing library raises ``RuntimeError``
(there is no fallback path).
"""

from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass

import torch

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libexfold.so")
_lib = None

(OK, ERR_NULL, ERR_SHAPE, ERR_BUDGET, ERR_DTYPE, ERR_WORKSPACE, ERR_DEVICE, ERR_UNSUPPORTED, ERR_ARG, ERR_ALIGN,
 ERR_SCRATCH) = range(11)
SCRATCH_BYTES = 64 << 20   # EXFOLD_SCRATCH_BYTES
F32, BF16 = 0, 1
PHASE = {"dense": 0, "prefill": 1, "decode": 2, "decode_static": 3, "prefill_diag": 4}
CAL_MODE = {"corouted": 0, "common": 1}
SCORE = {"softmax": 0, "sigmoid": 1}
ACT = {"none": 0, "relu": 1, "silu": 2, "gelu": 3, "gelu_tanh": 4}

EXPORTED = [
    "exfold_select_prefill", "exfold_select_decode_pool", "exfold_fold_gates", "exfold_static_pool",
    "exfold_moe_workspace_size", "exfold_moe_forward", "exfold_moe_forward_scratch",
    "exfold_execute_workspace_size",
    "exfold_moe_execute", "exfold_calibrate_workspace_size", "exfold_calibrate_projectors",
    "exfold_calibrate_diagonal",
    "exfold_status_str", "exfold_gemm_plan",
    "exfold_route_experts", "exfold_linear_workspace_size", "exfold_linear_forward", "exfold_linear_plan",
]


class ExfoldError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: status {status} ({status_str(status)})")


class _Layer(ctypes.Structure):
    _fields_ = [("d", ctypes.c_int64), ("inter", ctypes.c_int64), ("n_experts", ctypes.c_int64),
                ("top_k", ctypes.c_int64), ("shared_inter", ctypes.c_int64), ("dtype", ctypes.c_int32),
                ("reserved", ctypes.c_int32), ("w_router", ctypes.c_void_p), ("router_bias", ctypes.c_void_p),
                ("w_gate_up", ctypes.c_void_p), ("w_down", ctypes.c_void_p),
                ("ws_gate_up", ctypes.c_void_p), ("ws_down", ctypes.c_void_p)]


class _Tables(ctypes.Structure):
    _fields_ = [("S", ctypes.c_void_p), ("L", ctypes.c_void_p), ("h", ctypes.c_void_p),
                ("tgt", ctypes.c_void_p), ("scl", ctypes.c_void_p), ("loss_cap", ctypes.c_float),
                ("fold_flags", ctypes.c_int32), ("Dg", ctypes.c_void_p)]


class _Routing(ctypes.Structure):
    _fields_ = [("score", ctypes.c_int32), ("group_value", ctypes.c_int32), ("n_groups", ctypes.c_int64),
                ("keep_groups", ctypes.c_int64), ("renorm", ctypes.c_int32), ("scale", ctypes.c_float),
                ("select_bias", ctypes.c_void_p)]


class _Linear(ctypes.Structure):
    _fields_ = [("n_in", ctypes.c_int64), ("n_out", ctypes.c_int64), ("ldw", ctypes.c_int64), ("w", ctypes.c_void_p),
                ("bias", ctypes.c_void_p), ("dtype", ctypes.c_int32), ("out_dtype", ctypes.c_int32),
                ("act", ctypes.c_int32), ("gated", ctypes.c_int32)]


FOLD_LOSS_CAP, FOLD_RENORM, FOLD_CONFIDENCE = 1, 2, 4


def fold_opts(loss_cap=None, renorm=False, confidence=False):
    """(loss_cap, fold_flags) of the prefill fold safeguards (EXFOLD_FOLD_* in the header)."""
    flags = (FOLD_LOSS_CAP if loss_cap is not None else 0) | (FOLD_RENORM if renorm else 0) | \
        (FOLD_CONFIDENCE if confidence else 0)
    return (0.0 if loss_cap is None else float(loss_cap)), flags


_DEBUG_FIELDS = ["logits", "topk_ids", "topk_w", "keep", "pool", "pool_size", "tgt_ids", "tgt_scale",
                 "fold_ids", "fold_w", "offsets", "row_slot"]


N_EVENTS = 7
EVENT_NAMES = ["start", "router", "fold", "permute", "gate_up", "down", "end"]


class _Debug(ctypes.Structure):
    _fields_ = [(f, ctypes.c_void_p) for f in _DEBUG_FIELDS] + [("events", ctypes.c_void_p)]


def lib() -> ctypes.CDLL:
    """Load libexfold.so (built in-tree by paper_2608_24938_amd.build)."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise RuntimeError(f"libexfold.so is not built ({_LIB_PATH}); run paper_2608_24938_amd.build")
        L = ctypes.CDLL(_LIB_PATH)
        i64, i32, vp, sz = ctypes.c_int64, ctypes.c_int32, ctypes.c_void_p, ctypes.c_size_t
        dbl = ctypes.c_double
        sig = {
            "exfold_select_prefill": (i32, [vp, i64, i64, i64, i64, vp, vp, vp, vp, vp]),
            "exfold_select_decode_pool": (i32, [vp, i64, i64, i64, i64, vp, vp, vp, vp, vp, vp]),
            "exfold_fold_gates": (i32, [i32, i64, i64, i64, i64, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp,
                                        ctypes.c_float, i32, vp]),
            "exfold_static_pool": (i32, [vp, i64, i64, vp, vp, vp, vp, vp, vp, vp]),
            "exfold_moe_workspace_size": (sz, [vp, i64, i32, i64]),
            "exfold_moe_forward": (i32, [vp, vp, vp, i64, i32, i64, vp, vp, vp, sz, vp]),
            "exfold_moe_forward_scratch": (i32, [vp, vp, vp, i64, i32, i64, vp, vp, vp]),
            "exfold_execute_workspace_size": (sz, [vp, i64, i64]),
            "exfold_moe_execute": (i32, [vp, vp, i64, i64, vp, vp, vp, vp, vp, sz, vp]),
            "exfold_calibrate_workspace_size": (sz, [vp, i64, i32]),
            "exfold_calibrate_projectors": (i32, [vp, vp, i64, dbl, dbl, i32, vp, vp, vp, vp, vp, sz, vp]),
            "exfold_calibrate_diagonal": (i32, [vp, vp, i64, dbl, i32, vp, vp, vp, sz, vp]),
            "exfold_status_str": (ctypes.c_char_p, [i32]),
            "exfold_gemm_plan": (i32, [vp, i64, i64, i32, vp]),
            "exfold_route_experts": (i32, [vp, vp, i32, i64, i64, i64, i64, vp, vp, vp]),
            "exfold_linear_workspace_size": (sz, [vp, i64]),
            "exfold_linear_forward": (i32, [vp, vp, i64, i64, vp, i64, vp, i64, vp, sz, vp]),
            "exfold_linear_plan": (i32, [vp, i64, i32, i32, vp]),
        }
        for name, (res, args) in sig.items():
            fn = getattr(L, name)
            fn.restype = res
            fn.argtypes = args
        _lib = L
    return _lib


def status_str(status: int) -> str:
    return lib().exfold_status_str(status).decode()


def _check(status: int, where: str):
    if status != OK:
        raise ExfoldError(status, where)


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream=None):
    s = stream if stream is not None else torch.cuda.current_stream()
    return ctypes.c_void_p(s.cuda_stream)


def _need(t, dtype, shape, name):
    if t.dtype != dtype or tuple(t.shape) != tuple(shape) or not t.is_contiguous() or not t.is_cuda:
        raise ValueError(f"{name}: expected contiguous {dtype} {tuple(shape)} on the GPU, "
                         f"got {t.dtype} {tuple(t.shape)} on {t.device}")


@dataclass
class Layer:
    """Device weights of one MoE layer (bf16 weights are torch.bfloat16 tensors)."""
    w_router: torch.Tensor          # [N, d]
    w_gate_up: torch.Tensor         # [N, 2I, d]
    w_down: torch.Tensor            # [N, d, I]
    top_k: int
    router_bias: torch.Tensor | None = None   # [N] float32
    ws_gate_up: torch.Tensor | None = None    # [2I_s, d]
    ws_down: torch.Tensor | None = None       # [d, I_s]

    @property
    def n_experts(self):
        return self.w_router.shape[0]

    @property
    def d(self):
        return self.w_router.shape[1]

    @property
    def inter(self):
        return self.w_down.shape[2]

    @property
    def dtype(self):
        return self.w_router.dtype

    def struct(self) -> _Layer:
        code = {torch.bfloat16: BF16, torch.float32: F32}[self.dtype]
        return _Layer(self.d, self.inter, self.n_experts, self.top_k,
                      0 if self.ws_down is None else self.ws_down.shape[1], code, 0,
                      self.w_router.data_ptr(), None if self.router_bias is None else self.router_bias.data_ptr(),
                      self.w_gate_up.data_ptr(), self.w_down.data_ptr(),
                      None if self.ws_gate_up is None else self.ws_gate_up.data_ptr(),
                      None if self.ws_down is None else self.ws_down.data_ptr())


def _workspace(nbytes: int, device, stream=None) -> torch.Tensor:
    """Temporary workspace for one call.  torch's caching allocator returns 256-byte aligned
    blocks (512 in practice).  When the call runs on another stream than the current one, the
    block is tied to that stream too (record_stream), so the allocator does not hand it out
    again while the call's kernels may still use it."""
    ws = torch.empty(max(int(nbytes), 1), dtype=torch.uint8, device=device)
    if stream is not None:
        ws.record_stream(stream)
    return ws


def select_prefill(h, k_pre, logits=None, topk_ids=None, topk_w=None, top_k=None, stream=None):
    """Top-K routes (from logits, or given) and the prefill keep mask. Returns (ids, w, keep)."""
    if logits is not None:
        T, N = logits.shape
        K = top_k
        topk_ids = torch.empty((T, K), dtype=torch.int32, device=logits.device)
        topk_w = torch.empty((T, K), dtype=torch.float32, device=logits.device)
    else:
        T, K = topk_ids.shape
        N = h.shape[0]
    keep = torch.empty((T, K), dtype=torch.uint8, device=h.device)
    _check(lib().exfold_select_prefill(_ptr(logits), T, N, K, k_pre, _ptr(h), _ptr(topk_ids), _ptr(topk_w),
                                       _ptr(keep), _stream(stream)), "exfold_select_prefill")
    return topk_ids, topk_w, keep


def select_decode_pool(h, budget, logits=None, topk_ids=None, topk_w=None, top_k=None, stream=None):
    """Top-K routes (from logits, or given) and the decode pool. Returns (ids, w, pool, pool_size)."""
    N = h.shape[0]
    if logits is not None:
        B = logits.shape[0]
        K = top_k
        topk_ids = torch.empty((B, K), dtype=torch.int32, device=logits.device)
        topk_w = torch.empty((B, K), dtype=torch.float32, device=logits.device)
    else:
        B, K = topk_ids.shape
    pool = torch.empty((min(budget, N),), dtype=torch.int32, device=h.device)
    pool_size = torch.empty((1,), dtype=torch.int32, device=h.device)
    _check(lib().exfold_select_decode_pool(_ptr(logits), B, N, K, budget, _ptr(h), _ptr(topk_ids), _ptr(topk_w),
                                           _ptr(pool), _ptr(pool_size), _stream(stream)),
           "exfold_select_decode_pool")
    return topk_ids, topk_w, pool, pool_size


def fold_gates(phase, budget, topk_ids, topk_w, S, L, keep=None, pool=None, pool_size=None, tables=False,
               stream=None, loss_cap=None, renorm=False, confidence=False):
    """Fold route metadata. Returns (out_ids, out_w) or (out_ids, out_w, tgt, scl) with tables=True.

    loss_cap/renorm/confidence: the prefill safeguards (see fold_opts)."""
    T, K = topk_ids.shape
    N = S.shape[0]
    ph = PHASE[phase]
    k_out = min(budget, K) if phase == "prefill" else K
    dev = S.device
    out_ids = torch.empty((T, k_out), dtype=torch.int32, device=dev)
    out_w = torch.empty((T, k_out), dtype=torch.float32, device=dev)
    tgt = torch.empty((N,), dtype=torch.int32, device=dev) if tables else None
    scl = torch.empty((N,), dtype=torch.float32, device=dev) if tables else None
    _check(lib().exfold_fold_gates(ph, T, N, K, budget, _ptr(topk_ids), _ptr(topk_w), _ptr(keep), _ptr(pool),
                                   _ptr(pool_size), _ptr(S), _ptr(L), _ptr(out_ids), _ptr(out_w), _ptr(tgt),
                                   _ptr(scl), *fold_opts(loss_cap, renorm, confidence), _stream(stream)),
           "exfold_fold_gates")
    return (out_ids, out_w, tgt, scl) if tables else (out_ids, out_w)


def static_pool(h, budget, S, L, stream=None):
    """Static decode pool TopK(h, D) and its per-source tables. Returns (pool, pool_size, tgt, scl)."""
    N = h.shape[0]
    dev = h.device
    pool = torch.empty((min(budget, N),), dtype=torch.int32, device=dev)
    pool_size = torch.empty((1,), dtype=torch.int32, device=dev)
    tgt = torch.empty((N,), dtype=torch.int32, device=dev)
    scl = torch.empty((N,), dtype=torch.float32, device=dev)
    _check(lib().exfold_static_pool(_ptr(h), N, budget, _ptr(S), _ptr(L), _ptr(pool), _ptr(pool_size), _ptr(tgt),
                                    _ptr(scl), _stream(stream)), "exfold_static_pool")
    return pool, pool_size, tgt, scl


def moe_workspace_size(layer: Layer, T: int, phase: str, budget: int) -> int:
    ls = layer.struct()
    n = lib().exfold_moe_workspace_size(ctypes.byref(ls), T, PHASE[phase], budget)
    if n == 0 and T > 0:
        raise ValueError("invalid layer/shape for exfold_moe_forward")
    return n


def debug_buffers(layer: Layer, T: int, phase: str, budget: int, device) -> dict:
    """Device buffers for every intermediate of the forward (see exfold_debug)."""
    N, K = layer.n_experts, layer.top_k
    k_out = min(budget, K) if phase == "prefill" else K
    R = T * k_out
    i32, f32 = torch.int32, torch.float32
    return {
        "logits": torch.empty((T, N), dtype=f32, device=device),
        "topk_ids": torch.empty((T, K), dtype=i32, device=device),
        "topk_w": torch.empty((T, K), dtype=f32, device=device),
        "keep": torch.empty((T, K), dtype=torch.uint8, device=device),
        "pool": torch.empty((max(1, min(budget, N)),), dtype=i32, device=device),
        "pool_size": torch.empty((1,), dtype=i32, device=device),
        "tgt_ids": torch.empty((N,), dtype=i32, device=device),
        "tgt_scale": torch.empty((N,), dtype=f32, device=device),
        "fold_ids": torch.empty((T, k_out), dtype=i32, device=device),
        "fold_w": torch.empty((T, k_out), dtype=f32, device=device),
        "offsets": torch.empty((N + 2,), dtype=i32, device=device),
        "row_slot": torch.empty((R + (T if layer.ws_down is not None else 0),), dtype=i32, device=device),
    }


def moe_forward(layer: Layer, x, phase: str = "dense", budget: int = 0, S=None, L=None, h=None, y=None,
                debug: dict | None = None, workspace=None, stream=None, events=None, static_tables=None,
                safeguards: dict | None = None, diag=None):
    """Folded MoE layer forward; returns y [T, d] (dtype of the layer).

    static_tables: (tgt, scl) from static_pool, for phase "decode_static".
    safeguards: prefill fold safeguards, keyword arguments of fold_opts.
    diag: [N, N, d] diagonal maps from calibrate_diagonal, for phase "prefill_diag" (L is then the
    diagonal loss table).
    events: optional ctypes array of N_EVENTS hipEvent_t handles recorded at the stage boundaries."""
    T = x.shape[0]
    _need(x, layer.dtype, (T, layer.d), "x")
    if y is None:
        y = torch.empty_like(x)
    ls = layer.struct()
    tgt, scl = static_tables if static_tables is not None else (None, None)
    cap, flags = fold_opts(**(safeguards or {}))
    tb = _Tables(_ptr(S), _ptr(L), _ptr(h), _ptr(tgt), _ptr(scl), cap, flags, _ptr(diag)) \
        if (S is not None or L is not None or tgt is not None) else None
    dbg = None
    if debug is not None or events is not None:
        debug = debug or {}
        dbg = _Debug(*[_ptr(debug.get(f)) for f in _DEBUG_FIELDS],
                     None if events is None else ctypes.cast(events, ctypes.c_void_p))
    need = lib().exfold_moe_workspace_size(ctypes.byref(ls), T, PHASE[phase], budget)
    if workspace is None:
        workspace = _workspace(need, x.device, stream)
    _check(lib().exfold_moe_forward(ctypes.byref(ls), None if tb is None else ctypes.byref(tb), _ptr(x), T,
                                    PHASE[phase], budget, _ptr(y), None if dbg is None else ctypes.byref(dbg),
                                    _ptr(workspace), workspace.numel(), _stream(stream)), "exfold_moe_forward")
    return y


def moe_forward_scratch(layer: Layer, x, phase: str = "dense", budget: int = 0, S=None, L=None, h=None, y=None,
                        debug: dict | None = None, stream=None, static_tables=None,
                        safeguards: dict | None = None, diag=None):
    """moe_forward on the library's static scratch (exfold_moe_forward_scratch): no workspace is
    allocated; y must be given by callers that cannot allocate (otherwise it is created here)."""
    T = x.shape[0]
    _need(x, layer.dtype, (T, layer.d), "x")
    if y is None:
        y = torch.empty_like(x)
    ls = layer.struct()
    tgt, scl = static_tables if static_tables is not None else (None, None)
    cap, flags = fold_opts(**(safeguards or {}))
    tb = _Tables(_ptr(S), _ptr(L), _ptr(h), _ptr(tgt), _ptr(scl), cap, flags, _ptr(diag)) \
        if (S is not None or L is not None or tgt is not None) else None
    dbg = None
    if debug is not None:
        dbg = _Debug(*[_ptr(debug.get(f)) for f in _DEBUG_FIELDS], None)
    _check(lib().exfold_moe_forward_scratch(ctypes.byref(ls), None if tb is None else ctypes.byref(tb), _ptr(x), T,
                                            PHASE[phase], budget, _ptr(y),
                                            None if dbg is None else ctypes.byref(dbg), _stream(stream)),
           "exfold_moe_forward_scratch")
    return y


def moe_execute(layer: Layer, x, route_ids, route_w, y=None, debug: dict | None = None, stream=None):
    """Run the experts on given routes [T, K_out] and combine; returns y."""
    T, k_out = route_ids.shape
    if y is None:
        y = torch.empty_like(x)
    ls = layer.struct()
    dbg = None
    if debug is not None:
        dbg = _Debug(*[_ptr(debug.get(f)) for f in _DEBUG_FIELDS], None)
    need = lib().exfold_execute_workspace_size(ctypes.byref(ls), T, k_out)
    ws = _workspace(need, x.device, stream)
    _check(lib().exfold_moe_execute(ctypes.byref(ls), _ptr(x), T, k_out, _ptr(route_ids), _ptr(route_w), _ptr(y),
                                    None if dbg is None else ctypes.byref(dbg), _ptr(ws), ws.numel(),
                                    _stream(stream)), "exfold_moe_execute")
    return y


def calibrate_projectors(layer: Layer, x_cal, lam: float = 1e-3, clip: float = 4.0, mode: str = "corouted",
                         with_stats: bool = False, stream=None):
    """Projector calibration; returns (S, L, h) float32 device tensors (+ stats [N,N,4] float64)."""
    m = x_cal.shape[0]
    N = layer.n_experts
    dev = x_cal.device
    ls = layer.struct()
    S = torch.empty((N, N), dtype=torch.float32, device=dev)
    L = torch.empty((N, N), dtype=torch.float32, device=dev)
    h = torch.empty((N,), dtype=torch.float32, device=dev)
    stats = torch.empty((N, N, 4), dtype=torch.float64, device=dev) if with_stats else None
    need = lib().exfold_calibrate_workspace_size(ctypes.byref(ls), m, CAL_MODE[mode])
    ws = _workspace(need, dev, stream)
    _check(lib().exfold_calibrate_projectors(ctypes.byref(ls), _ptr(x_cal), m, lam, clip, CAL_MODE[mode], _ptr(S),
                                             _ptr(L), _ptr(h), _ptr(stats), _ptr(ws), ws.numel(), _stream(stream)),
           "exfold_calibrate_projectors")
    return (S, L, h, stats) if with_stats else (S, L, h)


def calibrate_diagonal(layer: Layer, x_cal, lam: float = 1e-3, mode: str = "corouted", stream=None):
    """Diagonal projector calibration; returns (Dg [N, N, d], Ld [N, N]) float32 device tensors."""
    m = x_cal.shape[0]
    N, d = layer.n_experts, layer.d
    dev = x_cal.device
    ls = layer.struct()
    Dg = torch.empty((N, N, d), dtype=torch.float32, device=dev)
    Ld = torch.empty((N, N), dtype=torch.float32, device=dev)
    need = lib().exfold_calibrate_workspace_size(ctypes.byref(ls), m, CAL_MODE[mode])
    ws = _workspace(need, dev, stream)
    _check(lib().exfold_calibrate_diagonal(ctypes.byref(ls), _ptr(x_cal), m, lam, CAL_MODE[mode], _ptr(Dg), _ptr(Ld),
                                           _ptr(ws), ws.numel(), _stream(stream)), "exfold_calibrate_diagonal")
    return Dg, Ld


_DTYPE = {torch.float32: F32, torch.bfloat16: BF16}
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
    (lambda index: torch.cuda.current_stream(index).cuda_stream)   # the handle without the Stream object's 2.5 us


def _matrix(t, name, dtype=None, shape=None, device=None):
    """Row stride of a 2-D GPU tensor whose rows are contiguous (gaps between rows allowed)."""
    sh = t.shape
    if len(sh) != 2 or not t.is_cuda or t.dtype not in _DTYPE or (sh[1] > 1 and t.stride(1) != 1) \
            or (dtype is not None and t.dtype != dtype) or (shape is not None and sh != shape) \
            or (device is not None and t.device != device):
        raise ValueError(f"{name}: expected a 2-D {dtype or 'float32 or bfloat16'} tensor"
                         f"{'' if shape is None else f' {tuple(shape)}'} with contiguous rows on "
                         f"{'the GPU' if device is None else device}, got {t.dtype} {tuple(sh)} with strides "
                         f"{t.stride()} on {t.device}")
    return t.stride(0) if sh[0] > 1 else sh[1]


def _vector(t, n, name, device):
    """Address of a float32 vector of n entries, or None."""
    if t is None:
        return None
    if t.dtype != torch.float32 or t.shape != (n,) or not t.is_contiguous() or t.device != device:
        raise ValueError(f"{name}: expected contiguous float32 ({n},) on {device}, got {t.dtype} {tuple(t.shape)} "
                         f"on {t.device}")
    return t.data_ptr()


def _output(t, dtype, shape, name, device):
    _need(t, dtype, shape, name)
    if t.device != device:
        raise ValueError(f"{name}: expected on {device}, got {t.device}")


def _call(device, fn, *args):
    """fn(*args, stream) with the tensors' device current, on that device's current stream."""
    index = device.index
    if index == torch.cuda.current_device():
        return fn(*args, _raw_stream(index))
    with torch.cuda.device(index):
        return fn(*args, _raw_stream(index))


def _on_stream(stream, device):
    """The context of a call on a given stream: what it allocates belongs to that stream too."""
    if stream.device != device:
        raise ValueError(f"the stream is on {stream.device}, the tensors on {device}")
    return torch.cuda.stream(stream)


def route_experts(logits, top_k, score="softmax", select_bias=None, groups=1, keep_groups=1, group_top2=False,
                  renorm=True, scale=1.0, topk_ids=None, topk_w=None, stream=None):
    """Routes of every token from its router logits [T, N] (float32 or bfloat16): (ids [T, K] int32, w [T, K] float32).

    score: "softmax" or "sigmoid" over all experts.  select_bias: [N] float32 added to the scores for the
    selection only.  groups, keep_groups: the selection is limited to the keep_groups of `groups` groups of
    consecutive experts with the largest value (their largest expert, or group_top2: the sum of the two
    largest).  renorm: the weights of a token's routes are divided by their sum; scale multiplies them.
    A logit of -inf masks its expert (see exfold_routing in the header).  topk_ids/topk_w: optional outputs.
    stream: as under torch.cuda.stream(stream)."""
    ld = _matrix(logits, "logits")
    T, N = logits.shape
    dev = logits.device
    if stream is not None:
        with _on_stream(stream, dev):
            return route_experts(logits, top_k, score, select_bias, groups, keep_groups, group_top2, renorm, scale,
                                 topk_ids, topk_w)
    bias = _vector(select_bias, N, "select_bias", dev)
    if score not in SCORE:
        raise ValueError(f"score: expected one of {sorted(SCORE)}, got {score!r}")
    if topk_ids is None:
        topk_ids = torch.empty(T, top_k, dtype=torch.int32, device=dev)
    else:
        _output(topk_ids, torch.int32, (T, top_k), "topk_ids", dev)
    if topk_w is None:
        topk_w = torch.empty(T, top_k, dtype=torch.float32, device=dev)
    else:
        _output(topk_w, torch.float32, (T, top_k), "topk_w", dev)
    r = _Routing(SCORE[score], 1 if group_top2 else 0, groups, keep_groups, 1 if renorm else 0, scale, bias)
    status = _call(dev, lib().exfold_route_experts, ctypes.byref(r), logits.data_ptr(), _DTYPE[logits.dtype], ld, T, N,
                   top_k, topk_ids.data_ptr(), topk_w.data_ptr())
    if status != OK:
        raise ExfoldError(status, "exfold_route_experts")
    return topk_ids, topk_w


def linear_workspace_size(w, rows, gated=False) -> int:
    """Bytes of workspace that linear() of exactly `rows` rows of x and this weight needs (0: none; fewer rows may need
    more).  Enough for any x: one whose rows start on 16 bytes may need less."""
    ldw = _matrix(w, "w")
    n_out = w.shape[0] // 2 if gated else w.shape[0]
    code = _DTYPE[w.dtype]
    ls = _Linear(w.shape[1], n_out, ldw, w.data_ptr(), None, code, code, 0, 1 if gated else 0)
    return _call(w.device, lambda _: lib().exfold_linear_workspace_size(ctypes.byref(ls), rows))


def linear(x, w, bias=None, act="none", gated=False, residual=None, out_dtype=None, y=None, workspace=None, stream=None):
    """y = act(x w^T + bias) + residual; gated: y = act(x w_g^T + b_g) * (x w_u^T + b_u) + residual.

    x [M, n_in] and w [n_out, n_in] (gated: [2 n_out, n_in], gate rows first) of one type, float32 or
    bfloat16, rows contiguous; bias [n_out] (gated [2 n_out]) float32; residual and y [M, n_out] of
    out_dtype (x's type unless given; float32 is always allowed).  y may be the residual (y += ...).
    act: "none", "relu", "silu", "gelu" or "gelu_tanh".  workspace: a tensor of at least
    linear_workspace_size bytes for these rows; made here, where one is needed, unless given.  stream: as under
    torch.cuda.stream(stream)."""
    ldx = _matrix(x, "x")
    dev, dtype = x.device, x.dtype
    if stream is not None:
        with _on_stream(stream, dev):
            return linear(x, w, bias, act, gated, residual, out_dtype, y, workspace)
    M, K = x.shape
    ldw = _matrix(w, "w", dtype, None, dev)
    rows, kw = w.shape
    n_out = rows
    if gated:
        if rows % 2:
            raise ValueError(f"w: a gated product has as many gate as up rows, got {rows} rows")
        n_out = rows // 2
    if kw != K:
        raise ValueError(f"w: expected rows of {K} elements, those of x, got {kw}")
    b = _vector(bias, rows, "bias", dev)
    if out_dtype is None:
        out_dtype = dtype if y is None else y.dtype
    if out_dtype not in _DTYPE:
        raise ValueError(f"out_dtype: expected float32 or bfloat16, got {out_dtype}")
    if act not in ACT:
        raise ValueError(f"act: expected one of {sorted(ACT)}, got {act!r}")
    res, ldr = None, 0
    if residual is not None:
        ldr, res = _matrix(residual, "residual", out_dtype, (M, n_out), dev), residual.data_ptr()
    if y is None:
        y, ldy = torch.empty(M, n_out, dtype=out_dtype, device=dev), n_out
    else:
        ldy = _matrix(y, "y", out_dtype, (M, n_out), dev)
    if workspace is not None and (workspace.device != dev or not workspace.is_contiguous()):
        raise ValueError(f"workspace: expected a contiguous tensor on {dev}, got one on {workspace.device}")
    p = ctypes.byref(_Linear(K, n_out, ldw, w.data_ptr(), b, _DTYPE[dtype], _DTYPE[out_dtype], ACT[act], 1 if gated else 0))
    L = lib()
    args = (p, x.data_ptr(), ldx, M, res, ldr, y.data_ptr(), ldy)
    if workspace is None:  # most small products need none: ask for its size only when the call does
        status = _call(dev, L.exfold_linear_forward, *args, None, 0)
        if status == ERR_WORKSPACE:
            workspace = _workspace(_call(dev, lambda _: L.exfold_linear_workspace_size(p, M)), dev)
    if workspace is not None:
        status = _call(dev, L.exfold_linear_forward, *args, workspace.data_ptr(),
                       workspace.numel() * workspace.element_size())
    if status != OK:
        raise ExfoldError(status, "exfold_linear_forward")
    return y
