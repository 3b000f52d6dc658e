"""ctypes binding of libswitch_moe.so: the same entry points as include/switch_moe.h, taking torch tensors.

Argument marshalling only: every step of the layer runs in the library's CUDA kernels.  PyTorch is used for
device memory and streams.  There is no fallback: if the shared library is missing, loading raises.
"""
from __future__ import annotations

import ctypes
import os

import torch

_PKG_DIR = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG_DIR, "libswitch_moe.so")

BF16, F32 = 0, 1
STAGE_EVENTS = 13
STAGE_NAMES = ["router_fwd", "dispatch_plan", "gather_x", "gemm1_relu", "gemm2_combine", None,
               "gather_dy", "dgrad2_mask", "wgrad2", "dgrad1_scatter", "wgrad1", "router_bwd"]
GEMM_DEFAULT, GEMM_SIMT, GEMM_TC_1CTA = 0, 1, 2

OK = 0
INVALID_ARGUMENT, UNSUPPORTED_SHAPE, WORKSPACE_TOO_SMALL, CUDA_ERROR, DEVICE_TIMEOUT = -1, -2, -3, -4, -5

WS_STATUS, WS_EXPERT_INDEX, WS_GATE, WS_SLOT, WS_TOKEN_OF_SLOT, WS_COUNT, WS_KEPT, WS_PSUM, WS_PROBS, WS_XD, WS_H, \
    WS_DYD, WS_DH, WS_DGATE, WS_DLOGITS, WS_LAYER_Y, WS_EXPERT_PROC, WS_SECOND_CHOICE = range(18)
FLAG_RESIDUAL, FLAG_REROUTE, FLAG_INPUT_JITTER, FLAG_GEGLU, FLAG_TOP2, FLAG_EXPERT_DROPOUT = 1, 2, 4, 8, 16, 32

EXPORTED_SYMBOLS = [
    "switch_moe_capacity", "switch_moe_workspace_bytes", "switch_moe_workspace_view", "switch_moe_fwd",
    "switch_moe_bwd", "switch_moe_router_fwd", "switch_moe_dispatch_plan", "switch_moe_router_bwd",
    "switch_moe_dispatch_plan_static", "switch_moe_step_host", "switch_moe_step_host_enqueue",
    "switch_moe_check_device_status", "switch_moe_launches_per_step", "switch_moe_stage_launches",
    "switch_moe_status_string",
    "switch_moe_linear_workspace_bytes", "switch_moe_linear_fwd", "switch_moe_linear_bwd",
    "switch_moe_linear_check_device_status", "switch_moe_dropout_fwd", "switch_moe_dropout_bwd",
    "switch_moe_balance_workspace_bytes", "switch_moe_balance_fwd", "switch_moe_balance_bwd",
]


class SwitchMoeConfig(ctypes.Structure):
    """Mirror of `switch_moe_config`."""

    _fields_ = [
        ("T", ctypes.c_int32), ("d_model", ctypes.c_int32), ("d_ff", ctypes.c_int32), ("E", ctypes.c_int32),
        ("capacity_factor", ctypes.c_float), ("alpha", ctypes.c_float),
        ("capacity_override", ctypes.c_int32), ("dtype", ctypes.c_int32), ("gemm_path", ctypes.c_int32),
        ("flags", ctypes.c_int32), ("groups", ctypes.c_int32), ("reroute_stages", ctypes.c_int32),
        ("reserved", ctypes.c_int32 * 2),
        ("stage_events", ctypes.POINTER(ctypes.c_void_p)),
        ("router_noise", ctypes.c_void_p),
        ("router_jitter", ctypes.c_void_p),
        ("expert_keep", ctypes.c_void_p),
        ("expert_dropout", ctypes.c_float),
    ]


ACT_NONE, ACT_RELU, ACT_GELU = 0, 1, 2


class LinearConfig(ctypes.Structure):
    """Mirror of `switch_moe_linear_config`."""

    _fields_ = [
        ("M", ctypes.c_int32), ("K", ctypes.c_int32), ("N", ctypes.c_int32), ("dtype", ctypes.c_int32),
        ("activation", ctypes.c_int32), ("site", ctypes.c_int32), ("dropout", ctypes.c_float),
        ("ldx", ctypes.c_int32), ("ldw", ctypes.c_int32), ("ldy", ctypes.c_int32), ("reserved", ctypes.c_int32 * 2),
    ]


class DropoutConfig(ctypes.Structure):
    """Mirror of `switch_moe_dropout_config`."""

    _fields_ = [
        ("rows", ctypes.c_int32), ("cols", ctypes.c_int32), ("ld", ctypes.c_int32), ("dtype", ctypes.c_int32),
        ("site", ctypes.c_int32), ("rate", ctypes.c_float), ("reserved", ctypes.c_int32 * 2),
    ]


class BalanceConfig(ctypes.Structure):
    """Mirror of `switch_moe_balance_config`."""

    _fields_ = [
        ("T", ctypes.c_int32), ("E", ctypes.c_int32), ("k", ctypes.c_int32), ("groups", ctypes.c_int32),
        ("dtype", ctypes.c_int32), ("ld", ctypes.c_int32), ("alpha", ctypes.c_float), ("reserved", ctypes.c_int32 * 2),
    ]


class SwitchMoeError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} ({status})")


_lib = None


def load_library() -> ctypes.CDLL:
    """Loads libswitch_moe.so (built in-tree by paper_2101_03961_b200.build); raises if it is not there."""
    global _lib
    if _lib is not None:
        return _lib
    path = os.environ.get("SWITCH_MOE_LIBRARY", LIB_PATH)      # override: another build of the same library
    if not os.path.exists(path):
        raise FileNotFoundError(
            f"{path} not found: build it with `python -m paper_2101_03961_b200.build` (there is no fallback path)")
    lib = ctypes.CDLL(path)
    vp, cp = ctypes.c_void_p, ctypes.POINTER(SwitchMoeConfig)
    i32p, szp = ctypes.POINTER(ctypes.c_int32), ctypes.POINTER(ctypes.c_size_t)
    lib.switch_moe_capacity.argtypes = [cp, i32p]
    lib.switch_moe_workspace_bytes.argtypes = [cp, szp]
    lib.switch_moe_workspace_view.argtypes = [cp, vp, ctypes.c_int32, ctypes.POINTER(vp), szp]
    lib.switch_moe_fwd.argtypes = [cp, vp, vp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
    lib.switch_moe_bwd.argtypes = [cp, vp, ctypes.c_float, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp, vp, vp, vp, vp]
    lib.switch_moe_router_fwd.argtypes = [cp, vp, vp, vp, vp, ctypes.c_size_t, vp]
    lib.switch_moe_dispatch_plan.argtypes = [cp, vp, vp, vp, ctypes.c_size_t, vp]
    lib.switch_moe_dispatch_plan_static.argtypes = [cp, vp, vp, vp, vp, vp, vp]
    lib.switch_moe_router_bwd.argtypes = [cp, vp, vp, vp, ctypes.c_float, vp, ctypes.c_size_t, vp, vp, vp]
    lib.switch_moe_step_host.argtypes = [cp, vp, vp, ctypes.c_float] + [vp] * 15 + [vp, ctypes.c_size_t, vp, vp, vp]
    lib.switch_moe_step_host_enqueue.argtypes = lib.switch_moe_step_host.argtypes + [vp, vp]
    lib.switch_moe_check_device_status.argtypes = [cp, vp, i32p, vp]
    lib.switch_moe_launches_per_step.argtypes = [cp, i32p]
    lib.switch_moe_stage_launches.argtypes = [cp, i32p]
    lib.switch_moe_status_string.argtypes = [ctypes.c_int]
    lib.switch_moe_status_string.restype = ctypes.c_char_p
    lp, dp, bp = ctypes.POINTER(LinearConfig), ctypes.POINTER(DropoutConfig), ctypes.POINTER(BalanceConfig)
    lib.switch_moe_linear_workspace_bytes.argtypes = [lp, ctypes.c_int32, szp]
    lib.switch_moe_linear_fwd.argtypes = [lp] + [vp] * 8 + [ctypes.c_size_t, vp]
    lib.switch_moe_linear_bwd.argtypes = [lp] + [vp] * 6 + [ctypes.c_size_t] + [vp] * 4
    lib.switch_moe_linear_check_device_status.argtypes = [lp, vp, i32p, vp]
    lib.switch_moe_dropout_fwd.argtypes = [dp] + [vp] * 5
    lib.switch_moe_dropout_bwd.argtypes = [dp] + [vp] * 4
    lib.switch_moe_balance_workspace_bytes.argtypes = [bp, szp]
    lib.switch_moe_balance_fwd.argtypes = [bp] + [vp] * 7 + [ctypes.c_size_t, vp]
    lib.switch_moe_balance_bwd.argtypes = [bp] + [vp] * 4 + [ctypes.c_float, vp, vp]
    for name in EXPORTED_SYMBOLS:
        if name != "switch_moe_status_string":
            getattr(lib, name).restype = ctypes.c_int
    _lib = lib
    return lib


def make_config(T, d_model, d_ff, E, capacity_factor, alpha=0.01, dtype=BF16, capacity_override=0,
                gemm_path=GEMM_DEFAULT, residual=False, groups=1, reroute=False, input_jitter=False, geglu=False, top2=False, expert_dropout=None, reroute_stages=1) -> SwitchMoeConfig:
    cfg = SwitchMoeConfig()
    cfg.T, cfg.d_model, cfg.d_ff, cfg.E = int(T), int(d_model), int(d_ff), int(E)
    cfg.capacity_factor, cfg.alpha = float(capacity_factor), float(alpha)
    cfg.capacity_override, cfg.dtype, cfg.gemm_path = int(capacity_override), int(dtype), int(gemm_path)
    cfg.flags = ((FLAG_RESIDUAL if residual else 0) | (FLAG_REROUTE if reroute else 0)
                 | (FLAG_INPUT_JITTER if input_jitter else 0) | (FLAG_GEGLU if geglu else 0)
                 | (FLAG_TOP2 if top2 else 0) | (FLAG_EXPERT_DROPOUT if expert_dropout is not None else 0))
    cfg.expert_dropout = float(expert_dropout or 0.0)              # set cfg.expert_keep to the device pointer of the mask     # set cfg.router_jitter to the device pointer of u
    cfg.groups = int(groups)
    cfg.reroute_stages = int(reroute_stages) if reroute else 0
    return cfg


def set_stage_events(cfg: SwitchMoeConfig, events) -> None:
    """Attach STAGE_EVENTS recorded-once torch.cuda.Event objects (enable_timing=True) for per-stage timing, or None."""
    if events is None:
        cfg.stage_events = None
        cfg._stage_event_handles = None
        return
    assert len(events) == STAGE_EVENTS
    handles = (ctypes.c_void_p * STAGE_EVENTS)(*[ev.cuda_event for ev in events])
    cfg._stage_event_handles = handles                      # keep the array alive as long as the config
    cfg.stage_events = ctypes.cast(handles, ctypes.POINTER(ctypes.c_void_p))


def status_string(status: int) -> str:
    return load_library().switch_moe_status_string(int(status)).decode()


def _check(status: int, where: str) -> None:
    if status != OK:
        raise SwitchMoeError(status, where)


def _ptr(t) -> int | None:
    if t is None or isinstance(t, int):
        return t
    return t.data_ptr()


# The current stream's handle without a Stream object around it (3 us of host time per call).
_raw_stream, _device = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream) -> int | None:
    if stream is None:
        if _raw_stream is not None and _device is not None and torch.cuda.is_initialized():
            return _raw_stream(_device())
        stream = torch.cuda.current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def switch_moe_capacity(cfg: SwitchMoeConfig) -> int:
    out = ctypes.c_int32(0)
    _check(load_library().switch_moe_capacity(ctypes.byref(cfg), ctypes.byref(out)), "switch_moe_capacity")
    return out.value


def switch_moe_workspace_bytes(cfg: SwitchMoeConfig) -> int:
    out = ctypes.c_size_t(0)
    _check(load_library().switch_moe_workspace_bytes(ctypes.byref(cfg), ctypes.byref(out)),
           "switch_moe_workspace_bytes")
    return out.value


def allocate_workspace(cfg: SwitchMoeConfig, device="cuda") -> torch.Tensor:
    """A 1024-byte aligned uint8 device tensor of switch_moe_workspace_bytes(cfg) bytes (torch owns the memory)."""
    n = switch_moe_workspace_bytes(cfg)
    raw = torch.empty(n + 1024, dtype=torch.uint8, device=device)
    off = (-raw.data_ptr()) % 1024
    return raw[off:off + n]


_REGION_DTYPES = {
    WS_STATUS: torch.int32, WS_EXPERT_INDEX: torch.int32, WS_GATE: torch.float32, WS_SLOT: torch.int32,
    WS_TOKEN_OF_SLOT: torch.int32, WS_COUNT: torch.int32, WS_KEPT: torch.int32, WS_PSUM: torch.float32,
    WS_PROBS: torch.float32, WS_DGATE: torch.float32, WS_DLOGITS: torch.float32, WS_EXPERT_PROC: torch.int32,
    WS_SECOND_CHOICE: torch.int32,
}


def switch_moe_workspace_view(cfg: SwitchMoeConfig, workspace: torch.Tensor, region: int) -> torch.Tensor:
    """A typed 1-D tensor aliasing one region of the workspace (no copy)."""
    ptr, nbytes = ctypes.c_void_p(0), ctypes.c_size_t(0)
    _check(load_library().switch_moe_workspace_view(ctypes.byref(cfg), workspace.data_ptr(), int(region),
                                                    ctypes.byref(ptr), ctypes.byref(nbytes)),
           "switch_moe_workspace_view")
    off = ptr.value - workspace.data_ptr()
    raw = workspace[off:off + nbytes.value]
    dt = _REGION_DTYPES.get(region, torch.bfloat16 if cfg.dtype == BF16 else torch.float32)
    return raw.view(dt)


def switch_moe_fwd(cfg, x, W_r, router_bias, W_in, W_out, y, aux_loss, workspace, stream=None) -> None:
    _check(load_library().switch_moe_fwd(ctypes.byref(cfg), _ptr(x), _ptr(W_r), _ptr(router_bias), _ptr(W_in),
                                         _ptr(W_out), _ptr(y), _ptr(aux_loss), _ptr(workspace), workspace.numel(),
                                         _stream(stream)), "switch_moe_fwd")


def switch_moe_bwd(cfg, dy, d_aux, x, W_r, W_in, W_out, y, workspace, dx, dW_r, dW_in, dW_out, stream=None) -> None:
    _check(load_library().switch_moe_bwd(ctypes.byref(cfg), _ptr(dy), float(d_aux), _ptr(x), _ptr(W_r), _ptr(W_in),
                                         _ptr(W_out), _ptr(y), _ptr(workspace), workspace.numel(), _ptr(dx),
                                         _ptr(dW_r), _ptr(dW_in), _ptr(dW_out), _stream(stream)), "switch_moe_bwd")


def switch_moe_router_fwd(cfg, x, W_r, router_bias, workspace, stream=None) -> None:
    _check(load_library().switch_moe_router_fwd(ctypes.byref(cfg), _ptr(x), _ptr(W_r), _ptr(router_bias),
                                                _ptr(workspace), workspace.numel(), _stream(stream)),
           "switch_moe_router_fwd")


def switch_moe_dispatch_plan(cfg, expert_index, aux_loss, workspace, stream=None) -> None:
    _check(load_library().switch_moe_dispatch_plan(ctypes.byref(cfg), _ptr(expert_index), _ptr(aux_loss),
                                                   _ptr(workspace), workspace.numel(), _stream(stream)),
           "switch_moe_dispatch_plan")


def switch_moe_dispatch_plan_static(cfg, expert_index, count, kept, slot, token_of_slot, stream=None) -> None:
    """Dispatch plan without a workspace and without any allocation (scratch is a static array inside the library);
    for callers that cannot call cudaMalloc.  Outputs go to the four caller-owned int32 tensors."""
    _check(load_library().switch_moe_dispatch_plan_static(ctypes.byref(cfg), _ptr(expert_index), _ptr(count),
                                                          _ptr(kept), _ptr(slot), _ptr(token_of_slot),
                                                          _stream(stream)), "switch_moe_dispatch_plan_static")


def switch_moe_router_bwd(cfg, x, W_r, dgate, d_aux, workspace, dx_router, dW_r, stream=None) -> None:
    _check(load_library().switch_moe_router_bwd(ctypes.byref(cfg), _ptr(x), _ptr(W_r), _ptr(dgate), float(d_aux),
                                                _ptr(workspace), workspace.numel(), _ptr(dx_router), _ptr(dW_r),
                                                _stream(stream)), "switch_moe_router_bwd")


def switch_moe_step_host(cfg, x_host, dy_host, d_aux, W_r, router_bias, W_in, W_out, x_dev, dy_dev, y_dev, dx_dev,
                         aux_dev, dW_r, dW_in, dW_out, y_host, dx_host, aux_host, workspace, stream=None,
                         h2d_stream=None, d2h_stream=None) -> None:
    _check(load_library().switch_moe_step_host(
        ctypes.byref(cfg), _ptr(x_host), _ptr(dy_host), float(d_aux), _ptr(W_r), _ptr(router_bias), _ptr(W_in),
        _ptr(W_out), _ptr(x_dev), _ptr(dy_dev), _ptr(y_dev), _ptr(dx_dev), _ptr(aux_dev), _ptr(dW_r), _ptr(dW_in),
        _ptr(dW_out), _ptr(y_host), _ptr(dx_host), _ptr(aux_host), _ptr(workspace), workspace.numel(),
        _stream(stream), None if h2d_stream is None else _stream(h2d_stream),
        None if d2h_stream is None else _stream(d2h_stream)), "switch_moe_step_host")


def switch_moe_step_host_enqueue(cfg, x_host, dy_host, d_aux, W_r, router_bias, W_in, W_out, x_dev, dy_dev, y_dev, dx_dev,
                                 aux_dev, dW_r, dW_in, dW_out, y_host, dx_host, aux_host, workspace, stream, h2d_stream,
                                 d2h_stream, slot_free_event, step_done_event) -> None:
    """Non-blocking step: `slot_free_event` / `step_done_event` are torch.cuda.Event objects (the first may be None).
    torch creates the CUDA event behind an Event object on its first record(), so `step_done_event` is recorded once
    on `d2h_stream` here before its handle is passed down (the library records it again after the last download)."""
    if not step_done_event.cuda_event:
        step_done_event.record(d2h_stream)
    _check(load_library().switch_moe_step_host_enqueue(
        ctypes.byref(cfg), _ptr(x_host), _ptr(dy_host), float(d_aux), _ptr(W_r), _ptr(router_bias), _ptr(W_in),
        _ptr(W_out), _ptr(x_dev), _ptr(dy_dev), _ptr(y_dev), _ptr(dx_dev), _ptr(aux_dev), _ptr(dW_r), _ptr(dW_in),
        _ptr(dW_out), _ptr(y_host), _ptr(dx_host), _ptr(aux_host), _ptr(workspace), workspace.numel(),
        _stream(stream), _stream(h2d_stream), _stream(d2h_stream),
        None if slot_free_event is None else ctypes.c_void_p(slot_free_event.cuda_event),
        ctypes.c_void_p(step_done_event.cuda_event)), "switch_moe_step_host_enqueue")


def switch_moe_check_device_status(cfg, workspace, stream=None) -> list:
    """Synchronises the stream; raises SwitchMoeError on a device-side timeout, returns the raw status words."""
    info = (ctypes.c_int32 * 16)()
    rc = load_library().switch_moe_check_device_status(ctypes.byref(cfg), _ptr(workspace), info, _stream(stream))
    if rc != OK:
        raise SwitchMoeError(rc, f"switch_moe_check_device_status info={list(info)}")
    return list(info)


def switch_moe_launches_per_step(cfg) -> int:
    out = ctypes.c_int32(0)
    _check(load_library().switch_moe_launches_per_step(ctypes.byref(cfg), ctypes.byref(out)),
           "switch_moe_launches_per_step")
    return out.value


def switch_moe_stage_launches(cfg) -> dict:
    """Kernel launches per stage, keyed by STAGE_NAMES."""
    out = (ctypes.c_int32 * (STAGE_EVENTS - 1))()
    _check(load_library().switch_moe_stage_launches(ctypes.byref(cfg), out), "switch_moe_stage_launches")
    return {name: int(out[i]) for i, name in enumerate(STAGE_NAMES) if name is not None}


# ------------------------------------------------------------------ operators around the layer (switch_moe.h, second part)
# These calls state rows and distances in their configs; a tensor that does not fit them is refused here, before its
# pointer goes down.  (An int, taken as a device address, is the caller's word.)

def make_linear_config(M, K, N, dtype=BF16, activation=ACT_NONE, dropout=0.0, site=0, ldx=0, ldw=0, ldy=0) -> LinearConfig:
    """y = residual + dropout(activation(x W + bias)), x [M, K], W [K, N]; ld..: elements between rows, 0: dense."""
    return LinearConfig(int(M), int(K), int(N), int(dtype), int(activation), int(site), float(dropout), int(ldx), int(ldw),
                        int(ldy))


def make_dropout_config(rows, cols, rate, dtype=BF16, site=0, ld=0) -> DropoutConfig:
    return DropoutConfig(int(rows), int(cols), int(ld), int(dtype), int(site), float(rate))


def make_balance_config(T, E, k=1, groups=1, alpha=0.01, dtype=F32, ld=0) -> BalanceConfig:
    return BalanceConfig(int(T), int(E), int(k), int(groups), int(dtype), int(ld), float(alpha))


_TORCH_TYPES = {BF16: torch.bfloat16, F32: torch.float32}
_RNG_TYPES = (torch.int64, torch.uint64)
_MASK_TYPES = (torch.uint8, torch.bool)
_FLOAT, _INT = (torch.float32,), (torch.int32,)


def _refuse(where: str, name: str, why: str):
    raise SwitchMoeError(INVALID_ARGUMENT, f"{where}: {name} {why}")


# A call's host time is most of a small call's time, so a check that passes is a few attribute reads (0.5 us a tensor); what
# did not fit is worked out only to be reported.
def _matrix(where, dev, name, t, dtype, rows, cols, ld):
    """Pointer of a [rows, cols] tensor with `ld` elements between rows (0: cols), or of None."""
    if t is None or t.__class__ is int:
        return t
    if t.dtype is dtype and t.shape == (rows, cols) and t.get_device() == dev:
        s = t.stride()
        if (s[0] == (ld or cols) or rows <= 1) and (s[1] == 1 or cols == 1):
            return t.data_ptr()
    if t.dtype is not dtype:
        _refuse(where, name, f"is {t.dtype}, not {dtype}")
    if t.shape != (rows, cols):
        _refuse(where, name, f"is {tuple(t.shape)}, not {(rows, cols)}")
    _check_device(where, name, t)
    _refuse(where, name, f"has strides {t.stride()}, not {(ld or cols, 1)}")


def _vector(where, dev, name, t, dtypes, n):
    """Pointer of a contiguous tensor of n elements, or of None."""
    if t is None or t.__class__ is int:
        return t
    if t.dtype in dtypes and t.numel() == n and t.is_contiguous() and t.get_device() == dev:
        return t.data_ptr()
    if t.dtype not in dtypes:
        _refuse(where, name, f"is {t.dtype}")
    if t.numel() != n or not t.is_contiguous():
        _refuse(where, name, f"is {tuple(t.shape)} with strides {t.stride()}, not {n} contiguous elements")
    _check_device(where, name, t)


def _workspace_args(where, dev, t):
    if t is None:
        return None, 0
    if t.is_contiguous() and t.get_device() == dev:
        return t.data_ptr(), t.nbytes
    _check_device(where, "workspace", t)
    _refuse(where, "workspace", "is not contiguous")


def _current_device() -> int:
    if _device is None:
        return torch.cuda.current_device() if torch.cuda.is_available() else -2
    try:
        return _device()
    except RuntimeError:                                    # no driver: no tensor is on a GPU
        return -2


def _check_device(where, name, t):
    if not t.is_cuda:
        _refuse(where, name, "is not on a GPU")
    if t.get_device() != _current_device():
        _refuse(where, name, "is not on the current device")


def switch_moe_linear_workspace_bytes(cfg: LinearConfig, backward=False) -> int:
    out = ctypes.c_size_t(0)
    _check(load_library().switch_moe_linear_workspace_bytes(ctypes.byref(cfg), int(backward), ctypes.byref(out)),
           "switch_moe_linear_workspace_bytes")
    return out.value


def switch_moe_balance_workspace_bytes(cfg: BalanceConfig) -> int:
    out = ctypes.c_size_t(0)
    _check(load_library().switch_moe_balance_workspace_bytes(ctypes.byref(cfg), ctypes.byref(out)),
           "switch_moe_balance_workspace_bytes")
    return out.value


def _aligned_bytes(n: int, device) -> torch.Tensor:
    raw = torch.empty(n + 1024, dtype=torch.uint8, device=device)
    off = (-raw.data_ptr()) % 1024
    return raw[off:off + n]


def allocate_linear_workspace(cfg: LinearConfig, backward=False, device="cuda") -> torch.Tensor:
    return _aligned_bytes(switch_moe_linear_workspace_bytes(cfg, backward), device)


def allocate_balance_workspace(cfg: BalanceConfig, device="cuda") -> torch.Tensor:
    return _aligned_bytes(switch_moe_balance_workspace_bytes(cfg), device)


def switch_moe_linear_fwd(cfg, x, W, bias, residual, rng, y, pre, workspace, stream=None) -> None:
    """x [M, K], W [K, N], bias float32 [N] or None, residual [M, N] or None, rng int64 [2] {key, offset} (None without
    dropout); writes y [M, N] and, unless it is None, pre [M, N]."""
    f, dev, M, K, N, ldy, dt = "switch_moe_linear_fwd", _current_device(), cfg.M, cfg.K, cfg.N, cfg.ldy, _TORCH_TYPES.get(cfg.dtype)
    _check((_lib or load_library()).switch_moe_linear_fwd(
        cfg, _matrix(f, dev, "x", x, dt, M, K, cfg.ldx), _matrix(f, dev, "W", W, dt, K, N, cfg.ldw), _vector(f, dev, "bias", bias, _FLOAT, N),
        _matrix(f, dev, "residual", residual, dt, M, N, ldy), _vector(f, dev, "rng", rng, _RNG_TYPES, 2), _matrix(f, dev, "y", y, dt, M, N, ldy),
        _matrix(f, dev, "pre", pre, dt, M, N, ldy), *_workspace_args(f, dev, workspace), _stream(stream)), f)


def switch_moe_linear_bwd(cfg, dy, x, W, pre, rng, workspace, dx, dW, dbias, stream=None) -> None:
    """Writes dx [M, K], dW [K, N], dbias float32 [N]; each may be None.  The residual's gradient is dy."""
    f, dev, M, K, N, ldx, ldw, ldy = "switch_moe_linear_bwd", _current_device(), cfg.M, cfg.K, cfg.N, cfg.ldx, cfg.ldw, cfg.ldy
    dt = _TORCH_TYPES.get(cfg.dtype)
    _check((_lib or load_library()).switch_moe_linear_bwd(
        cfg, _matrix(f, dev, "dy", dy, dt, M, N, ldy), _matrix(f, dev, "x", x, dt, M, K, ldx), _matrix(f, dev, "W", W, dt, K, N, ldw),
        _matrix(f, dev, "pre", pre, dt, M, N, ldy), _vector(f, dev, "rng", rng, _RNG_TYPES, 2), *_workspace_args(f, dev, workspace),
        _matrix(f, dev, "dx", dx, dt, M, K, ldx), _matrix(f, dev, "dW", dW, dt, K, N, ldw), _vector(f, dev, "dbias", dbias, _FLOAT, N),
        _stream(stream)), f)


def switch_moe_linear_check_device_status(cfg, workspace, stream=None) -> list:
    """Synchronises the stream; raises SwitchMoeError on a device-side timeout, returns the raw status words."""
    info = (ctypes.c_int32 * 16)()
    rc = load_library().switch_moe_linear_check_device_status(ctypes.byref(cfg), _ptr(workspace), info, _stream(stream))
    if rc != OK:
        raise SwitchMoeError(rc, f"switch_moe_linear_check_device_status info={list(info)}")
    return list(info)


def switch_moe_dropout_fwd(cfg, x, residual, rng, y, stream=None) -> None:
    """y = residual + dropout(x); residual may be None, y may be x or residual."""
    f, dev, rows, cols, ld, dt = "switch_moe_dropout_fwd", _current_device(), cfg.rows, cfg.cols, cfg.ld, _TORCH_TYPES.get(cfg.dtype)
    _check((_lib or load_library()).switch_moe_dropout_fwd(
        cfg, _matrix(f, dev, "x", x, dt, rows, cols, ld), _matrix(f, dev, "residual", residual, dt, rows, cols, ld),
        _vector(f, dev, "rng", rng, _RNG_TYPES, 2), _matrix(f, dev, "y", y, dt, rows, cols, ld), _stream(stream)), f)


def switch_moe_dropout_bwd(cfg, dy, rng, dx, stream=None) -> None:
    """dx = dropout(dy) with the mask of the forward call; dx may be dy."""
    f, dev, rows, cols, ld, dt = "switch_moe_dropout_bwd", _current_device(), cfg.rows, cfg.cols, cfg.ld, _TORCH_TYPES.get(cfg.dtype)
    _check((_lib or load_library()).switch_moe_dropout_bwd(
        cfg, _matrix(f, dev, "dy", dy, dt, rows, cols, ld), _vector(f, dev, "rng", rng, _RNG_TYPES, 2),
        _matrix(f, dev, "dx", dx, dt, rows, cols, ld), _stream(stream)), f)


def switch_moe_balance_fwd(cfg, logits, expert_index, token_mask, loss, counts, tokens, workspace, stream=None) -> None:
    """logits [T, E]; expert_index int32 [T, k] or None (the k largest logits); token_mask uint8 or bool [T] or None; writes
    loss float32 [1], counts int32 [groups, E], tokens int32 [groups]."""
    f, dev, T, E, G = "switch_moe_balance_fwd", _current_device(), cfg.T, cfg.E, cfg.groups or 1
    _check((_lib or load_library()).switch_moe_balance_fwd(
        cfg, _matrix(f, dev, "logits", logits, _TORCH_TYPES.get(cfg.dtype), T, E, cfg.ld),
        _vector(f, dev, "expert_index", expert_index, _INT, T * cfg.k), _vector(f, dev, "token_mask", token_mask, _MASK_TYPES, T),
        _vector(f, dev, "loss", loss, _FLOAT, 1), _vector(f, dev, "counts", counts, _INT, G * E), _vector(f, dev, "tokens", tokens, _INT, G),
        *_workspace_args(f, dev, workspace), _stream(stream)), f)


def switch_moe_balance_bwd(cfg, logits, token_mask, counts, tokens, d_loss, dlogits, stream=None) -> None:
    """dlogits [T, E] from the counts and tokens of the forward call; dlogits may be logits."""
    f, dev, T, E, G, ld, dt = "switch_moe_balance_bwd", _current_device(), cfg.T, cfg.E, cfg.groups or 1, cfg.ld, _TORCH_TYPES.get(cfg.dtype)
    _check((_lib or load_library()).switch_moe_balance_bwd(
        cfg, _matrix(f, dev, "logits", logits, dt, T, E, ld), _vector(f, dev, "token_mask", token_mask, _MASK_TYPES, T),
        _vector(f, dev, "counts", counts, _INT, G * E), _vector(f, dev, "tokens", tokens, _INT, G), float(d_loss),
        _matrix(f, dev, "dlogits", dlogits, dt, T, E, ld), _stream(stream)), f)
