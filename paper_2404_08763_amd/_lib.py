"""ctypes binding of libcats (the C ABI declared in include/cats.h).

Argument marshalling only: every function passes device pointers of torch
tensors and the current HIP stream to the library, which does all the work
in its own kernels.  torch supplies device memory and streams.  There is no
fallback: if libcats.so is missing the import fails.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass
from typing import Callable, Optional

# torch is imported first so that libcats binds to the HIP runtime torch
# already loaded (both carry the soname libamdhip64.so.7); loading libcats
# first would pull in a second runtime.
import torch

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libcats.so")

CATS_F32 = 0
CATS_BF16 = 1
CATS_SCALE_F32 = 0
CATS_SCALE_E8M0 = 1
FP8_BLOCK = 128  # columns (and, for weights, rows) that share a scale
# size of the fixed scratch array behind cats_mlp_forward_noalloc
NOALLOC_SCRATCH_BYTES = 32 << 20
STATUS_NAMES = {
    0: "CATS_OK", 1: "CATS_ERR_NULL", 2: "CATS_ERR_SHAPE", 3: "CATS_ERR_RANGE",
    4: "CATS_ERR_DTYPE", 5: "CATS_ERR_ALIGN", 6: "CATS_ERR_WORKSPACE", 7: "CATS_ERR_HIP",
    8: "CATS_ERR_UNIMPLEMENTED",
}


class CatsError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {message}")
        self.status = status


class _Layer(ctypes.Structure):
    _fields_ = [("d", ctypes.c_int32), ("m", ctypes.c_int32), ("wdtype", ctypes.c_int32),
                ("w_gate_t", ctypes.c_void_p), ("w_up_t", ctypes.c_void_p),
                ("w_down", ctypes.c_void_p)]


class _Aux(ctypes.Structure):
    _fields_ = [("active_idx", ctypes.c_void_p), ("active_cnt", ctypes.c_void_p),
                ("active_v", ctypes.c_void_p), ("active_h", ctypes.c_void_p)]


class _KvCache(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("pages", ctypes.c_int32), ("page", ctypes.c_int32),
                ("heads", ctypes.c_int32), ("d", ctypes.c_int32)]


_vp = ctypes.c_void_p
_i32 = ctypes.c_int32
_i64 = ctypes.c_int64
_sz = ctypes.c_size_t
_f32 = ctypes.c_float
_f64 = ctypes.c_double

_SIGNATURES = {
    "cats_version": ([], _i32),
    "cats_status_string": ([_i32], ctypes.c_char_p),
    "cats_last_error": ([], ctypes.c_char_p),
    "cats_workspace_bytes": ([_i32, _i32, _i32, _i64], _sz),
    "cats_pack_weights": ([_vp, _vp, _i32, _i32, _i32, _vp], _i32),
    "cats_calib_activations": ([ctypes.POINTER(_Layer), _vp, _i32, _vp, _vp], _i32),
    "cats_threshold_from_acts": ([_vp, _i64, _f64, _vp, _sz, _vp, ctypes.POINTER(_f32)], _i32),
    "cats_calibrate_threshold": ([ctypes.POINTER(_Layer), _vp, _i32, _f64, _vp, _sz, _vp,
                                  ctypes.POINTER(_f32)], _i32),
    "cats_mlp_forward": ([ctypes.POINTER(_Layer), _vp, _i32, _f32, _vp, _vp, ctypes.POINTER(_Aux),
                          _vp, _sz, _vp], _i32),
    "cats_mlp_forward_noalloc": ([ctypes.POINTER(_Layer), _vp, _i32, _f32, _vp, _vp, ctypes.POINTER(_Aux), _vp],
                                 _i32),
    "cats_mlp_dense": ([ctypes.POINTER(_Layer), _vp, _i32, _vp, _vp, _vp, _sz, _vp], _i32),
    "cats_stack_forward": ([ctypes.POINTER(_Layer), _i32, ctypes.POINTER(_f32), _vp, _i32, _f32, _vp,
                            _vp, ctypes.POINTER(_Aux), _vp, _sz, _vp], _i32),
    "cats_calibrate_stack_workspace_bytes": ([_i32, _i32, _i32], _sz),
    "cats_calibrate_stack": ([ctypes.POINTER(_Layer), _i32, _vp, _i32, _f64, _f32, _vp, _sz, _vp,
                              ctypes.POINTER(_f32)], _i32),
    "cats_sparse_input_workspace_bytes": ([_i32, _i32, _i32], _sz),
    "cats_sparse_input_gemv": ([_vp, _i32, _i32, _i32, _vp, _i32, _f32, _vp, _vp, ctypes.POINTER(_Aux), _vp,
                                _sz, _vp], _i32),
    "cats_topk_workspace_bytes": ([_i32, _i32, _i32], _sz),
    "cats_mlp_forward_topk": ([ctypes.POINTER(_Layer), _vp, _i32, _f64, _vp, _vp, ctypes.POINTER(_Aux), _vp, _sz,
                               _vp, _vp], _i32),
    "cats_unfused_workspace_bytes": ([_i32, _i32, _i32], _sz),
    "cats_mlp_forward_unfused": ([ctypes.POINTER(_Layer), _vp, _i32, _f32, _i32, _vp, _vp, _vp, _sz, _vp], _i32),
    "cats_rmsnorm": ([_vp, _vp, _i32, _i32, _f32, _vp], _i32),
    "cats_fp8_ld": ([_i32], _i32),
    "cats_quantize_fp8": ([_vp, _i32, _i32, _i32, _i32, _i32, _vp, _vp, _vp], _i32),
    "cats_rmsnorm_fp8": ([_vp, _i32, _vp, _vp, _i32, _i32, _f32, _i32, _vp, _vp, _vp, _vp], _i32),
    "cats_silu_mul_fp8": ([_vp, _i32, _i32, _i32, _f32, _i32, _vp, _vp, _vp], _i32),
    "cats_linear_fp8_workspace_bytes": ([_i32, _i32, _i32], _sz),
    "cats_linear_fp8": ([_vp, _vp, _i32, _vp, _vp, _i32, _i32, _i32, _vp, _vp, _i32, _vp, _sz, _vp], _i32),
    "cats_qk_norm_rope": ([_vp, _i32, _i64, _i32, _i32, _i32, _i32, _i32, _vp, _vp, _f32, _vp, _vp, _i32, _i32, _vp,
                           _vp, _i32, _vp], _i32),
    "cats_kv_cache_bytes": ([_i32, _i32, _i32, _i32], _sz),
    "cats_kv_write": ([ctypes.POINTER(_KvCache), _vp, _i64, _vp, _i64, _i32, _vp, _i32, _vp], _i32),
    "cats_kv_read": ([ctypes.POINTER(_KvCache), _vp, _i32, _vp, _vp, _i32, _vp], _i32),
    "cats_kv_attention_workspace_bytes": ([_i32, _i32, _i32, _i32, _i32], _sz),
    "cats_kv_attention": ([_vp, _i32, _i32, _i32, ctypes.POINTER(_KvCache), _vp, _i32, _vp, _vp, _i32, _f32, _i32,
                           _vp, _vp, _sz, _vp], _i32),
    "cats_stream_read": ([_vp, _sz, _i32, _i32, _i32, _vp, _vp], _i32),
    "cats_timer_enable": ([_i32], _i32),
    "cats_timer_reset": ([], _i32),
    "cats_timer_count": ([], _i32),
    "cats_timer_get": ([_i32, ctypes.POINTER(ctypes.c_char_p), ctypes.POINTER(_i64),
                        ctypes.POINTER(_f64)], _i32),
}

_lib: Optional[ctypes.CDLL] = None


def lib_path() -> str:
    return _LIB_PATH


def raw() -> ctypes.CDLL:
    """The loaded libcats handle (signatures set).  Raises if not built."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise ImportError(f"libcats.so is not built ({_LIB_PATH}); run "
                              "`python -m paper_2404_08763_amd.build` first")
        L = ctypes.CDLL(_LIB_PATH, mode=ctypes.RTLD_GLOBAL)
        for name, (args, res) in _SIGNATURES.items():
            fn = getattr(L, name)
            fn.argtypes = args
            fn.restype = res
        _lib = L
    return _lib


def _check(status: int) -> None:
    if status != 0:
        msg = raw().cats_last_error().decode(errors="replace")
        raise CatsError(status, msg)


def _stream_of_torch() -> Callable[[], int]:
    """What returns the current stream's handle: torch's own record of it,
    without a Stream object around it (2.9 us of a call's 11), or torch's public
    call where this torch does not have those two functions."""
    raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    device = getattr(torch._C, "_cuda_getDevice", None)
    if raw_stream is None or device is None:
        return lambda: torch.cuda.current_stream().cuda_stream
    return lambda: raw_stream(device())


_stream = _stream_of_torch()
_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    # (an address or None, which the void* parameters take as they are)
    return None if t is None else t.data_ptr()


def _dev(t: torch.Tensor, name: str, dtype=None):
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")


def _wdtype(dt: torch.dtype) -> int:
    if dt == torch.bfloat16:
        return CATS_BF16
    if dt == torch.float32:
        return CATS_F32
    raise ValueError(f"unsupported weight dtype {dt}")


@dataclass
class Layer:
    """One gated-MLP block in neuron-major layout (all [m, d] device tensors)."""
    w_gate_t: torch.Tensor
    w_up_t: torch.Tensor
    w_down: torch.Tensor

    def __post_init__(self):
        m, d = self.w_gate_t.shape
        for n, w in (("w_gate_t", self.w_gate_t), ("w_up_t", self.w_up_t), ("w_down", self.w_down)):
            _dev(w, n, self.w_gate_t.dtype)
            if tuple(w.shape) != (m, d):
                raise ValueError(f"{n} has shape {tuple(w.shape)}, expected {(m, d)}")
        self._c = _Layer(d, m, _wdtype(self.w_gate_t.dtype), self.w_gate_t.data_ptr(),
                         self.w_up_t.data_ptr(), self.w_down.data_ptr())
        self._ref = ctypes.byref(self._c)

    @property
    def d(self) -> int:
        return int(self.w_gate_t.shape[1])

    @property
    def m(self) -> int:
        return int(self.w_gate_t.shape[0])

    @property
    def c(self):
        return self._ref


def version() -> int:
    return int(raw().cats_version())


def workspace_bytes(d: int, m: int, max_batch: int = 1, max_calib_values: int = 0) -> int:
    return int(raw().cats_workspace_bytes(d, m, max_batch, max_calib_values))


def workspace(d: int, m: int, max_batch: int = 1, max_calib_values: int = 0, device="cuda") -> torch.Tensor:
    """A zero-filled device byte buffer of cats_workspace_bytes(...) bytes."""
    n = workspace_bytes(d, m, max_batch, max_calib_values)
    if n == 0:
        raise ValueError("arguments outside the supported range")
    ws = torch.zeros(n, dtype=torch.uint8, device=device)
    assert ws.data_ptr() % 256 == 0
    return ws


def pack_weights(w: torch.Tensor, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """[rows, cols] -> [cols, rows] transpose on the device (bit-exact)."""
    _dev(w, "w")
    rows, cols = w.shape
    if out is None:
        out = torch.empty((cols, rows), dtype=w.dtype, device=w.device)
    _dev(out, "out", w.dtype)
    _check(raw().cats_pack_weights(_ptr(w), _ptr(out), rows, cols, _wdtype(w.dtype), _stream()))
    return out


def layer_from_math(w_gate: torch.Tensor, w_up: torch.Tensor, w_down: torch.Tensor) -> Layer:
    """Build a Layer from math-layout weights (W_gate, W_up [d, m]; W_down [m, d])."""
    return Layer(pack_weights(w_gate), pack_weights(w_up), w_down.contiguous())


def calib_activations(layer: Layer, x: torch.Tensor, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    N = _rows_of(x, layer.d)
    _numel_is(out, N * layer.m, "out")
    _dev(x, "x", torch.float32)
    if out is None:
        out = torch.empty((N, layer.m), dtype=torch.float32, device=x.device)
    _dev(out, "out", torch.float32)
    _numel_is(out, N * layer.m, "out")
    _check(raw().cats_calib_activations(layer.c, _ptr(x), N, _ptr(out), _stream()))
    return out


def threshold_from_acts(acts: torch.Tensor, sparsity: float, ws: Optional[torch.Tensor] = None) -> float:
    _dev(acts, "acts", torch.float32)
    if ws is None:
        ws = torch.empty(32768, dtype=torch.uint8, device=acts.device)
    t = _f32()
    _check(raw().cats_threshold_from_acts(_ptr(acts), acts.numel(), float(sparsity), _ptr(ws),
                                          ws.numel(), _stream(), ctypes.byref(t)))
    return float(t.value)


def calibrate_threshold(layer: Layer, calib_x: torch.Tensor, sparsity: float,
                        ws: Optional[torch.Tensor] = None) -> float:
    N = _rows_of(calib_x, layer.d, "calib_x")
    _dev(calib_x, "calib_x", torch.float32)
    if ws is None:
        ws = workspace(layer.d, layer.m, 1, N * layer.m, device=calib_x.device)
    t = _f32()
    _check(raw().cats_calibrate_threshold(layer.c, _ptr(calib_x), N, float(sparsity), _ptr(ws),
                                          ws.numel(), _stream(), ctypes.byref(t)))
    return float(t.value)


def _rows(x: torch.Tensor) -> int:
    return 1 if x.dim() == 1 else int(x.shape[0])


def _rows_of(x: torch.Tensor, d: int, name: str = "x") -> int:
    """Rows of a [B, d] (or [d]) activation tensor; raises before any call
    into the library when its width is not the layer's d, since the kernels
    read and write B * d floats through raw pointers."""
    shape = x.shape
    if len(shape) not in (1, 2):
        raise ValueError(f"{name} must be [d] or [B, d], got shape {tuple(shape)}")
    if shape[-1] != d:
        raise ValueError(f"{name} has width {int(shape[-1])}, the layer has d={d}")
    return 1 if len(shape) == 1 else shape[0]


def _numel_is(t: Optional[torch.Tensor], n: int, name: str) -> None:
    if t is not None and t.numel() != n:
        raise ValueError(f"{name} must hold {n} elements, has {t.numel()}")


def _io_checks(x: torch.Tensor, d: int, out: Optional[torch.Tensor], residual: Optional[torch.Tensor],
               n_out: Optional[int] = None) -> int:
    """Validate x, out and residual of a [B, d] -> [B, n_out] call; returns B.
    Shapes are checked first, so a mismatch raises whatever the device."""
    B = _rows_of(x, d)
    n_out = d if n_out is None else n_out
    _numel_is(out, B * n_out, "out")
    _numel_is(residual, B * n_out, "residual")
    _dev(x, "x", torch.float32)
    if out is not None:
        _dev(out, "out", torch.float32)
    if residual is not None:
        _dev(residual, "residual", torch.float32)
    return B


def mlp_forward(layer: Layer, x: torch.Tensor, t: float, residual: Optional[torch.Tensor] = None,
                out: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None,
                aux: bool = False):
    """CATS MLP forward.  Returns y, or (y, aux dict) when aux=True.

    The aux dict holds per row b: idx[b, :cnt[b]] (ascending active neurons),
    v and h (= v * x.W_up[:, j]) aligned with idx, and cnt.
    """
    B = _io_checks(x, layer.d, out, residual)
    if out is None:
        out = torch.empty_like(x)
    if ws is None:
        ws = workspace(layer.d, layer.m, B, device=x.device)
    aux_c = None
    bufs = None
    if aux:
        m = layer.m
        bufs = {
            "idx": torch.empty((B, m), dtype=torch.int32, device=x.device),
            "cnt": torch.empty((B,), dtype=torch.int32, device=x.device),
            "v": torch.empty((B, m), dtype=torch.float32, device=x.device),
            "h": torch.empty((B, m), dtype=torch.float32, device=x.device),
        }
        aux_c = _Aux(bufs["idx"].data_ptr(), bufs["cnt"].data_ptr(), bufs["v"].data_ptr(),
                     bufs["h"].data_ptr())
    _check(raw().cats_mlp_forward(layer.c, _ptr(x), B, float(t), _ptr(residual), _ptr(out),
                                  ctypes.byref(aux_c) if aux_c is not None else None, _ptr(ws),
                                  ws.numel(), _stream()))
    if aux:
        return out, bufs
    return out


CATS_UNFUSED_MASK = 0
CATS_UNFUSED_INDEX = 1
_UNFUSED_MODES = {"mask": CATS_UNFUSED_MASK, "index": CATS_UNFUSED_INDEX}


def mlp_forward_unfused(layer: Layer, x: torch.Tensor, t: float, mode: str = "mask",
                        residual: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                        ws: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The forward in separate gate / up / down kernels; mode "mask" or "index"."""
    B = _io_checks(x, layer.d, out, residual)
    if mode not in _UNFUSED_MODES:
        raise ValueError(f"mode must be one of {sorted(_UNFUSED_MODES)}")
    if out is None:
        out = torch.empty_like(x)
    if ws is None:
        nbytes = int(raw().cats_unfused_workspace_bytes(layer.d, layer.m, B))
        if nbytes == 0:
            raise ValueError("arguments outside the supported range")
        ws = torch.zeros(nbytes, dtype=torch.uint8, device=x.device)
    _check(raw().cats_mlp_forward_unfused(layer.c, _ptr(x), B, float(t), _UNFUSED_MODES[mode], _ptr(residual),
                                          _ptr(out), _ptr(ws), ws.numel(), _stream()))
    return out


def mlp_forward_topk(layer: Layer, x: torch.Tensor, sparsity: float, residual: Optional[torch.Tensor] = None,
                     out: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None, aux: bool = False):
    """Per-token top-k variant.  Returns (y, t [B]) or (y, t, aux dict)."""
    B = _io_checks(x, layer.d, out, residual)
    if out is None:
        out = torch.empty_like(x)
    if ws is None:
        nbytes = int(raw().cats_topk_workspace_bytes(layer.d, layer.m, B))
        if nbytes == 0:
            raise ValueError("arguments outside the supported range")
        ws = torch.zeros(nbytes, dtype=torch.uint8, device=x.device)
    t = torch.empty((B,), dtype=torch.float32, device=x.device)
    aux_c = None
    bufs = None
    if aux:
        m = layer.m
        bufs = {
            "idx": torch.empty((B, m), dtype=torch.int32, device=x.device),
            "cnt": torch.empty((B,), dtype=torch.int32, device=x.device),
            "v": torch.empty((B, m), dtype=torch.float32, device=x.device),
            "h": torch.empty((B, m), dtype=torch.float32, device=x.device),
        }
        aux_c = _Aux(bufs["idx"].data_ptr(), bufs["cnt"].data_ptr(), bufs["v"].data_ptr(), bufs["h"].data_ptr())
    _check(raw().cats_mlp_forward_topk(layer.c, _ptr(x), B, float(sparsity), _ptr(residual), _ptr(out),
                                       ctypes.byref(aux_c) if aux_c is not None else None, _ptr(ws), ws.numel(),
                                       _stream(), _ptr(t)))
    if aux:
        return out, t, bufs
    return out, t


def mlp_dense(layer: Layer, x: torch.Tensor, residual: Optional[torch.Tensor] = None,
              out: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None) -> torch.Tensor:
    B = _io_checks(x, layer.d, out, residual)
    if out is None:
        out = torch.empty_like(x)
    if ws is None:
        ws = workspace(layer.d, layer.m, B, device=x.device)
    _check(raw().cats_mlp_dense(layer.c, _ptr(x), B, _ptr(residual), _ptr(out), _ptr(ws), ws.numel(),
                                _stream()))
    return out


class Stack:
    """L blocks with one d, marshalled once for repeated stack calls.

    t: one threshold per layer, or None for the dense stack."""

    def __init__(self, layers, t=None):
        self.layers = list(layers)
        L = len(self.layers)
        if L == 0:
            raise ValueError("a stack needs at least one layer")
        self.d = self.layers[0].d
        self.max_m = max(l.m for l in self.layers)
        self._arr = (_Layer * L)(*[l._c for l in self.layers])
        self._t = None
        if t is not None:
            if len(t) != L:
                raise ValueError(f"{len(t)} thresholds for {L} layers")
            self._t = (_f32 * L)(*[float(v) for v in t])

    def __len__(self):
        return len(self.layers)


def stack_forward(stack: Stack, x0: torch.Tensor, eps: float = 1e-5, out: Optional[torch.Tensor] = None,
                  ws: Optional[torch.Tensor] = None, keep_all: bool = False, aux: bool = False):
    """x_{l+1} = x_l + MLP_l(RMSNorm(x_l)) over the stack's layers.

    Returns x_L, or a dict with "out", "x_all" [(L+1), B, d] (keep_all) and
    "aux" (a list of per-layer dicts as from mlp_forward, when aux=True)."""
    B = _rows_of(x0, stack.d, "x0")
    _numel_is(out, B * stack.d, "out")
    _dev(x0, "x0", torch.float32)
    L = len(stack)
    if out is None:
        out = torch.empty_like(x0)
    _dev(out, "out", torch.float32)
    if ws is None:
        ws = workspace(stack.d, stack.max_m, B, device=x0.device)
    x_all = torch.empty((L + 1,) + tuple(x0.shape), dtype=torch.float32, device=x0.device) if keep_all else None
    aux_bufs = None
    aux_c = None
    if aux:
        aux_bufs, cs = [], []
        for l in stack.layers:
            m = l.m
            b = {
                "idx": torch.empty((B, m), dtype=torch.int32, device=x0.device),
                "cnt": torch.empty((B,), dtype=torch.int32, device=x0.device),
                "v": torch.empty((B, m), dtype=torch.float32, device=x0.device),
                "h": torch.empty((B, m), dtype=torch.float32, device=x0.device),
            }
            aux_bufs.append(b)
            cs.append(_Aux(b["idx"].data_ptr(), b["cnt"].data_ptr(), b["v"].data_ptr(), b["h"].data_ptr()))
        aux_c = (_Aux * L)(*cs)
    _check(raw().cats_stack_forward(stack._arr, L, stack._t, _ptr(x0), B, float(eps), _ptr(out),
                                    _ptr(x_all), aux_c, _ptr(ws), ws.numel(), _stream()))
    if not keep_all and not aux:
        return out
    return {"out": out, "x_all": x_all, "aux": aux_bufs}


def calibrate_stack(stack: Stack, calib_x: torch.Tensor, sparsity: float, eps: float = 1e-5,
                    ws: Optional[torch.Tensor] = None) -> list:
    """Per-layer thresholds of a stack, the calibration vectors propagated
    densely through the earlier layers (cats_calibrate_stack)."""
    N = _rows_of(calib_x, stack.d, "calib_x")
    _dev(calib_x, "calib_x", torch.float32)
    L = len(stack)
    if ws is None:
        n = int(raw().cats_calibrate_stack_workspace_bytes(stack.d, stack.max_m, N))
        if n == 0:
            raise ValueError("arguments outside the supported range")
        ws = torch.zeros(n, dtype=torch.uint8, device=calib_x.device)
    t = (_f32 * L)()
    _check(raw().cats_calibrate_stack(stack._arr, L, _ptr(calib_x), N, float(sparsity), float(eps),
                                      _ptr(ws), ws.numel(), _stream(), t))
    return [float(v) for v in t]


def sparse_input_workspace(d: int, n: int, max_batch: int = 1, device="cuda") -> torch.Tensor:
    nbytes = int(raw().cats_sparse_input_workspace_bytes(d, n, max_batch))
    if nbytes == 0:
        raise ValueError("arguments outside the supported range")
    return torch.zeros(nbytes, dtype=torch.uint8, device=device)


def sparse_input_gemv(w: torch.Tensor, x: torch.Tensor, t: float, residual: Optional[torch.Tensor] = None,
                      out: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None, aux: bool = False):
    """y = residual + CATS_t(x) W for W [d, n] (channel-major, bf16).

    Returns y, or (y, aux dict) with per row the ascending kept channels
    idx[b, :cnt[b]] and their values v (= h)."""
    if w.dim() != 2:
        raise ValueError(f"w must be [d, n], got shape {tuple(w.shape)}")
    d, n = int(w.shape[0]), int(w.shape[1])
    B = _io_checks(x, d, out, residual, n_out=n)
    _dev(w, "w", torch.bfloat16)
    if out is None:
        out = torch.empty((B, n), dtype=torch.float32, device=x.device)
    if ws is None:
        ws = sparse_input_workspace(d, n, B, device=x.device)
    aux_c = None
    bufs = None
    if aux:
        bufs = {
            "idx": torch.empty((B, d), dtype=torch.int32, device=x.device),
            "cnt": torch.empty((B,), dtype=torch.int32, device=x.device),
            "v": torch.empty((B, d), dtype=torch.float32, device=x.device),
            "h": torch.empty((B, d), dtype=torch.float32, device=x.device),
        }
        aux_c = _Aux(bufs["idx"].data_ptr(), bufs["cnt"].data_ptr(), bufs["v"].data_ptr(), bufs["h"].data_ptr())
    _check(raw().cats_sparse_input_gemv(_ptr(w), d, n, CATS_BF16, _ptr(x), B, float(t), _ptr(residual),
                                        _ptr(out), ctypes.byref(aux_c) if aux_c is not None else None,
                                        _ptr(ws), ws.numel(), _stream()))
    if aux:
        return out, bufs
    return out


def rmsnorm(x: torch.Tensor, eps: float = 1e-5, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    _dev(x, "x", torch.float32)
    if x.dim() not in (1, 2):
        raise ValueError(f"x must be [d] or [B, d], got shape {tuple(x.shape)}")
    if out is None:
        out = torch.empty_like(x)
    _dev(out, "out", torch.float32)
    _numel_is(out, x.numel(), "out")
    B = _rows(x)
    d = int(x.shape[-1])
    _check(raw().cats_rmsnorm(_ptr(x), _ptr(out), B, d, float(eps), _stream()))
    return out


# ---- 8-bit operands ---------------------------------------------------------
# e4m3 values [rows, ld] (ld: the columns rounded up to FP8_BLOCK, zeros behind
# them) with a scale for each 1 (rows of x) or FP8_BLOCK (weights) rows by
# FP8_BLOCK columns, torch.float32 or torch.float8_e8m0fnu (powers of two).

_SCALE_TYPES = {torch.float32: CATS_SCALE_F32, torch.float8_e8m0fnu: CATS_SCALE_E8M0}


def fp8_ld(cols: int) -> int:
    """Columns of the e4m3 array of a matrix of `cols` columns."""
    return (cols + FP8_BLOCK - 1) // FP8_BLOCK * FP8_BLOCK


def _blocks(rows: int) -> int:
    return (rows + FP8_BLOCK - 1) // FP8_BLOCK


def _stype(dt: torch.dtype) -> int:
    st = _SCALE_TYPES.get(dt)
    if st is None:
        raise ValueError(f"scales are torch.float32 or torch.float8_e8m0fnu, not {dt}")
    return st


def _shape_is(t: torch.Tensor, shape: tuple, name: str) -> None:
    if t.shape != shape:
        raise ValueError(f"{name} must be {list(shape)}, has shape {list(t.shape)}")


def _refuse(name: str, t: torch.Tensor, dtype: torch.dtype, device: int) -> None:
    """Raises for a tensor that is not a contiguous one of that type on the
    current device, on whose stream the call runs (the callers' own test of the
    same costs a third of a call for each tensor)."""
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    raise ValueError(f"{name} is on device {t.get_device()}, the current device is {device}")


_E4M3 = torch.float8_e4m3fn


def _fp8_io(x: torch.Tensor, rows: int, cols: int, block_rows: int, scale_dtype: torch.dtype, out):
    """Checks a quantising call's input and returns its q and scale (out's, or
    new ones), the scale's type and the current device."""
    xt = x.dtype
    if xt is not torch.float32 and xt is not torch.bfloat16:
        raise ValueError(f"the input must be torch.float32 or torch.bfloat16, got {xt}")
    ld = (cols + FP8_BLOCK - 1) // FP8_BLOCK * FP8_BLOCK
    qs, ss = (rows, ld), (rows if block_rows == 1 else _blocks(rows), ld // FP8_BLOCK)
    if out is not None:
        q, scale = out
        if q.shape != qs:
            _shape_is(q, qs, "q")
        if scale.shape != ss:
            _shape_is(scale, ss, "scale")
        scale_dtype = scale.dtype
    st = _stype(scale_dtype)
    if not x.is_cuda:
        raise ValueError("the input must be a device tensor")
    if out is None:
        q = torch.empty(qs, dtype=_E4M3, device=x.device)
        scale = torch.empty(ss, dtype=scale_dtype, device=x.device)
    device = _device()
    if x.get_device() != device or not x.is_contiguous():
        _refuse("the input", x, xt, device)
    if q.dtype is not _E4M3 or q.get_device() != device or not q.is_contiguous():
        _refuse("q", q, _E4M3, device)
    if scale.get_device() != device or not scale.is_contiguous():
        _refuse("scale", scale, scale_dtype, device)
    return q, scale, st, device


def _two_dims(x: torch.Tensor, name: str) -> tuple:
    if x.dim() != 2:
        raise ValueError(f"{name} must have two dimensions, got shape {list(x.shape)}")
    return x.shape


def quantize_fp8(x: torch.Tensor, block_rows: int = 1, scale_dtype: torch.dtype = torch.float32, out=None):
    """x [rows, cols] (fp32 or bf16) -> (q [rows, fp8_ld(cols)] e4m3, scale), one
    scale per block_rows x 128 elements: 1 for rows of x, 128 for weights
    [n, k].  out: a (q, scale) pair to write to, whose scale's dtype then counts."""
    rows, cols = _two_dims(x, "x")
    if block_rows not in (1, FP8_BLOCK):
        raise ValueError(f"block_rows must be 1 or {FP8_BLOCK}")
    q, scale, st, _ = _fp8_io(x, rows, cols, block_rows, scale_dtype, out)
    _check(raw().cats_quantize_fp8(x.data_ptr(), _wdtype(x.dtype), rows, cols, block_rows, st, q.data_ptr(),
                                   scale.data_ptr(), _stream()))
    return q, scale


def rmsnorm_fp8(x: torch.Tensor, residual: Optional[torch.Tensor] = None, gain: Optional[torch.Tensor] = None,
                eps: float = 1e-5, scale_dtype: torch.dtype = torch.float32, out=None,
                sum_out: Optional[torch.Tensor] = None):
    """(q, scale) of gain * s / sqrt(mean(s^2) + eps), s = x + residual, x [N, d]
    fp32 or bf16, residual and sum_out [N, d] fp32 (sum_out receives s and may be
    the residual, or x if fp32), gain [d] fp32; a scale per row and 128 columns."""
    N, d = _two_dims(x, "x")
    q, scale, st, device = _fp8_io(x, N, d, 1, scale_dtype, out)
    for name, t, shape in (("residual", residual, (N, d)), ("gain", gain, (d,)), ("sum_out", sum_out, (N, d))):
        if t is not None:
            if t.shape != shape:
                _shape_is(t, shape, name)
            if t.dtype is not torch.float32 or t.get_device() != device or not t.is_contiguous():
                _refuse(name, t, torch.float32, device)
    _check(raw().cats_rmsnorm_fp8(x.data_ptr(), _wdtype(x.dtype), _ptr(residual), _ptr(gain), N, d, eps, st,
                                  _ptr(sum_out), q.data_ptr(), scale.data_ptr(), _stream()))
    return q, scale


def silu_mul_fp8(gate_up: torch.Tensor, t: float = 0.0, scale_dtype: torch.dtype = torch.float32, out=None):
    """(q, scale) of h = v u where |v| >= t, else 0, v = SiLU(g), for gate_up
    [N, 2 m] (a row's gate values, then its up values; fp32 or bf16); a scale
    per row and 128 neurons."""
    N, two_m = _two_dims(gate_up, "gate_up")
    if two_m % 2:
        raise ValueError(f"gate_up must be [N, 2 m], has {two_m} columns")
    m = two_m // 2
    q, scale, st, _ = _fp8_io(gate_up, N, m, 1, scale_dtype, out)
    _check(raw().cats_silu_mul_fp8(gate_up.data_ptr(), _wdtype(gate_up.dtype), N, m, t, st, q.data_ptr(),
                                   scale.data_ptr(), _stream()))
    return q, scale


def linear_fp8_workspace(N: int, n: int, k: int, device="cuda") -> torch.Tensor:
    """Scratch memory for linear_fp8 calls of up to N rows, n outputs and k columns."""
    nbytes = int(raw().cats_linear_fp8_workspace_bytes(N, n, k))
    if nbytes == 0:
        raise ValueError("arguments outside the supported range")
    return torch.empty(nbytes, dtype=torch.uint8, device=device)


def linear_fp8(xq: torch.Tensor, xs: torch.Tensor, wq: torch.Tensor, wscale: torch.Tensor,
               residual: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
               dtype: torch.dtype = torch.float32, ws: Optional[torch.Tensor] = None) -> torch.Tensor:
    """y = residual + x W^T for the rows (xq, xs) and the weight (wq, wscale), both
    as the quantising calls write them: xq [N, ld], wq [n, ld].  y [N, n] is fp32
    or bf16 (`dtype`, or out's), the residual of y's type; out may be the residual.
    Products are exact for fp32 y; for bf16 y of many rows they are cut at 2^-13 of the
    largest of their group of eight columns.
    ws: linear_fp8_workspace's for this or a larger call (None: one for this call)."""
    N, ld = _two_dims(xq, "xq")
    n, ldw = _two_dims(wq, "wq")
    if ld != ldw or ld % FP8_BLOCK:
        raise ValueError(f"xq and wq must have the same width, a multiple of {FP8_BLOCK}: got {ld} and {ldw}")
    nb = ld // FP8_BLOCK
    _shape_is(xs, (N, nb), "xs")
    _shape_is(wscale, (_blocks(n), nb), "wscale")
    sdt = xs.dtype
    st = _stype(sdt)
    if out is not None:
        _shape_is(out, (N, n), "out")
        dtype = out.dtype
    yt = _wdtype(dtype)
    if residual is not None:
        _shape_is(residual, (N, n), "residual")
    if not xq.is_cuda:
        raise ValueError("xq must be a device tensor")
    if out is None:
        out = torch.empty((N, n), dtype=dtype, device=xq.device)
    device = _device()
    for name, t, dt in (("xq", xq, _E4M3), ("xs", xs, sdt), ("wq", wq, _E4M3), ("wscale", wscale, sdt),
                        ("out", out, dtype), ("residual", residual, dtype), ("ws", ws, torch.uint8)):
        if t is not None and (t.dtype is not dt or t.get_device() != device or not t.is_contiguous()):
            _refuse(name, t, dt, device)
    if ws is None:
        ws = linear_fp8_workspace(N, n, ld, device=xq.device)
    _check(raw().cats_linear_fp8(xq.data_ptr(), xs.data_ptr(), N, wq.data_ptr(), wscale.data_ptr(), n, ld, st,
                                 _ptr(residual), out.data_ptr(), yt, ws.data_ptr(), ws.numel(), _stream()))
    return out


# ---- around attention ---------------------------------------------------------
# Norms and rotation of the heads, the cache of keys and values in 4 bits, and
# attention over it.  A cache is a uint8 tensor [pages, heads, page / 16, 17 d]: a
# record of 17 d bytes for 16 tokens of a head (cats.h has its layout).

_KV_RECORD = 17  # bytes of a record for each column


def kv_cache(pages: int, heads: int, d: int, page: int = 64, device="cuda") -> torch.Tensor:
    """Memory for a cache of `pages` pages of `page` tokens (a multiple of 16 up to
    256) of `heads` key heads of d = 64, 128 or 256 columns.  Not cleared: what is
    not written is not used."""
    if not raw().cats_kv_cache_bytes(pages, page, heads, d):
        raise ValueError("arguments outside the supported range")
    return torch.empty((pages, heads, page // 16, _KV_RECORD * d), dtype=torch.uint8, device=device)


def _kv(cache: torch.Tensor, device: int):
    """A cache's C structure, its heads and its columns."""
    if cache.dim() != 4:
        raise ValueError(f"cache must be [pages, heads, page / 16, 17 d], has shape {list(cache.shape)}")
    pages, heads, groups, rec = cache.shape
    if rec % _KV_RECORD:
        raise ValueError(f"cache must be [pages, heads, page / 16, 17 d], has shape {list(cache.shape)}")
    if cache.dtype is not torch.uint8 or cache.get_device() != device or not cache.is_contiguous():
        _refuse("cache", cache, torch.uint8, device)
    d = rec // _KV_RECORD
    return _KvCache(cache.data_ptr(), pages, 16 * groups, heads, d), heads, d


def _on(name: str, t: Optional[torch.Tensor], dtype: torch.dtype, device: int) -> None:
    if t is not None and (t.dtype is not dtype or t.get_device() != device or not t.is_contiguous()):
        _refuse(name, t, dtype, device)


_ROW_TYPES = {torch.float32: CATS_F32, torch.bfloat16: CATS_BF16}


def _row_type(name: str, t: torch.Tensor) -> int:
    dt = _ROW_TYPES.get(t.dtype)
    if dt is None:
        raise ValueError(f"{name} must be torch.float32 or torch.bfloat16, got {t.dtype}")
    return dt


def _pitch(name: str, t: torch.Tensor, device: int) -> int:
    """The pitch of rows [N, cols] or [N, heads, d] whose columns are dense."""
    if t.get_device() != device:
        _refuse(name, t, t.dtype, device)
    strides, shape = t.stride(), t.shape
    if strides[-1] != 1 or (len(shape) == 3 and shape[1] > 1 and strides[1] != shape[2]):
        raise ValueError(f"{name}'s rows must be dense")
    if shape[0] == 1:  # (a single row's stride is no pitch)
        return (shape[1] * (shape[2] if len(shape) == 3 else 1) + 7) // 8 * 8
    return strides[0]


def qk_norm_rope(qkv: torch.Tensor, heads: int, kv_heads: int, d: int, pos: Optional[torch.Tensor] = None,
                 freq: Optional[torch.Tensor] = None, norm: bool = False, gain_q: Optional[torch.Tensor] = None,
                 gain_k: Optional[torch.Tensor] = None, eps: float = 1e-5, interleaved: bool = False,
                 dtype: Optional[torch.dtype] = None, out=None):
    """(q [N, heads, d], k [N, kv_heads, d]) of qkv's rows (fp32 or bf16; a row's
    query heads, then its key heads; what follows is not read; rows may be
    strided): each head RMS-normed with gain_q or gain_k [d] fp32 (`norm`), then the
    first 2 len(freq) columns turned by pos [N] int32 times freq [rot / 2] fp32
    (freq None: none), in pairs (i, i + rot / 2) or, `interleaved`, (2 i, 2 i + 1).
    dtype: of q and k (None: qkv's); out: a (q, k) pair to write to."""
    N, cols = _two_dims(qkv, "qkv")
    if cols < (heads + kv_heads) * d:
        raise ValueError(f"qkv must have {(heads + kv_heads) * d} columns or more, has {cols}")
    xt = _row_type("qkv", qkv)
    if out is None:
        if not qkv.is_cuda:
            raise ValueError("qkv must be a device tensor")
        dtype = qkv.dtype if dtype is None else dtype
        q, k = (torch.empty((N, h, d), dtype=dtype, device=qkv.device) for h in (heads, kv_heads))
    else:
        q, k = out
        if q.shape != (N, heads, d):
            _shape_is(q, (N, heads, d), "q")
        if k.shape != (N, kv_heads, d):
            _shape_is(k, (N, kv_heads, d), "k")
    device = _device()
    ld = _pitch("qkv", qkv, device)
    yt, qt = _row_type("q", q), q.dtype
    if q.get_device() != device or not q.is_contiguous():
        _refuse("q", q, qt, device)
    if k.dtype is not qt or k.get_device() != device or not k.is_contiguous():
        _refuse("k", k, qt, device)
    rot, fp, pp = 0, None, None
    if freq is not None:
        if pos is None:
            raise ValueError("freq needs pos")
        if freq.dim() != 1:
            raise ValueError(f"freq must have one dimension, got shape {list(freq.shape)}")
        half = freq.shape[0]
        if pos.shape != (N,):
            _shape_is(pos, (N,), "pos")
        if freq.dtype is not torch.float32 or freq.get_device() != device or not freq.is_contiguous():
            _refuse("freq", freq, torch.float32, device)
        if pos.dtype is not torch.int32 or pos.get_device() != device or not pos.is_contiguous():
            _refuse("pos", pos, torch.int32, device)
        rot = 2 * half
        if rot:
            fp, pp = freq.data_ptr(), pos.data_ptr()
    if gain_q is not None or gain_k is not None:
        if not norm:
            raise ValueError("gain_q and gain_k need norm=True")
        for name, t in (("gain_q", gain_q), ("gain_k", gain_k)):
            if t is not None:
                _shape_is(t, (d,), name)
                _on(name, t, torch.float32, device)
    _check((_lib or raw()).cats_qk_norm_rope(
        qkv.data_ptr(), xt, ld, N, heads, kv_heads, d, 1 if norm else 0, _ptr(gain_q), _ptr(gain_k), eps, pp, fp, rot,
        1 if interleaved else 0, q.data_ptr(), k.data_ptr(), yt, _stream()))
    return q, k


def _slots_of(slots: torch.Tensor, device: int) -> int:
    if slots.dim() != 1:
        raise ValueError(f"slots must have one dimension, got shape {list(slots.shape)}")
    if slots.dtype is not torch.int32 or slots.get_device() != device or not slots.is_contiguous():
        _refuse("slots", slots, torch.int32, device)
    return slots.shape[0]


def kv_write(cache: torch.Tensor, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor) -> None:
    """Quantises rows of keys and values ([N, heads, d] or [N, heads d] fp32 or bf16,
    each row dense, rows strided as they like) into the cache's slots [N] int32
    (token s % page of page s // page; outside the cache: the row is left out).  The
    slots inside the cache must differ."""
    device = _device()
    c, heads, d = _kv(cache, device)
    N = _slots_of(slots, device)
    whole, flat = (N, heads, d), (N, heads * d)
    ks, vs = k.shape, v.shape
    if ks != whole and ks != flat:
        raise ValueError(f"k must be {list(whole)} or {list(flat)}, has shape {list(ks)}")
    if vs != whole and vs != flat:
        raise ValueError(f"v must be {list(whole)} or {list(flat)}, has shape {list(vs)}")
    if k.dtype is not v.dtype:
        raise ValueError(f"k and v must have one type, got {k.dtype} and {v.dtype}")
    dt = _row_type("k", k)
    ldk, ldv = _pitch("k", k, device), _pitch("v", v, device)
    _check((_lib or raw()).cats_kv_write(ctypes.byref(c), k.data_ptr(), ldk, v.data_ptr(), ldv, dt, slots.data_ptr(), N,
                                         _stream()))


def kv_read(cache: torch.Tensor, slots: torch.Tensor, dtype: torch.dtype = torch.bfloat16, out=None):
    """(k, v) [N, heads, d] of the cache's slots [N] int32, fp32 or bf16, both exact.
    Rows whose slot is outside the cache are left as they are in `out` (without
    `out`: undefined)."""
    device = _device()
    c, heads, d = _kv(cache, device)
    N = _slots_of(slots, device)
    if out is None:
        out = tuple(torch.empty((N, heads, d), dtype=dtype, device=cache.device) for _ in range(2))
    k, v = out
    shape = (N, heads, d)
    if k.shape != shape:
        _shape_is(k, shape, "k")
    if v.shape != shape:
        _shape_is(v, shape, "v")
    dt, kt = _row_type("k", k), k.dtype
    if k.get_device() != device or not k.is_contiguous():
        _refuse("k", k, kt, device)
    if v.dtype is not kt or v.get_device() != device or not v.is_contiguous():
        _refuse("v", v, kt, device)
    _check((_lib or raw()).cats_kv_read(ctypes.byref(c), slots.data_ptr(), N, k.data_ptr(), v.data_ptr(), dt, _stream()))
    return k, v


def kv_attention_workspace(N: int, B: int, heads: int, kv_heads: int, d: int, device="cuda") -> torch.Tensor:
    """Scratch memory for kv_attention calls of up to N rows of B sequences."""
    nbytes = int(raw().cats_kv_attention_workspace_bytes(N, B, heads, kv_heads, d))
    if nbytes == 0:
        raise ValueError("arguments outside the supported range")
    return torch.empty(nbytes, dtype=torch.uint8, device=device)


def kv_attention(q: torch.Tensor, cache: torch.Tensor, table: torch.Tensor, lens: torch.Tensor,
                 q_start: Optional[torch.Tensor] = None, scale: Optional[float] = None, window: int = 0,
                 out: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Causal attention of q [N, heads, d] (fp32 or bf16; out has its type) over the
    cache: table [B, width] int32 has each sequence's pages, lens [B] int32 its
    tokens (the rows' own among them), q_start [B + 1] int32 its rows, which are its
    last ones (None: one row for each sequence).  scale: None is d ** -0.5; window:
    0, or how many tokens a row sees.  Rows that see no key become 0; rows of no
    sequence are left as they are in `out` (without `out`: undefined).
    ws: kv_attention_workspace's for this or a larger call (None: one for this call)."""
    if q.dim() != 3:
        raise ValueError(f"q must be [N, heads, d], got shape {list(q.shape)}")
    device = _device()
    c, kv_heads, d = _kv(cache, device)
    N, heads, dq = q.shape
    if dq != d:
        raise ValueError(f"q's heads have {dq} columns, the cache's {d}")
    B, width = _two_dims(table, "table")
    if lens.shape != (B,):
        _shape_is(lens, (B,), "lens")
    starts = None
    if q_start is not None:
        if q_start.shape != (B + 1,):
            _shape_is(q_start, (B + 1,), "q_start")
        if q_start.dtype is not torch.int32 or q_start.get_device() != device or not q_start.is_contiguous():
            _refuse("q_start", q_start, torch.int32, device)
        starts = q_start.data_ptr()
    elif N != B:
        raise ValueError(f"without q_start q must have a row for each of {B} sequences, has {N}")
    dt, dtype = _row_type("q", q), q.dtype
    if out is None:
        if not q.is_cuda:
            raise ValueError("q must be a device tensor")
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
    else:
        if out.shape != q.shape:
            _shape_is(out, (N, heads, d), "out")
        if out.dtype is not dtype or out.get_device() != device or not out.is_contiguous():
            _refuse("out", out, dtype, device)
    if q.get_device() != device or not q.is_contiguous():
        _refuse("q", q, dtype, device)
    if table.dtype is not torch.int32 or table.get_device() != device or not table.is_contiguous():
        _refuse("table", table, torch.int32, device)
    if lens.dtype is not torch.int32 or lens.get_device() != device or not lens.is_contiguous():
        _refuse("lens", lens, torch.int32, device)
    if ws is None:
        ws = kv_attention_workspace(N, B, heads, kv_heads, d, device=q.device)
    elif ws.dtype is not torch.uint8 or ws.get_device() != device or not ws.is_contiguous():
        _refuse("ws", ws, torch.uint8, device)
    _check((_lib or raw()).cats_kv_attention(
        q.data_ptr(), dt, N, heads, ctypes.byref(c), table.data_ptr(), width, lens.data_ptr(), starts, B,
        d ** -0.5 if scale is None else scale, window, out.data_ptr(), ws.data_ptr(), ws.numel(), _stream()))
    return out


def stream_read(buf: torch.Tensor, blocks: int, inflight: int = 8, runs: bool = False,
                sink: Optional[torch.Tensor] = None) -> None:
    """Enqueue one plain read of a device tensor's bytes (attainable-bandwidth
    probe; time it with timer_* under the name "stream_read")."""
    if not buf.is_cuda or not buf.is_contiguous():
        raise ValueError("buf must be a contiguous device tensor")
    if sink is None:
        sink = torch.empty(blocks, dtype=torch.int32, device=buf.device)
    _check(raw().cats_stream_read(_ptr(buf), buf.numel() * buf.element_size(), int(blocks), int(inflight),
                                  1 if runs else 0, _ptr(sink), _stream()))


def timer_enable(on: bool = True) -> None:
    _check(raw().cats_timer_enable(1 if on else 0))


def timer_reset() -> None:
    _check(raw().cats_timer_reset())


def timer_read() -> dict:
    """{kernel name: (launches, total ms)} for the kernels timed so far."""
    L = raw()
    out = {}
    for i in range(int(L.cats_timer_count())):
        name = ctypes.c_char_p()
        n = _i64()
        ms = _f64()
        _check(L.cats_timer_get(i, ctypes.byref(name), ctypes.byref(n), ctypes.byref(ms)))
        out[name.value.decode()] = (int(n.value), float(ms.value))
    return out
