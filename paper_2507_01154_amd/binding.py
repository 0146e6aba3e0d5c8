"""ctypes binding of libflashdp.so: argument marshalling only.

Every function has the name and the arguments of the C entry point it wraps (see
include/flashdp.h).  Tensors are torch CUDA tensors used as device buffers; nothing is
computed here.  A missing library is an error: there is no fallback path.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence

PKG_DIR = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG_DIR, "libflashdp.so")

BF16, F32, F16 = 0, 1, 2
SCHEDULE_AUTO, SCHEDULE_TWOPASS, SCHEDULE_SCRATCH, SCHEDULE_EXPLICIT, SCHEDULE_OVERLAP, SCHEDULE_GHOST, SCHEDULE_FUSED = 0, 1, 2, 3, 4, 5, 6
ACT_NONE, ACT_RELU, ACT_GELU, ACT_GELU_TANH, ACT_SILU = 0, 1, 2, 3, 4
_ACTIVATIONS = {None: 0, "none": 0, "relu": 1, "gelu": 2, "gelu_tanh": 3, "silu": 4}
FIELD_BIAS, FIELD_NORM = 1, 2
_SCHEDULES = {"auto": 0, "twopass": 1, "scratch": 2, "explicit": 3, "overlap": 4, "ghost": 5, "fused": 6}

OK = 0
INVALID_ARGUMENT, MISALIGNED, UNSUPPORTED_SHAPE, WORKSPACE_TOO_SMALL, NO_DEVICE, HIP_ERROR = -1, -2, -3, -4, -5, -6


class FlashDPError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} ({status})")


class flashdp_layer_t(ctypes.Structure):
    _fields_ = [
        ("X", ctypes.c_void_p), ("dY", ctypes.c_void_p),
        ("d_in", ctypes.c_int64), ("d_out", ctypes.c_int64),
        ("C", ctypes.c_float), ("sigma", ctypes.c_float),
        ("seed", ctypes.c_uint64), ("layer", ctypes.c_uint32),
        ("out_grad", ctypes.c_void_p), ("out_norms", ctypes.c_void_p),
    ]


_lib = None


def lib() -> ctypes.CDLL:
    """The loaded shared library; built by __graft_entry__.build() / build.py beforehand."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(
                f"{LIB_PATH} is missing: build it first (python -m paper_2507_01154_amd.build). "
                "There is no fallback implementation.")
        L = ctypes.CDLL(LIB_PATH)
        vp, i64, f32, u64, u32, sz, ci = (ctypes.c_void_p, ctypes.c_int64, ctypes.c_float, ctypes.c_uint64,
                                          ctypes.c_uint32, ctypes.c_size_t, ctypes.c_int)
        lp = ctypes.POINTER(flashdp_layer_t)
        L.flashdp_linear_dp_grad.argtypes = [vp, vp, i64, i64, i64, i64, f32, f32, u64, vp, vp]
        L.flashdp_linear_dp_grad.restype = ci
        L.flashdp_block_dp_grad.argtypes = [lp, ci, i64, i64, ci, ci, vp, sz, vp]
        L.flashdp_block_dp_grad.restype = ci
        L.flashdp_block_dp_grad_micro.argtypes = [lp, ci, i64, i64, ci, ci, vp, sz, vp, ci, ci]
        L.flashdp_block_dp_grad_micro.restype = ci
        L.flashdp_workspace_bytes.argtypes = [lp, ci, i64, i64, ci, ci]
        L.flashdp_workspace_bytes.restype = sz
        L.flashdp_workspace_bytes_chunked.argtypes = [lp, ci, i64, i64, ci, i64, ci]
        L.flashdp_workspace_bytes_chunked.restype = sz
        L.flashdp_last_chunk.restype = i64
        L.flashdp_linear_dp_grad_static.argtypes = [vp, vp, i64, i64, i64, i64, ci, f32, f32, u64, u32, vp, vp, vp]
        L.flashdp_linear_dp_grad_static.restype = ci
        L.flashdp_static_scratch_bytes.argtypes = []
        L.flashdp_static_scratch_bytes.restype = sz
        L.flashdp_linear_forward.argtypes = [vp, vp, vp, vp, i64, i64, i64, ci, ci, vp, vp, ci, vp]
        L.flashdp_activation_dp_grad.argtypes = [vp, vp, ci, i64, i64, i64, ci, ci, f32, f32, u64, u32, vp, vp, vp, vp, sz, vp, ci, ci]
        L.flashdp_layernorm_forward.argtypes = [vp, vp, vp, i64, i64, ci, f32, vp, vp, vp, vp]
        L.flashdp_layernorm_dp_grad.argtypes = [vp, vp, vp, vp, vp, i64, i64, i64, ci, f32, f32, u64, u32, vp, vp, vp, ci, vp, sz, vp, ci, ci]
        L.flashdp_checkpoint8_pack.argtypes = [vp, i64, i64, ci, vp, vp]
        L.flashdp_checkpoint8_unpack.argtypes = [vp, i64, i64, ci, vp, vp]
        L.flashdp_block_dp_grad_checkpoint8.argtypes = [lp, ci, i64, i64, ci, ci, vp, sz, vp, ci, ci]
        for n in ("flashdp_linear_forward", "flashdp_activation_dp_grad", "flashdp_layernorm_forward", "flashdp_layernorm_dp_grad",
                  "flashdp_checkpoint8_pack", "flashdp_checkpoint8_unpack", "flashdp_block_dp_grad_checkpoint8"):
            getattr(L, n).restype = ci
        L.flashdp_activation_workspace_bytes.argtypes = [i64, i64, i64, ci]
        L.flashdp_layernorm_workspace_bytes.argtypes = [i64, i64, i64, ci, ci]
        L.flashdp_checkpoint8_bytes.argtypes = [i64, i64]
        L.flashdp_workspace_bytes_checkpoint8.argtypes = [lp, ci, i64, i64, ci, ci]
        for n in ("flashdp_activation_workspace_bytes", "flashdp_layernorm_workspace_bytes", "flashdp_checkpoint8_bytes",
                  "flashdp_workspace_bytes_checkpoint8"):
            getattr(L, n).restype = sz
        L.flashdp_plain_grad.argtypes = [vp, vp, i64, i64, i64, i64, ci, vp, vp]
        L.flashdp_plain_grad.restype = ci
        L.flashdp_plain_grad_balanced.argtypes = [vp, vp, i64, i64, i64, i64, ci, vp, vp, sz, vp]
        L.flashdp_plain_grad_balanced.restype = ci
        L.flashdp_plain_grad_balanced_workspace_bytes.argtypes = []
        L.flashdp_plain_grad_balanced_workspace_bytes.restype = sz
        L.flashdp_noise_field.argtypes = [u64, u32, i64, vp, vp]
        L.flashdp_noise_field.restype = ci
        L.flashdp_box_muller.argtypes = [vp, i64, vp, vp]
        L.flashdp_box_muller.restype = ci
        L.flashdp_contraction_timeline.argtypes = [vp, vp, i64, i64, i64, i64, ci, vp, sz, vp, i64, vp]
        L.flashdp_contraction_timeline.restype = i64
        L.flashdp_mfma_probe.argtypes = [ci, ci, ci, vp, vp]
        L.flashdp_mfma_probe.restype = ci
        L.flashdp_set_stream.argtypes = [vp]
        L.flashdp_set_workspace.argtypes = [vp, sz]
        L.flashdp_set_dtype.argtypes = [ci]
        L.flashdp_set_layer.argtypes = [u32]
        L.flashdp_set_schedule.argtypes = [ci]
        L.flashdp_set_stages.argtypes = [ci]
        for n in ("flashdp_set_stream", "flashdp_set_workspace", "flashdp_set_dtype", "flashdp_set_layer",
                  "flashdp_set_schedule", "flashdp_set_stages", "flashdp_release", "flashdp_version"):
            getattr(L, n).restype = ci
        L.flashdp_last_schedule.restype = ctypes.c_char_p
        L.flashdp_last_kernel.restype = ctypes.c_char_p
        L.flashdp_status_string.argtypes = [ci]
        L.flashdp_status_string.restype = ctypes.c_char_p
        _lib = L
    return _lib


def status_string(status: int) -> str:
    return lib().flashdp_status_string(int(status)).decode()


def _check(status: int, where: str):
    if status != OK:
        raise FlashDPError(status, where)


def _ptr(t) -> Optional[int]:
    return None if t is None else int(t.data_ptr())


def _stream_handle(stream) -> Optional[int]:
    if stream is None:
        import torch
        return int(torch.cuda.current_stream().cuda_stream) or None
    if isinstance(stream, int):
        return stream or None
    return int(stream.cuda_stream) or None


def dtype_code(t) -> int:
    import torch
    return {torch.bfloat16: BF16, torch.float32: F32, torch.float16: F16}[t.dtype]


def schedule_code(s) -> int:
    return _SCHEDULES[s] if isinstance(s, str) else int(s)


def activation_code(a) -> int:
    if a is None or isinstance(a, str):
        if a not in _ACTIVATIONS:
            raise FlashDPError(INVALID_ARGUMENT, f"activation {a!r}")
        return _ACTIVATIONS[a]
    return int(a)


# ---- thread-local context -------------------------------------------------------------------------

def flashdp_set_stream(stream=None):
    _check(lib().flashdp_set_stream(_stream_handle(stream)), "flashdp_set_stream")


def flashdp_set_workspace(workspace=None):
    if workspace is None:
        _check(lib().flashdp_set_workspace(None, 0), "flashdp_set_workspace")
    else:
        _check(lib().flashdp_set_workspace(_ptr(workspace), workspace.numel() * workspace.element_size()),
               "flashdp_set_workspace")


def flashdp_set_dtype(dtype: int):
    _check(lib().flashdp_set_dtype(int(dtype)), "flashdp_set_dtype")


def flashdp_set_layer(layer: int):
    _check(lib().flashdp_set_layer(int(layer)), "flashdp_set_layer")


def flashdp_set_schedule(schedule):
    _check(lib().flashdp_set_schedule(schedule_code(schedule)), "flashdp_set_schedule")


STAGE_CONTRACT, STAGE_CLIP, STAGE_AGGREGATE, STAGE_ALL = 1, 2, 4, 7


def flashdp_set_stages(mask: int = STAGE_ALL):
    _check(lib().flashdp_set_stages(int(mask)), "flashdp_set_stages")


def flashdp_release():
    _check(lib().flashdp_release(), "flashdp_release")


def flashdp_last_schedule() -> str:
    return lib().flashdp_last_schedule().decode()


def flashdp_last_kernel() -> str:
    return lib().flashdp_last_kernel().decode()


def flashdp_version() -> int:
    return lib().flashdp_version()


# ---- entry points ---------------------------------------------------------------------------------

def flashdp_linear_dp_grad(X, dY, B: int, T: int, d_in: int, d_out: int, C: float, sigma: float, seed: int,
                           out_grad, out_norms=None):
    """X [B,T,d_in], dY [B,T,d_out] device tensors of the context dtype; out_grad [d_out,d_in] fp32,
    out_norms [B] fp32 (or None).  Uses the thread's context (stream, dtype, layer, schedule, workspace)."""
    _check(lib().flashdp_linear_dp_grad(_ptr(X), _ptr(dY), B, T, d_in, d_out, C, sigma, seed,
                                        _ptr(out_grad), _ptr(out_norms)), "flashdp_linear_dp_grad")


def make_layers(layers: Sequence[dict]):
    """layers: dicts with X, dY, d_in, d_out, C, sigma, seed, layer, out_grad, out_norms (tensors or None)."""
    arr = (flashdp_layer_t * len(layers))()
    for k, L in enumerate(layers):
        arr[k].X = _ptr(L["X"])
        arr[k].dY = _ptr(L["dY"])
        arr[k].d_in = int(L["d_in"])
        arr[k].d_out = int(L["d_out"])
        arr[k].C = float(L["C"])
        arr[k].sigma = float(L["sigma"])
        arr[k].seed = int(L["seed"])
        arr[k].layer = int(L["layer"])
        arr[k].out_grad = _ptr(L["out_grad"])
        arr[k].out_norms = _ptr(L.get("out_norms"))
    return arr


def flashdp_workspace_bytes(layers, B: int, T: int, dtype: int, schedule=SCHEDULE_SCRATCH) -> int:
    arr = layers if not isinstance(layers, (list, tuple)) else make_layers(layers)
    return int(lib().flashdp_workspace_bytes(arr, len(arr), B, T, int(dtype), schedule_code(schedule)))


def flashdp_workspace_bytes_chunked(layers, B: int, T: int, dtype: int, chunk_samples: int, slots: int = 1) -> int:
    arr = layers if not isinstance(layers, (list, tuple)) else make_layers(layers)
    return int(lib().flashdp_workspace_bytes_chunked(arr, len(arr), B, T, int(dtype), int(chunk_samples), int(slots)))


def flashdp_last_chunk() -> int:
    return int(lib().flashdp_last_chunk())


def flashdp_block_dp_grad(layers, B: int, T: int, dtype: int, schedule=SCHEDULE_AUTO, workspace=None, stream=None):
    arr = layers if not isinstance(layers, (list, tuple)) else make_layers(layers)
    ws_ptr = _ptr(workspace)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().flashdp_block_dp_grad(arr, len(arr), B, T, int(dtype), schedule_code(schedule), ws_ptr, ws_bytes,
                                       _stream_handle(stream)), "flashdp_block_dp_grad")


def flashdp_block_dp_grad_micro(layers, B: int, T: int, dtype: int, schedule=SCHEDULE_AUTO, workspace=None, stream=None,
                                accumulate: bool = False, add_noise: bool = True):
    arr = layers if not isinstance(layers, (list, tuple)) else make_layers(layers)
    ws_ptr = _ptr(workspace)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().flashdp_block_dp_grad_micro(arr, len(arr), B, T, int(dtype), schedule_code(schedule), ws_ptr, ws_bytes,
                                             _stream_handle(stream), int(bool(accumulate)), int(bool(add_noise))),
           "flashdp_block_dp_grad_micro")


def flashdp_linear_dp_grad_static(X, dY, B: int, T: int, d_in: int, d_out: int, dtype: int, C: float, sigma: float,
                                  seed: int, layer: int, out_grad, out_norms=None, stream=None):
    """The entry point that allocates nothing: one layer, scratch schedule, workspace in the library's static array."""
    _check(lib().flashdp_linear_dp_grad_static(_ptr(X), _ptr(dY), B, T, d_in, d_out, int(dtype), C, sigma, seed, layer,
                                               _ptr(out_grad), _ptr(out_norms), _stream_handle(stream)),
           "flashdp_linear_dp_grad_static")


def flashdp_static_scratch_bytes() -> int:
    return int(lib().flashdp_static_scratch_bytes())


def flashdp_plain_grad(X, dY, B: int, T: int, d_in: int, d_out: int, dtype: int, out_grad, stream=None):
    _check(lib().flashdp_plain_grad(_ptr(X), _ptr(dY), B, T, d_in, d_out, int(dtype), _ptr(out_grad),
                                    _stream_handle(stream)), "flashdp_plain_grad")


def flashdp_plain_grad_balanced(X, dY, B: int, T: int, d_in: int, d_out: int, dtype: int, out_grad, workspace=None, stream=None):
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().flashdp_plain_grad_balanced(_ptr(X), _ptr(dY), B, T, d_in, d_out, int(dtype), _ptr(out_grad),
                                             _ptr(workspace), ws_bytes, _stream_handle(stream)), "flashdp_plain_grad_balanced")


def flashdp_plain_grad_balanced_workspace_bytes() -> int:
    return int(lib().flashdp_plain_grad_balanced_workspace_bytes())


def flashdp_noise_field(seed: int, layer: int, n: int, z, stream=None):
    _check(lib().flashdp_noise_field(seed, layer, n, _ptr(z), _stream_handle(stream)), "flashdp_noise_field")


def flashdp_box_muller(words, n_groups: int, z, stream=None):
    _check(lib().flashdp_box_muller(_ptr(words), n_groups, _ptr(z), _stream_handle(stream)), "flashdp_box_muller")


def flashdp_contraction_timeline(X, dY, B: int, T: int, d_in: int, d_out: int, park: bool, workspace, trace, stream=None) -> int:
    """trace: int64 device tensor of 8 words per workgroup, zeroed; returns the number of workgroups launched."""
    n = lib().flashdp_contraction_timeline(_ptr(X), _ptr(dY), B, T, d_in, d_out, int(bool(park)), _ptr(workspace),
                                           workspace.numel() * workspace.element_size(), _ptr(trace), trace.numel() // 8,
                                           _stream_handle(stream))
    if n < 0:
        raise FlashDPError(int(n), "flashdp_contraction_timeline")
    return int(n)


def flashdp_mfma_probe(pattern: int, iters: int, workgroups: int, sink, stream=None):
    _check(lib().flashdp_mfma_probe(int(pattern), int(iters), int(workgroups), _ptr(sink), _stream_handle(stream)),
           "flashdp_mfma_probe")


# ---- the layers around the weight gradient ----------------------------------------------------------

_FLOATS = {}
_torch = None


def _float_type(dtype: int):
    global _torch
    if _torch is None:
        import torch
        _FLOATS.update({BF16: torch.bfloat16, F32: torch.float32, F16: torch.float16})
        _torch = torch
    return _FLOATS.get(dtype)


def _buffer(t, n: int, dtype, where: str, device: int) -> Optional[int]:
    """Address of a tensor that a call uses as a buffer of n elements on its device: rows lie one after the other, and the type is
    the call's.  (A view with strides of its own, or a shorter one, would be read and written past its end.)"""
    if t is None:
        return None
    if t.dtype is not dtype or not t.is_contiguous() or t.numel() < n or t.get_device() != device:
        raise FlashDPError(INVALID_ARGUMENT, f"{where}: a contiguous tensor of {dtype} with {n} elements on device {device} is needed, "
                                             f"not {tuple(t.shape)} {t.dtype} on {t.device}")
    return t.data_ptr()


def _here(t, stream, where: str):
    """Handle of the stream to enqueue on, and the device.  The library works on the current device; so has the caller's tensor to be."""
    device = t.get_device()
    if device < 0 or device != _torch.cuda.current_device():
        raise FlashDPError(INVALID_ARGUMENT, f"{where}: the tensors are on {t.device}, which is not the current device")
    if stream is None:
        return _torch._C._cuda_getCurrentRawStream(device) or None, device      # (torch.cuda.current_stream() makes an object, a microsecond)
    return _stream_handle(stream), device


def _room(workspace, where: str, device: int):
    if workspace is None:
        return None, 0
    return _buffer(workspace, 0, workspace.dtype, where, device), workspace.numel() * workspace.element_size()


def flashdp_linear_forward(X, W, bias, residual, rows: int, d_in: int, d_out: int, dtype: int, activation, Y, Z=None, z_8bit: bool = False,
                           stream=None):
    """Y = act(X W^T + bias) + residual; Z, if given, receives X W^T + bias, in the call's type or as an 8-bit checkpoint (a uint8
    tensor of flashdp_checkpoint8_bytes(rows, d_out)).  activation: a name or code."""
    w, f = "flashdp_linear_forward", _float_type(dtype)
    st, dev = _here(X, stream, w)
    z = _buffer(Z, flashdp_checkpoint8_bytes(rows, d_out), _torch.uint8, w, dev) if z_8bit else _buffer(Z, rows * d_out, f, w, dev)
    _check(lib().flashdp_linear_forward(_buffer(X, rows * d_in, f, w, dev), _buffer(W, d_out * d_in, f, w, dev), _buffer(bias, d_out, f, w, dev),
                                        _buffer(residual, rows * d_out, f, w, dev), rows, d_in, d_out, int(dtype), activation_code(activation),
                                        _buffer(Y, rows * d_out, f, w, dev), z, int(bool(z_8bit)), st), w)


def flashdp_activation_workspace_bytes(B: int, T: int, d_out: int, dtype: int) -> int:
    return int(lib().flashdp_activation_workspace_bytes(B, T, d_out, int(dtype)))


def flashdp_activation_dp_grad(dY, Z, z_8bit: bool, B: int, T: int, d_out: int, dtype: int, activation, C: float, sigma: float, seed: int, layer: int,
                               dZ, out_grad, out_norms=None, workspace=None, stream=None, accumulate: bool = False, add_noise: bool = True):
    """dZ = dY act'(Z) and the clipped, noised gradient of the bias (out_grad [d_out] fp32, or None)."""
    w, f, n = "flashdp_activation_dp_grad", _float_type(dtype), B * T * d_out
    st, dev = _here(dY, stream, w)
    z = _buffer(Z, flashdp_checkpoint8_bytes(B * T, d_out), _torch.uint8, w, dev) if z_8bit else _buffer(Z, n, f, w, dev)
    ws, ws_bytes = _room(workspace, w, dev)
    _check(lib().flashdp_activation_dp_grad(_buffer(dY, n, f, w, dev), z, int(bool(z_8bit)), B, T, d_out, int(dtype), activation_code(activation), C, sigma, seed, layer,
                                            _buffer(dZ, n, f, w, dev), _buffer(out_grad, d_out, _torch.float32, w, dev), _buffer(out_norms, B, _torch.float32, w, dev),
                                            ws, ws_bytes, st, int(bool(accumulate)), int(bool(add_noise))), w)


def flashdp_layernorm_forward(X, gamma, beta, rows: int, d: int, dtype: int, eps: float, Y, mean=None, rstd=None, stream=None):
    """Y = (X - mean) rstd gamma + beta over rows of d features; mean and rstd [rows] fp32 are kept for the backward pass if given."""
    w, f = "flashdp_layernorm_forward", _float_type(dtype)
    st, dev = _here(X, stream, w)
    _check(lib().flashdp_layernorm_forward(_buffer(X, rows * d, f, w, dev), _buffer(gamma, d, f, w, dev), _buffer(beta, d, f, w, dev), rows, d, int(dtype), eps,
                                           _buffer(Y, rows * d, f, w, dev), _buffer(mean, rows, _torch.float32, w, dev), _buffer(rstd, rows, _torch.float32, w, dev), st), w)


def flashdp_layernorm_workspace_bytes(B: int, T: int, d: int, dtype: int, bias: bool = True) -> int:
    return int(lib().flashdp_layernorm_workspace_bytes(B, T, d, int(dtype), int(bool(bias))))


def flashdp_layernorm_dp_grad(X, dY, gamma, mean, rstd, B: int, T: int, d: int, dtype: int, C: float, sigma: float, seed: int, layer: int, dX, out_grad,
                              out_norms=None, bias: bool = True, workspace=None, stream=None, accumulate: bool = False, add_noise: bool = True):
    """dX and the clipped, noised gradient of gamma and beta (out_grad [2, d] fp32; [d] without a bias; or None)."""
    w, f, n = "flashdp_layernorm_dp_grad", _float_type(dtype), B * T * d
    st, dev = _here(X, stream, w)
    ws, ws_bytes = _room(workspace, w, dev)
    _check(lib().flashdp_layernorm_dp_grad(_buffer(X, n, f, w, dev), _buffer(dY, n, f, w, dev), _buffer(gamma, d, f, w, dev), _buffer(mean, B * T, _torch.float32, w, dev),
                                           _buffer(rstd, B * T, _torch.float32, w, dev), B, T, d, int(dtype), C, sigma, seed, layer, _buffer(dX, n, f, w, dev),
                                           _buffer(out_grad, (2 if bias else 1) * d, _torch.float32, w, dev), _buffer(out_norms, B, _torch.float32, w, dev), int(bool(bias)),
                                           ws, ws_bytes, st, int(bool(accumulate)), int(bool(add_noise))), w)


def flashdp_checkpoint8_bytes(rows: int, d: int) -> int:
    return int(lib().flashdp_checkpoint8_bytes(rows, d))


def flashdp_checkpoint8_pack(X, rows: int, d: int, dtype: int, packed, stream=None):
    w, f = "flashdp_checkpoint8_pack", _float_type(dtype)
    st, dev = _here(X, stream, w)
    _check(lib().flashdp_checkpoint8_pack(_buffer(X, rows * d, f, w, dev), rows, d, int(dtype),
                                          _buffer(packed, flashdp_checkpoint8_bytes(rows, d), _torch.uint8, w, dev), st), w)


def flashdp_checkpoint8_unpack(packed, rows: int, d: int, dtype: int, X, stream=None):
    w, f = "flashdp_checkpoint8_unpack", _float_type(dtype)
    st, dev = _here(packed, stream, w)
    _check(lib().flashdp_checkpoint8_unpack(_buffer(packed, flashdp_checkpoint8_bytes(rows, d), _torch.uint8, w, dev), rows, d, int(dtype),
                                            _buffer(X, rows * d, f, w, dev), st), w)


def flashdp_workspace_bytes_checkpoint8(layers, B: int, T: int, dtype: int, schedule=SCHEDULE_SCRATCH) -> int:
    arr = layers if not isinstance(layers, (list, tuple)) else make_layers(layers)
    return int(lib().flashdp_workspace_bytes_checkpoint8(arr, len(arr), B, T, int(dtype), schedule_code(schedule)))


def flashdp_block_dp_grad_checkpoint8(layers, B: int, T: int, dtype: int, schedule=SCHEDULE_AUTO, workspace=None, stream=None,
                                      accumulate: bool = False, add_noise: bool = True):
    """flashdp_block_dp_grad_micro with each layer's X an 8-bit checkpoint (a uint8 tensor of flashdp_checkpoint8_bytes(B * T, d_in))."""
    w, f = "flashdp_block_dp_grad_checkpoint8", _float_type(dtype)
    arr, st, dev = layers, None, None
    if isinstance(layers, (list, tuple)):
        for L in layers:
            st, dev = _here(L["X"], stream, w)
            _buffer(L["X"], flashdp_checkpoint8_bytes(B * T, L["d_in"]), _torch.uint8, w, dev)
            _buffer(L["dY"], B * T * L["d_out"], f, w, dev)
            _buffer(L["out_grad"], L["d_in"] * L["d_out"], _torch.float32, w, dev)
            _buffer(L.get("out_norms"), B, _torch.float32, w, dev)
        arr = make_layers(layers)
    else:
        st, dev = _stream_handle(stream), _torch.cuda.current_device() if workspace is not None else None
    ws, ws_bytes = _room(workspace, w, dev)
    _check(lib().flashdp_block_dp_grad_checkpoint8(arr, len(arr), B, T, int(dtype), schedule_code(schedule), ws, ws_bytes, st,
                                                   int(bool(accumulate)), int(bool(add_noise))), w)
