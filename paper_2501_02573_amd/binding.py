"""ctypes binding of libleet_attn.so: argument marshalling only.

Every function takes torch tensors that already live on the GPU, checks shapes,
dtypes and contiguity on the host, and passes raw device pointers plus the current
torch stream to the C ABI declared in ``include/leet_attn.h``.  No arithmetic of the
operator happens here, and there is no fallback: if the native library is missing the
import of this module fails.
"""
from __future__ import annotations

import ctypes
import os
import struct
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libleet_attn.so")

LEET_F32, LEET_BF16, LEET_F16 = 0, 1, 2
LEET_MASK_DECAY, LEET_MASK_CAUSAL = 0, 1
LEET_OK, LEET_ERR_INVALID_ARG, LEET_ERR_UNSUPPORTED, LEET_ERR_LAUNCH, LEET_ERR_TOO_LARGE = 0, 1, 2, 3, 4
LEET_ERR_CAPTURE, LEET_ERR_SCRATCH_LIMIT = 5, 6
LEET_CHOICE_DEFAULT = -1
ROPE_HALF, ROPE_INTERLEAVED = 0, 1
ROPE_SCALING_NONE, ROPE_SCALING_LINEAR, ROPE_SCALING_BASE, ROPE_SCALING_BANDS, ROPE_SCALING_TURNS = 0, 1, 2, 3, 4
GATE_DECAY, GATE_LOG, GATE_SIGMOID = 0, 1, 2

EXPORTED_SYMBOLS = (
    "leet_attn_forward",
    "leet_attn_decode_step",
    "leet_attn_decode_step_ex",
    "leet_attn_forward_ex",
    "leet_attn_forward_v2",
    "leet_attn_decode_step_v2",
    "leet_attn_forward_recurrent",
    "leet_attn_forward_rd",
    "leet_attn_forward_recurrent_rd",
    "leet_attn_forward_fleet",
    "leet_attn_decode_step_rd",
    "leet_attn_workspace_bytes_rd",
    "leet_attn_forward_v3",
    "leet_attn_workspace_bytes_v3",
    "leet_attn_query_plan_v3",
    "leet_attn_decode_step_v3",
    "leet_attn_forward_static",
    "leet_attn_static_scratch_bytes",
    "leet_attn_forward_profile",
    "leet_attn_calibration_stream",
    "leet_attn_set_bf16_kernel",
    "leet_attn_get_bf16_kernel",
    "leet_attn_query_plan",
    "leet_attn_query_plan_rd",
    "leet_attn_set_decode_store",
    "leet_attn_get_decode_store",
    "leet_attn_workspace_bytes",
    "leet_attn_release_workspace",
    "leet_attn_rope_frequencies",
    "leet_attn_rope",
    "leet_attn_qk_norm_rope",
    "leet_attn_qk_norm_rope_backward",
    "leet_attn_qk_norm_rope_workspace_bytes",
    "leet_attn_gated_scan",
    "leet_attn_gated_scan_backward",
    "leet_attn_gated_scan_workspace_bytes",
    "leet_attn_gated_scan_step",
    "leet_attn_strerror",
    "leet_attn_version",
)


class LeetAttnError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: status {status}: {strerror(status)}")


# The library's small argument structures, packed: a tenth of a ctypes.Structure's time, and a call takes up to seven.
# A call passes the bytes where the library takes a pointer to the structure.
_pack_heads = struct.Struct("@P3q").pack      # leet_attn_heads: data, batch, head, token
_pack_rows = struct.Struct("@P2q").pack       # leet_attn_rows: data, batch, token
_pack_rotation = struct.Struct("@PiiPqqf4x").pack  # leet_attn_rotation


def _load() -> ctypes.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} is missing: build it with `python -m paper_2501_02573_amd.build` "
            "(there is no CPU or PyTorch fallback for this library)")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
    lib.leet_attn_forward.argtypes = [vp, vp, vp, vp, vp, i, i, i, i, i, vp]
    lib.leet_attn_forward.restype = i
    lib.leet_attn_forward_ex.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, sz, i, i, i, i, i, i, vp]
    lib.leet_attn_forward_ex.restype = i
    lib.leet_attn_forward_v2.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, sz, i, i, i, i, i, i, i, i, vp]
    lib.leet_attn_forward_v2.restype = i
    lib.leet_attn_decode_step_v2.argtypes = [vp, vp, vp, vp, vp, vp, i, i, i, i, i, vp]
    lib.leet_attn_decode_step_v2.restype = i
    lib.leet_attn_forward_recurrent.argtypes = [vp, vp, vp, vp, vp, vp, vp, i, i, i, i, i, i, vp]
    lib.leet_attn_forward_recurrent.restype = i
    lib.leet_attn_forward_rd.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, sz, i, i, i, i, i, i, i, i, i, vp]
    lib.leet_attn_forward_rd.restype = i
    lib.leet_attn_forward_recurrent_rd.argtypes = [vp, vp, vp, vp, vp, vp, vp, i, i, i, i, i, i, i, vp]
    lib.leet_attn_forward_recurrent_rd.restype = i
    lib.leet_attn_forward_fleet.argtypes = [vp, vp, vp, vp, vp, vp, vp, i, i, i, i, i, i, i, vp]
    lib.leet_attn_forward_fleet.restype = i
    lib.leet_attn_decode_step_rd.argtypes = [vp, vp, vp, vp, vp, vp, i, i, i, i, i, i, vp]
    lib.leet_attn_decode_step_rd.restype = i
    lib.leet_attn_workspace_bytes_rd.argtypes = [i, i, i, i, i, i, i]
    lib.leet_attn_workspace_bytes_rd.restype = sz
    lib.leet_attn_forward_v3.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, sz, i, i, i, i, i, i, i, i, i, i, vp]
    lib.leet_attn_forward_v3.restype = i
    lib.leet_attn_workspace_bytes_v3.argtypes = [i, i, i, i, i, i, i, i]
    lib.leet_attn_workspace_bytes_v3.restype = sz
    lib.leet_attn_query_plan_v3.argtypes = [i, i, i, i, i, i, i, i, ctypes.POINTER(i), ctypes.POINTER(i)]
    lib.leet_attn_query_plan_v3.restype = i
    lib.leet_attn_decode_step_v3.argtypes = [vp, vp, vp, vp, vp, vp, i, i, i, i, i, i, i, vp]
    lib.leet_attn_decode_step_v3.restype = i
    lib.leet_attn_forward_static.argtypes = [vp, vp, vp, vp, vp, vp, vp, i, i, i, i, i, i, vp]
    lib.leet_attn_forward_static.restype = i
    lib.leet_attn_static_scratch_bytes.argtypes = []
    lib.leet_attn_static_scratch_bytes.restype = sz
    lib.leet_attn_forward_profile.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, sz, i, i, i, i, i, i, vp,
                                              ctypes.POINTER(ctypes.c_float)]
    lib.leet_attn_forward_profile.restype = i
    lib.leet_attn_calibration_stream.argtypes = [i, vp, vp, sz, i, vp]
    lib.leet_attn_calibration_stream.restype = i
    lib.leet_attn_decode_step.argtypes = [vp, vp, vp, vp, vp, vp, i, i, i, vp]
    lib.leet_attn_decode_step.restype = i
    lib.leet_attn_decode_step_ex.argtypes = [vp, vp, vp, vp, vp, vp, i, i, i, i, vp]
    lib.leet_attn_decode_step_ex.restype = i
    lib.leet_attn_workspace_bytes.argtypes = [i, i, i, i, i, i]
    lib.leet_attn_workspace_bytes.restype = sz
    lib.leet_attn_release_workspace.argtypes = []
    lib.leet_attn_release_workspace.restype = i
    lib.leet_attn_set_bf16_kernel.argtypes = [i]
    lib.leet_attn_set_bf16_kernel.restype = i
    lib.leet_attn_get_bf16_kernel.argtypes = []
    lib.leet_attn_get_bf16_kernel.restype = i
    lib.leet_attn_query_plan.argtypes = [i, i, i, i, i, i, ctypes.POINTER(i), ctypes.POINTER(i)]
    lib.leet_attn_query_plan.restype = i
    lib.leet_attn_query_plan_rd.argtypes = [i, i, i, i, i, i, i, ctypes.POINTER(i), ctypes.POINTER(i)]
    lib.leet_attn_query_plan_rd.restype = i
    lib.leet_attn_set_decode_store.argtypes = [i]
    lib.leet_attn_set_decode_store.restype = i
    lib.leet_attn_get_decode_store.argtypes = []
    lib.leet_attn_get_decode_store.restype = i
    heads = rotation = rows = vp  # packed structures
    d = ctypes.c_double
    lib.leet_attn_rope_frequencies.argtypes = [i, d, i, d, i, d, d, vp, ctypes.POINTER(ctypes.c_float)]
    lib.leet_attn_rope_frequencies.restype = i
    lib.leet_attn_rope.argtypes = [heads, heads, i, heads, heads, i, rotation, i, i, i, i, i, vp]
    lib.leet_attn_rope.restype = i
    lib.leet_attn_qk_norm_rope.argtypes = [heads, heads, i, heads, heads, i, vp, vp, i, ctypes.c_float, rotation,
                                           i, i, i, i, vp]
    lib.leet_attn_qk_norm_rope.restype = i
    lib.leet_attn_qk_norm_rope_backward.argtypes = [heads, heads, heads, i, heads, heads, heads, i, vp, vp, vp, vp, i,
                                                    ctypes.c_float, rotation, vp, sz, i, i, i, i, vp]
    lib.leet_attn_qk_norm_rope_backward.restype = i
    lib.leet_attn_qk_norm_rope_workspace_bytes.argtypes = [i, i, i, i, i]
    lib.leet_attn_qk_norm_rope_workspace_bytes.restype = sz
    lib.leet_attn_gated_scan.argtypes = [rows, rows, rows, vp, vp, vp, i, vp, sz, i, i, i, i, i, i, vp]
    lib.leet_attn_gated_scan.restype = i
    lib.leet_attn_gated_scan_backward.argtypes = [rows, rows, rows, rows, rows, rows, vp, vp, vp, vp, i, vp, sz,
                                                  i, i, i, i, i, i, vp]
    lib.leet_attn_gated_scan_backward.restype = i
    lib.leet_attn_gated_scan_workspace_bytes.argtypes = [i, i, i, i]
    lib.leet_attn_gated_scan_workspace_bytes.restype = sz
    lib.leet_attn_gated_scan_step.argtypes = [rows, rows, rows, vp, i, i, i, i, i, vp]
    lib.leet_attn_gated_scan_step.restype = i
    lib.leet_attn_strerror.argtypes = [i]
    lib.leet_attn_strerror.restype = ctypes.c_char_p
    lib.leet_attn_version.argtypes = []
    lib.leet_attn_version.restype = ctypes.c_char_p
    return lib


lib = _load()


def strerror(status: int) -> str:
    return lib.leet_attn_strerror(int(status)).decode()


def version() -> str:
    return lib.leet_attn_version().decode()


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return LEET_F32
    if t.dtype == torch.bfloat16:
        return LEET_BF16
    if t.dtype == torch.float16:
        return LEET_F16
    raise TypeError(f"unsupported dtype {t.dtype}: q, k, v must be float32, bfloat16 or float16")


def _check_dev(*tensors: Optional[torch.Tensor]) -> torch.device:
    dev = None
    for t in tensors:
        if t is None:
            continue
        if not t.is_cuda:
            raise ValueError("all tensors must be GPU tensors")
        if not t.is_contiguous():
            raise ValueError("all tensors must be contiguous")
        if dev is None:
            dev = t.device
        elif t.device != dev:
            raise ValueError("all tensors must be on one device")
    return dev


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


# What a short call costs is its host time (a decode step of one user: 3.8 us on the GPU, 13.7 us a call
# with a device guard, a Stream object and a c_void_p per argument; 9.1 us as below): the device
# guard is entered only where it would change the device, the stream is taken as the raw handle, and
# addresses travel as plain integers.
# The raw handle's call is private to torch; where it is missing, the public one makes an object for it.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda index: torch.cuda.current_stream(index).cuda_stream)


def _call(fn, dev: torch.device, *args) -> int:
    """fn(*args, the device's current stream) with ``dev`` current; returns the status."""
    index = dev.index
    if index == torch.cuda.current_device():
        return fn(*args, _raw_stream(index))
    with torch.cuda.device(dev):
        return fn(*args, _raw_stream(index))


_Tensor, _empty_like, _dense = torch.Tensor, torch.empty_like, torch.contiguous_format


def _new_out(like: torch.Tensor, dtype: torch.dtype) -> torch.Tensor:
    """A fresh dense tensor of ``like``'s shape and device: strides and class are not taken over."""
    if type(like) is _Tensor:  # 2 us less than torch.empty
        return _empty_like(like, dtype=dtype, memory_format=_dense)
    return torch.empty(like.shape, dtype=dtype, device=like.device)


KERNEL_WIDE, KERNEL_COLUMN_SPLIT, KERNEL_AUTO = 0, 1, 2


def set_bf16_kernel(which: int) -> None:
    st = lib.leet_attn_set_bf16_kernel(int(which))
    if st != LEET_OK:
        raise LeetAttnError(st, "leet_attn_set_bf16_kernel")


def get_bf16_kernel() -> int:
    return int(lib.leet_attn_get_bf16_kernel())


DECODE_STORE_AUTO, DECODE_STORE_CACHED, DECODE_STORE_STREAM = 0, 1, 2


def set_decode_store(mode: int) -> None:
    st = lib.leet_attn_set_decode_store(int(mode))
    if st != LEET_OK:
        raise LeetAttnError(st, "leet_attn_set_decode_store")


def get_decode_store() -> int:
    return int(lib.leet_attn_get_decode_store())


def query_plan(B: int, H: int, N: int, d: int, dtype: int, segments: int = 0):
    """(segments per sequence, kernel) the library would use for this shape (host-only query)."""
    nseg, kern = ctypes.c_int(0), ctypes.c_int(0)
    st = lib.leet_attn_query_plan(B, H, N, d, dtype, segments, ctypes.byref(nseg), ctypes.byref(kern))
    if st != LEET_OK:
        raise LeetAttnError(st, "leet_attn_query_plan")
    return nseg.value, kern.value


def query_plan_rd(B: int, H: int, N: int, r: int, dv: int, dtype: int, segments: int = 0):
    """``query_plan`` for rank r and value width dv given separately."""
    nseg, kern = ctypes.c_int(0), ctypes.c_int(0)
    st = lib.leet_attn_query_plan_rd(B, H, N, r, dv, dtype, segments, ctypes.byref(nseg), ctypes.byref(kern))
    if st != LEET_OK:
        raise LeetAttnError(st, "leet_attn_query_plan_rd")
    return nseg.value, kern.value


def workspace_bytes(B: int, H: int, N: int, d: int, dtype: int, segments: int = 0) -> int:
    return int(lib.leet_attn_workspace_bytes(B, H, N, d, dtype, segments))


def release_workspace() -> None:
    st = lib.leet_attn_release_workspace()
    if st != LEET_OK:
        raise LeetAttnError(st, "leet_attn_release_workspace")


def _check_forward(q, k, v, gamma, out, any_out_dtype: bool = False):
    if q.dim() != 4 or q.shape != k.shape or q.shape != v.shape:
        raise ValueError("q, k, v must share one [B, H, N, d] shape")
    if k.dtype != q.dtype or v.dtype != q.dtype:
        raise TypeError("q, k, v must share one dtype")
    B, H, N, d = q.shape
    if gamma is not None and (gamma.dtype != torch.float32 or gamma.numel() != H):
        raise ValueError("gamma must be float32 with one value per head")
    if out.shape != q.shape or (out.dtype != torch.float32 and not any_out_dtype):
        raise ValueError("out must be float32 [B, H, N, d]")
    return B, H, N, d


def leet_attn_forward(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, gamma: torch.Tensor,
                      out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Chunked prefill with zero initial state; returns fp32 ``out`` [B, H, N, d]."""
    if out is None:
        out = _new_out(q, torch.float32)
    B, H, N, d = _check_forward(q, k, v, gamma, out)
    dev = _check_dev(q, k, v, gamma, out)
    st = _call(lib.leet_attn_forward, dev, _ptr(q), _ptr(k), _ptr(v), _ptr(gamma), _ptr(out), B, H, N, d,
               _dtype_code(q))
    if st != LEET_OK:
        raise LeetAttnError(st, "leet_attn_forward")
    return out


def leet_attn_forward_ex(q, k, v, gamma, out: Optional[torch.Tensor] = None,
                         state_in: Optional[torch.Tensor] = None,
                         state_out: Optional[torch.Tensor] = None,
                         workspace: Optional[torch.Tensor] = None, segments: int = 0) -> torch.Tensor:
    """Chunked prefill with state hand-off and optional caller-owned workspace."""
    if out is None:
        out = _new_out(q, torch.float32)
    B, H, N, d = _check_forward(q, k, v, gamma, out)
    for name, s in (("state_in", state_in), ("state_out", state_out)):
        if s is not None and (s.dtype != torch.float32 or tuple(s.shape) != (B, H, d, d)):
            raise ValueError(f"{name} must be float32 [B, H, d, d]")
    ws_bytes = 0
    if workspace is not None:
        if workspace.dtype != torch.uint8:
            raise TypeError("workspace must be a uint8 tensor")
        ws_bytes = workspace.numel()
    dev = _check_dev(q, k, v, gamma, out, state_in, state_out, workspace)
    st = _call(lib.leet_attn_forward_ex, dev, _ptr(q), _ptr(k), _ptr(v), _ptr(gamma), _ptr(out), _ptr(state_in),
               _ptr(state_out), _ptr(workspace), ws_bytes, int(segments),
               B, H, N, d, _dtype_code(q))
    if st != LEET_OK:
        raise LeetAttnError(st, "leet_attn_forward_ex")
    return out


def leet_attn_forward_v2(q, k, v, gamma: Optional[torch.Tensor], out: Optional[torch.Tensor] = None,
                         state_in: Optional[torch.Tensor] = None,
                         state_out: Optional[torch.Tensor] = None,
                         workspace: Optional[torch.Tensor] = None, segments: int = 0,
                         out_dtype: Optional[torch.dtype] = None,
                         mask: int = LEET_MASK_DECAY) -> torch.Tensor:
    """Chunked prefill with every option: fp16 inputs, output in the input type, 0/1 causal mask.

    ``out_dtype`` (used when ``out`` is None) defaults to float32; ``gamma`` may be None with
    ``mask=LEET_MASK_CAUSAL``.  Unsupported combinations are reported by the library.
    """
    if out is None:
        out = _new_out(q, out_dtype or torch.float32)
    B, H, N, d = _check_forward(q, k, v, gamma, out, any_out_dtype=True)
    for name, s in (("state_in", state_in), ("state_out", state_out)):
        if s is not None and (s.dtype != torch.float32 or tuple(s.shape) != (B, H, d, d)):
            raise ValueError(f"{name} must be float32 [B, H, d, d]")
    ws_bytes = 0
    if workspace is not None:
        if workspace.dtype != torch.uint8:
            raise TypeError("workspace must be a uint8 tensor")
        ws_bytes = workspace.numel()
    dev = _check_dev(q, k, v, gamma, out, state_in, state_out, workspace)
    st = _call(lib.leet_attn_forward_v2, dev, _ptr(q), _ptr(k), _ptr(v), _ptr(gamma), _ptr(out), _ptr(state_in),
               _ptr(state_out), _ptr(workspace), ws_bytes, int(segments),
               B, H, N, d, _dtype_code(q), _dtype_code(out), int(mask))
    if st != LEET_OK:
        raise LeetAttnError(st, "leet_attn_forward_v2")
    return out


def leet_attn_forward_recurrent(q, k, v, gamma: Optional[torch.Tensor], out: Optional[torch.Tensor] = None,
                                state_in: Optional[torch.Tensor] = None,
                                state_out: Optional[torch.Tensor] = None,
                                mask: int = LEET_MASK_DECAY) -> torch.Tensor:
    """Row-based (token-by-token) prefill on the GPU: the comparison point for the chunked path."""
    if out is None:
        out = _new_out(q, torch.float32)
    B, H, N, d = _check_forward(q, k, v, gamma, out)
    for name, s in (("state_in", state_in), ("state_out", state_out)):
        if s is not None and (s.dtype != torch.float32 or tuple(s.shape) != (B, H, d, d)):
            raise ValueError(f"{name} must be float32 [B, H, d, d]")
    dev = _check_dev(q, k, v, gamma, out, state_in, state_out)
    st = _call(lib.leet_attn_forward_recurrent, dev, _ptr(q), _ptr(k), _ptr(v), _ptr(gamma), _ptr(out), _ptr(state_in),
               _ptr(state_out), B, H, N, d, _dtype_code(q), int(mask))
    if st != LEET_OK:
        raise LeetAttnError(st, "leet_attn_forward_recurrent")
    return out


def leet_attn_forward_profile(q, k, v, gamma, out: Optional[torch.Tensor] = None, segments: int = 0):
    """One prefill with per-kernel HIP-event timing; returns (out, [pre-pass ms, scan ms, walk ms])."""
    if out is None:
        out = _new_out(q, torch.float32)
    B, H, N, d = _check_forward(q, k, v, gamma, out)
    dev = _check_dev(q, k, v, gamma, out)
    ms = (ctypes.c_float * 3)()
    with torch.cuda.device(dev):
        st = lib.leet_attn_forward_profile(_ptr(q), _ptr(k), _ptr(v), _ptr(gamma), _ptr(out), None, None,
                                           None, 0, int(segments), B, H, N, d, _dtype_code(q),
                                           _raw_stream(dev.index), ms)
    if st != LEET_OK:
        raise LeetAttnError(st, "leet_attn_forward_profile")
    return out, [float(x) for x in ms]


def calibration_stream(mode: str, src: Optional[torch.Tensor], dst: torch.Tensor, nbytes: int,
                       workgroups: int = 4096) -> None:
    """Launches the plain copy / read / fill kernel over ``nbytes`` (measurement aid)."""
    code = {"copy": 0, "read": 1, "fill": 2, "copy_nt": 3, "fill_nt": 4}[mode]
    dev = _check_dev(src, dst)
    st = _call(lib.leet_attn_calibration_stream, dev, code, _ptr(src), _ptr(dst), int(nbytes), int(workgroups))
    if st != LEET_OK:
        raise LeetAttnError(st, "leet_attn_calibration_stream")


def _check_decode(q, k, v, gamma, state, out):
    if q.dim() != 3 or q.shape != k.shape or q.shape != v.shape:
        raise ValueError("q, k, v must share one [B, H, d] shape")
    if k.dtype != q.dtype or v.dtype != q.dtype:
        raise TypeError("q, k, v must share one dtype")
    B, H, d = q.shape
    if gamma is not None and (gamma.dtype != torch.float32 or gamma.numel() != H):
        raise ValueError("gamma must be float32 with one value per head")
    if state.dtype != torch.float32 or tuple(state.shape) != (B, H, d, d):
        raise ValueError("state must be float32 [B, H, d, d]")
    if out.dtype != torch.float32 or tuple(out.shape) != (B, H, d):
        raise ValueError("out must be float32 [B, H, d]")
    return B, H, d


def leet_attn_decode_step(q, k, v, gamma, state, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """One decode step with bf16 q, k, v: ``state`` is updated in place; returns fp32 ``out`` [B, H, d]."""
    if q.dtype != torch.bfloat16:
        raise TypeError("leet_attn_decode_step takes bfloat16 q, k, v (use leet_attn_decode_step_ex for float32)")
    if out is None:
        out = _new_out(q, torch.float32)
    B, H, d = _check_decode(q, k, v, gamma, state, out)
    dev = _check_dev(q, k, v, gamma, state, out)
    st = _call(lib.leet_attn_decode_step, dev, _ptr(q), _ptr(k), _ptr(v), _ptr(gamma), _ptr(state), _ptr(out),
               B, H, d)
    if st != LEET_OK:
        raise LeetAttnError(st, "leet_attn_decode_step")
    return out


def leet_attn_decode_step_ex(q, k, v, gamma, state, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """One decode step with float32 or bfloat16 q, k, v."""
    if out is None:
        out = _new_out(q, torch.float32)
    B, H, d = _check_decode(q, k, v, gamma, state, out)
    dev = _check_dev(q, k, v, gamma, state, out)
    st = _call(lib.leet_attn_decode_step_ex, dev, _ptr(q), _ptr(k), _ptr(v), _ptr(gamma), _ptr(state), _ptr(out),
               B, H, d, _dtype_code(q))
    if st != LEET_OK:
        raise LeetAttnError(st, "leet_attn_decode_step_ex")
    return out


def leet_attn_decode_step_v2(q, k, v, gamma: Optional[torch.Tensor], state, out: Optional[torch.Tensor] = None,
                             mask: int = LEET_MASK_DECAY) -> torch.Tensor:
    """One decode step with float32, bfloat16 or float16 q, k, v and either mask."""
    if out is None:
        out = _new_out(q, torch.float32)
    B, H, d = _check_decode(q, k, v, gamma, state, out)
    dev = _check_dev(q, k, v, gamma, state, out)
    st = _call(lib.leet_attn_decode_step_v2, dev, _ptr(q), _ptr(k), _ptr(v), _ptr(gamma), _ptr(state), _ptr(out),
               B, H, d, _dtype_code(q), int(mask))
    if st != LEET_OK:
        raise LeetAttnError(st, "leet_attn_decode_step_v2")
    return out


# ---------------------------------------------------------------- rank r different from the value width dv
def workspace_bytes_rd(B: int, H: int, N: int, r: int, dv: int, dtype: int, segments: int = 0) -> int:
    return int(lib.leet_attn_workspace_bytes_rd(B, H, N, r, dv, dtype, segments))


def _check_rd(q, k, v, gamma, out, any_out_dtype):
    if q.dim() != 4 or q.shape != k.shape or v.dim() != 4 or q.shape[:3] != v.shape[:3]:
        raise ValueError("q, k must share one [B, H, N, r] shape and v be [B, H, N, dv]")
    if k.dtype != q.dtype or v.dtype != q.dtype:
        raise TypeError("q, k, v must share one dtype")
    B, H, N, r = q.shape
    dv = v.shape[3]
    if gamma is not None and (gamma.dtype != torch.float32 or gamma.numel() != H):
        raise ValueError("gamma must be float32 with one value per head")
    if out.shape != v.shape or (out.dtype != torch.float32 and not any_out_dtype):
        raise ValueError("out must be [B, H, N, dv]" + ("" if any_out_dtype else " float32"))
    return B, H, N, r, dv


def _check_states_rd(B, H, r, dv, **states):
    for name, s in states.items():
        if s is not None and (s.dtype != torch.float32 or tuple(s.shape) != (B, H, r, dv)):
            raise ValueError(f"{name} must be float32 [B, H, r, dv]")


def leet_attn_forward_rd(q, k, v, gamma: Optional[torch.Tensor], out: Optional[torch.Tensor] = None,
                         state_in: Optional[torch.Tensor] = None, state_out: Optional[torch.Tensor] = None,
                         workspace: Optional[torch.Tensor] = None, segments: int = 0,
                         out_dtype: Optional[torch.dtype] = None, mask: int = LEET_MASK_DECAY) -> torch.Tensor:
    """Chunked prefill with q, k of width r and v, out of width dv; states are [B, H, r, dv]."""
    if out is None:
        out = _new_out(v, out_dtype or torch.float32)
    B, H, N, r, dv = _check_rd(q, k, v, gamma, out, True)
    _check_states_rd(B, H, r, dv, state_in=state_in, state_out=state_out)
    ws_bytes = 0
    if workspace is not None:
        if workspace.dtype != torch.uint8:
            raise TypeError("workspace must be a uint8 tensor")
        ws_bytes = workspace.numel()
    dev = _check_dev(q, k, v, gamma, out, state_in, state_out, workspace)
    st = _call(lib.leet_attn_forward_rd, dev, _ptr(q), _ptr(k), _ptr(v), _ptr(gamma), _ptr(out), _ptr(state_in),
               _ptr(state_out), _ptr(workspace), ws_bytes, int(segments),
               B, H, N, r, dv, _dtype_code(q), _dtype_code(out), int(mask))
    if st != LEET_OK:
        raise LeetAttnError(st, "leet_attn_forward_rd")
    return out


def leet_attn_forward_v3(q, k, v, gamma: Optional[torch.Tensor], out: Optional[torch.Tensor] = None,
                         state_in: Optional[torch.Tensor] = None, state_out: Optional[torch.Tensor] = None,
                         workspace: Optional[torch.Tensor] = None, segments: int = 0,
                         kernel: int = LEET_CHOICE_DEFAULT,
                         out_dtype: Optional[torch.dtype] = None, mask: int = LEET_MASK_DECAY) -> torch.Tensor:
    """``leet_attn_forward_rd`` with the kernel choice given per call."""
    if out is None:
        out = _new_out(v, out_dtype or torch.float32)
    B, H, N, r, dv = _check_rd(q, k, v, gamma, out, True)
    _check_states_rd(B, H, r, dv, state_in=state_in, state_out=state_out)
    ws_bytes = 0
    if workspace is not None:
        if workspace.dtype != torch.uint8:
            raise TypeError("workspace must be a uint8 tensor")
        ws_bytes = workspace.numel()
    dev = _check_dev(q, k, v, gamma, out, state_in, state_out, workspace)
    st = _call(lib.leet_attn_forward_v3, dev, _ptr(q), _ptr(k), _ptr(v), _ptr(gamma), _ptr(out), _ptr(state_in),
               _ptr(state_out), _ptr(workspace), ws_bytes, int(segments), int(kernel),
               B, H, N, r, dv, _dtype_code(q), _dtype_code(out), int(mask))
    if st != LEET_OK:
        raise LeetAttnError(st, "leet_attn_forward_v3")
    return out


class PreparedForward:
    """``leet_attn_forward_v3`` with the argument checks and the marshalling done once.

    For a serving loop that calls the library again and again on the same buffers (contents may
    change, addresses and shapes may not): calling the object makes one ctypes call into
    ``leet_attn_forward_v3`` on the device's current stream (or on ``stream``, a raw stream handle,
    if one was given) and nothing else.  The object keeps the tensors alive."""

    def __init__(self, q, k, v, gamma: Optional[torch.Tensor], out: torch.Tensor,
                 state_in: Optional[torch.Tensor] = None, state_out: Optional[torch.Tensor] = None,
                 workspace: Optional[torch.Tensor] = None, segments: int = 0,
                 kernel: int = LEET_CHOICE_DEFAULT, mask: int = LEET_MASK_DECAY, stream: Optional[int] = None):
        B, H, N, r, dv = _check_rd(q, k, v, gamma, out, True)
        _check_states_rd(B, H, r, dv, state_in=state_in, state_out=state_out)
        ws_bytes = 0
        if workspace is not None:
            if workspace.dtype != torch.uint8:
                raise TypeError("workspace must be a uint8 tensor")
            ws_bytes = workspace.numel()
        self._dev = _check_dev(q, k, v, gamma, out, state_in, state_out, workspace)
        self._keep = (q, k, v, gamma, out, state_in, state_out, workspace)
        self._args = (_ptr(q), _ptr(k), _ptr(v), _ptr(gamma), _ptr(out), _ptr(state_in), _ptr(state_out),
                      _ptr(workspace), ws_bytes, int(segments), int(kernel), B, H, N, r, dv,
                      _dtype_code(q), _dtype_code(out), int(mask))
        self._stream = None if stream is None else ctypes.c_void_p(stream)  # refuses what is not a handle
        self._fn = lib.leet_attn_forward_v3
        self.out = out

    def __call__(self) -> torch.Tensor:
        if torch.cuda.current_device() != self._dev.index:
            raise ValueError("PreparedForward called with another device current")
        stream = self._stream if self._stream is not None else _raw_stream(self._dev.index)
        st = self._fn(*self._args, stream)
        if st != LEET_OK:
            raise LeetAttnError(st, "leet_attn_forward_v3")
        return self.out


def workspace_bytes_v3(B: int, H: int, N: int, r: int, dv: int, dtype: int, segments: int = 0,
                       kernel: int = LEET_CHOICE_DEFAULT) -> int:
    return int(lib.leet_attn_workspace_bytes_v3(B, H, N, r, dv, dtype, segments, kernel))


def query_plan_v3(B: int, H: int, N: int, r: int, dv: int, dtype: int, segments: int = 0,
                  kernel: int = LEET_CHOICE_DEFAULT):
    """``query_plan_rd`` with the kernel choice given per call."""
    nseg, kern = ctypes.c_int(0), ctypes.c_int(0)
    st = lib.leet_attn_query_plan_v3(B, H, N, r, dv, dtype, segments, kernel, ctypes.byref(nseg), ctypes.byref(kern))
    if st != LEET_OK:
        raise LeetAttnError(st, "leet_attn_query_plan_v3")
    return nseg.value, kern.value


def static_scratch_bytes() -> int:
    return int(lib.leet_attn_static_scratch_bytes())


def leet_attn_forward_static(q, k, v, gamma, out: torch.Tensor, state_in: Optional[torch.Tensor] = None,
                             state_out: Optional[torch.Tensor] = None, segments: int = 0) -> torch.Tensor:
    """Chunked prefill that allocates nothing: segment states in the library's static scratch.

    ``out`` is required (this binding allocates nothing for the call either)."""
    B, H, N, d = _check_forward(q, k, v, gamma, out)
    for name, s in (("state_in", state_in), ("state_out", state_out)):
        if s is not None and (s.dtype != torch.float32 or tuple(s.shape) != (B, H, d, d)):
            raise ValueError(f"{name} must be float32 [B, H, d, d]")
    dev = _check_dev(q, k, v, gamma, out, state_in, state_out)
    st = _call(lib.leet_attn_forward_static, dev, _ptr(q), _ptr(k), _ptr(v), _ptr(gamma), _ptr(out), _ptr(state_in),
               _ptr(state_out), int(segments), B, H, N, d, _dtype_code(q))
    if st != LEET_OK:
        raise LeetAttnError(st, "leet_attn_forward_static")
    return out


def leet_attn_forward_recurrent_rd(q, k, v, gamma: Optional[torch.Tensor], out: Optional[torch.Tensor] = None,
                                   state_in: Optional[torch.Tensor] = None,
                                   state_out: Optional[torch.Tensor] = None,
                                   mask: int = LEET_MASK_DECAY) -> torch.Tensor:
    """Row-based prefill with q, k of width r and v, out of width dv."""
    if out is None:
        out = _new_out(v, torch.float32)
    B, H, N, r, dv = _check_rd(q, k, v, gamma, out, False)
    _check_states_rd(B, H, r, dv, state_in=state_in, state_out=state_out)
    dev = _check_dev(q, k, v, gamma, out, state_in, state_out)
    st = _call(lib.leet_attn_forward_recurrent_rd, dev, _ptr(q), _ptr(k), _ptr(v), _ptr(gamma), _ptr(out),
               _ptr(state_in), _ptr(state_out), B, H, N, r, dv, _dtype_code(q), int(mask))
    if st != LEET_OK:
        raise LeetAttnError(st, "leet_attn_forward_recurrent_rd")
    return out


def leet_attn_forward_fleet(q, k, v, gamma: Optional[torch.Tensor], out: Optional[torch.Tensor] = None,
                            state_in: Optional[torch.Tensor] = None,
                            state_out: Optional[torch.Tensor] = None,
                            mask: int = LEET_MASK_DECAY) -> torch.Tensor:
    """FleetAttention prefill (rank-sum of discounted cumulative sums); q, k [B, H, N, r], v [B, H, N, dv]."""
    if out is None:
        out = _new_out(v, torch.float32)
    B, H, N, r, dv = _check_rd(q, k, v, gamma, out, False)
    _check_states_rd(B, H, r, dv, state_in=state_in, state_out=state_out)
    dev = _check_dev(q, k, v, gamma, out, state_in, state_out)
    st = _call(lib.leet_attn_forward_fleet, dev, _ptr(q), _ptr(k), _ptr(v), _ptr(gamma), _ptr(out), _ptr(state_in),
               _ptr(state_out), B, H, N, r, dv, _dtype_code(q), int(mask))
    if st != LEET_OK:
        raise LeetAttnError(st, "leet_attn_forward_fleet")
    return out


def leet_attn_decode_step_rd(q, k, v, gamma: Optional[torch.Tensor], state, out: Optional[torch.Tensor] = None,
                             mask: int = LEET_MASK_DECAY, store: Optional[int] = None) -> torch.Tensor:
    """One decode step with q, k [B, H, r], v [B, H, dv] and state [B, H, r, dv] (updated in place).

    ``store`` (a DECODE_STORE_* value) routes the call through ``leet_attn_decode_step_v3``, which takes
    the state store policy per call."""
    if q.dim() != 3 or q.shape != k.shape or v.dim() != 3 or q.shape[:2] != v.shape[:2]:
        raise ValueError("q, k must share one [B, H, r] shape and v be [B, H, dv]")
    if k.dtype != q.dtype or v.dtype != q.dtype:
        raise TypeError("q, k, v must share one dtype")
    B, H, r = q.shape
    dv = v.shape[2]
    if out is None:
        out = _new_out(v, torch.float32)
    if gamma is not None and (gamma.dtype != torch.float32 or gamma.numel() != H):
        raise ValueError("gamma must be float32 with one value per head")
    _check_states_rd(B, H, r, dv, state=state)
    if out.dtype != torch.float32 or tuple(out.shape) != (B, H, dv):
        raise ValueError("out must be float32 [B, H, dv]")
    dev = _check_dev(q, k, v, gamma, state, out)
    if store is None:
        st = _call(lib.leet_attn_decode_step_rd, dev, _ptr(q), _ptr(k), _ptr(v), _ptr(gamma), _ptr(state), _ptr(out),
                   B, H, r, dv, _dtype_code(q), int(mask))
    else:
        st = _call(lib.leet_attn_decode_step_v3, dev, _ptr(q), _ptr(k), _ptr(v), _ptr(gamma), _ptr(state), _ptr(out),
                   B, H, r, dv, _dtype_code(q), int(mask), int(store))
    if st != LEET_OK:
        raise LeetAttnError(st, "leet_attn_decode_step_v3" if store is not None else "leet_attn_decode_step_rd")
    return out


# ---- operators beside the attention -------------------------------------------------------------------------------
# Their tensors may have any strides but for the last dimension's, which must be 1, and outputs that the caller does not
# bring are dense.  A workspace that the caller does not bring comes from torch's allocator, on the current stream: it
# belongs to this call alone, also while a graph is captured.
# Like the attention's calls they record nothing for autograd: outputs require no gradient even where inputs do.  Who
# trains with them puts a call and its _backward (the rotation's: the transposed rotation) into a torch.autograd.Function.

def _on(*tensors: Optional[torch.Tensor]) -> int:
    """Index of the one device of all tensors that are there."""
    index = None
    for t in tensors:
        if t is None:
            continue
        at = t.get_device()  # -1 for host memory
        if at < 0:
            raise ValueError("all tensors must be GPU tensors")
        if index is None:
            index = at
        elif at != index:
            raise ValueError("all tensors must be on one device")
    return index


def _call_on(index: int, fn, *args) -> int:
    """fn(*args, the current stream of device ``index``) with that device current; returns the status."""
    if index == torch.cuda.current_device():
        return fn(*args, _raw_stream(index))
    with torch.cuda.device(index):
        return fn(*args, _raw_stream(index))


def _heads_view(t: torch.Tensor, name: str, shape, dtype: torch.dtype) -> bytes:
    """``t`` as a leet_attn_heads; ``shape`` [B, H, N, d] and ``dtype`` are what it has to have."""
    if t.shape != shape:
        raise ValueError(f"{name} must have the shape {list(shape)}")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}")
    b, h, n, e = t.stride()
    if e != 1 and t.shape[3] > 1:
        raise ValueError(f"{name}: the elements of a head row must be adjacent")
    return _pack_heads(t.data_ptr(), b, h, n)


def _rows_view(t: torch.Tensor, name: str, shape, dtype: torch.dtype) -> bytes:
    """``t`` as a leet_attn_rows; ``shape`` [B, N, C] or [B, C] and ``dtype`` are what it has to have."""
    if t.shape != shape:
        raise ValueError(f"{name} must have the shape {list(shape)}")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}")
    strides = t.stride()
    if strides[-1] != 1 and t.shape[-1] > 1:
        raise ValueError(f"{name}: the channels of a row must be adjacent")
    return _pack_rows(t.data_ptr(), strides[0], strides[1] if len(strides) == 3 else 0)


def _scratch(nbytes: int, workspace: Optional[torch.Tensor], index: int):
    """(pointer, bytes, tensor to keep until the launch) of a call's workspace."""
    if workspace is None:
        if not nbytes:
            return None, 0, None
        workspace = torch.empty(nbytes, dtype=torch.uint8, device=torch.device("cuda", index))
    elif workspace.dtype != torch.uint8 or not workspace.is_contiguous():
        raise TypeError("workspace must be a contiguous uint8 tensor")
    return workspace.data_ptr(), workspace.numel(), workspace


def rope_frequencies(rot: int, base: float = 10000.0, scaling: int = ROPE_SCALING_NONE, factor: float = 1.0,
                     trained: int = 0, slow: float = 1.0, fast: float = 32.0):
    """(float64 CPU tensor [rot / 2] of radians a position, scale): what the rotation takes as ``freq`` (on the GPU) and
    ``scale``.  ``factor``: how many times longer than ``trained`` tokens the contexts are; see leet_rope_scaling."""
    if rot < 2 or rot % 2:
        raise ValueError("rot must be even and positive")
    freq, scale = torch.empty(rot // 2, dtype=torch.float64), ctypes.c_float(1.0)
    st = lib.leet_attn_rope_frequencies(int(rot), float(base), int(scaling), float(factor), int(trained), float(slow),
                                        float(fast), freq.data_ptr(), ctypes.byref(scale))
    if st != LEET_OK:
        raise LeetAttnError(st, "leet_attn_rope_frequencies")
    return freq, scale.value


def _rotation(freq: torch.Tensor, layout: int, positions: Optional[torch.Tensor], pos0: int, scale: float, B: int,
              N: int) -> bytes:
    if freq.dtype != torch.float64 or freq.dim() != 1 or not freq.is_contiguous():
        raise ValueError("freq must be a contiguous float64 tensor [rot / 2]")
    at = stride = 0
    if positions is not None:
        if positions.dtype != torch.int64 or positions.shape not in ((N,), (B, N)):
            raise ValueError("positions must be int64 [N] or [B, N]")
        if N > 1 and positions.stride(-1) != 1:
            raise ValueError("positions of a sequence must be adjacent")
        at, stride = positions.data_ptr(), positions.stride(0) if positions.dim() == 2 else 0
    return _pack_rotation(freq.data_ptr(), 2 * freq.shape[0], layout, at, stride, pos0, scale)


def _sizes(where: str, *sizes: int) -> None:
    """Refuses sizes that would not arrive at the library as they are."""
    for n in sizes:
        if n > 0x7fffffff:
            raise LeetAttnError(LEET_ERR_TOO_LARGE, where)


def _heads_pair(q: torch.Tensor, k: Optional[torch.Tensor], where: str):
    """B, Hq, Hk, N, d of queries and keys."""
    if q.dim() != 4 or (k is not None and k.dim() != 4):
        raise ValueError("q and k must be [B, H, N, d]")
    B, Hq, N, d = q.shape
    Hk = 0
    if k is not None:
        if k.shape[0] != B or k.shape[2] != N or k.shape[3] != d:
            raise ValueError("q and k must agree in B, N and d")
        if k.dtype != q.dtype:
            raise TypeError("q and k must share one dtype")
        Hk = k.shape[1]
    _sizes(where, B, Hq, Hk, N, d)
    return B, Hq, Hk, N, d


def _new_dense(like: torch.Tensor) -> torch.Tensor:
    """A fresh dense tensor of ``like``'s shape, device and type."""
    if type(like) is _Tensor and like.is_contiguous():  # the least that torch has to look at
        return _empty_like(like)
    return _new_out(like, like.dtype)


def leet_attn_rope(q: torch.Tensor, freq: torch.Tensor, k: Optional[torch.Tensor] = None,
                   positions: Optional[torch.Tensor] = None, pos0: int = 0, layout: int = ROPE_HALF,
                   scale: float = 1.0, transposed: bool = False, out_q: Optional[torch.Tensor] = None,
                   out_k: Optional[torch.Tensor] = None):
    """Position rotation of q [B, Hq, N, d], and of k [B, Hk, N, d] in the same launch.

    The first ``2 * len(freq)`` elements of each row are rotated by the token's position (``positions`` or the token's
    number, plus ``pos0``).  ``transposed`` takes gradients of the outputs to gradients of the inputs; autograd sees
    nothing of the call.  Returns out_q, or (out_q, out_k); an output may be its input."""
    B, Hq, Hk, N, d = _heads_pair(q, k, "leet_attn_rope")
    if out_q is None:
        out_q = _new_dense(q)
    if k is None:
        if out_k is not None:
            raise ValueError("out_k without k")
    elif out_k is None:
        out_k = _new_dense(k)
    dev = _on(q, k, out_q, out_k, freq, positions)
    vk = ok = None
    if k is not None:
        vk, ok = _heads_view(k, "k", k.shape, q.dtype), _heads_view(out_k, "out_k", k.shape, q.dtype)
    st = _call_on(dev, lib.leet_attn_rope, _heads_view(q, "q", q.shape, q.dtype), _heads_view(out_q, "out_q", q.shape, q.dtype),
               Hq, vk, ok, Hk, _rotation(freq, layout, positions, pos0, scale, B, N), B, N, d, _dtype_code(q),
               1 if transposed else 0)
    if st != LEET_OK:
        raise LeetAttnError(st, "leet_attn_rope")
    return out_q if k is None else (out_q, out_k)


def _weights(q: torch.Tensor, wq: Optional[torch.Tensor], wk: Optional[torch.Tensor], d: int) -> int:
    """dtype code of the weights."""
    dtype = q.dtype
    for i, w in enumerate((wq, wk)):
        if w is None:
            continue
        if tuple(w.shape) != (d,) or not w.is_contiguous():
            raise ValueError("weights must be contiguous [d]")
        if i == 1 and wq is not None and w.dtype != wq.dtype:
            raise TypeError("q_weight and k_weight must share one dtype")
        dtype = w.dtype
    if dtype != q.dtype and dtype != torch.float32:
        raise TypeError("weights must have the type of q or be float32")
    return LEET_F32 if dtype == torch.float32 else _dtype_code(q)


def leet_attn_qk_norm_rope(q: torch.Tensor, k: torch.Tensor, q_weight: Optional[torch.Tensor],
                           k_weight: Optional[torch.Tensor], freq: torch.Tensor, eps: float = 1e-6,
                           positions: Optional[torch.Tensor] = None, pos0: int = 0, layout: int = ROPE_HALF,
                           scale: float = 1.0, out_q: Optional[torch.Tensor] = None,
                           out_k: Optional[torch.Tensor] = None):
    """Norm of every head of q [B, Hq, N, d] and k [B, Hk, N, d], times its weight [d], then the rotation of
    ``leet_attn_rope``, in one pass.  Returns (out_q, out_k): dense [B, H, N, d], as the prefill reads them, unless given;
    autograd sees nothing of it (``leet_attn_qk_norm_rope_backward``)."""
    B, Hq, Hk, N, d = _heads_pair(q, k, "leet_attn_qk_norm_rope")
    weight_dtype = _weights(q, q_weight, k_weight, d)
    if out_q is None:
        out_q = _new_dense(q)
    if out_k is None:
        out_k = _new_dense(k)
    dev = _on(q, k, out_q, out_k, q_weight, k_weight, freq, positions)
    st = _call_on(dev, lib.leet_attn_qk_norm_rope, _heads_view(q, "q", q.shape, q.dtype),
               _heads_view(out_q, "out_q", q.shape, q.dtype), Hq, _heads_view(k, "k", k.shape, q.dtype),
               _heads_view(out_k, "out_k", k.shape, q.dtype), Hk, _ptr(q_weight), _ptr(k_weight), weight_dtype, eps,
               _rotation(freq, layout, positions, pos0, scale, B, N), B, N, d, _dtype_code(q))
    if st != LEET_OK:
        raise LeetAttnError(st, "leet_attn_qk_norm_rope")
    return out_q, out_k


def qk_norm_rope_workspace_bytes(B: int, Hq: int, Hk: int, N: int, d: int) -> int:
    return int(lib.leet_attn_qk_norm_rope_workspace_bytes(B, Hq, Hk, N, d))


def leet_attn_qk_norm_rope_backward(dout_q: torch.Tensor, dout_k: torch.Tensor, q: torch.Tensor, k: torch.Tensor,
                                    q_weight: Optional[torch.Tensor], k_weight: Optional[torch.Tensor],
                                    freq: torch.Tensor, eps: float = 1e-6, positions: Optional[torch.Tensor] = None,
                                    pos0: int = 0, layout: int = ROPE_HALF, scale: float = 1.0,
                                    dx_q: Optional[torch.Tensor] = None, dx_k: Optional[torch.Tensor] = None,
                                    dq_weight: Optional[torch.Tensor] = None, dk_weight: Optional[torch.Tensor] = None,
                                    workspace: Optional[torch.Tensor] = None):
    """Gradients of ``leet_attn_qk_norm_rope``: (dx_q, dx_k, dq_weight, dk_weight) from those of its outputs and its
    inputs.  A weight that is None has the gradient None.  The attention here has no backward pass: where its q and k
    are what was normed, their gradients come from the caller's own."""
    B, Hq, Hk, N, d = _heads_pair(q, k, "leet_attn_qk_norm_rope_backward")
    weight_dtype = _weights(q, q_weight, k_weight, d)
    grads = []
    for w, g, name in ((q_weight, dq_weight, "dq_weight"), (k_weight, dk_weight, "dk_weight")):
        if w is None:
            if g is not None:
                raise ValueError(f"{name} without a weight")
        elif g is None:
            g = _new_dense(w)
        elif g.dtype != w.dtype or g.shape != w.shape or not g.is_contiguous():
            raise ValueError(f"{name} must be contiguous [d] of the weights' type")
        grads.append(g)
    dq_weight, dk_weight = grads
    if dx_q is None:
        dx_q = _new_dense(q)
    if dx_k is None:
        dx_k = _new_dense(k)
    dev = _on(dout_q, dout_k, q, k, dx_q, dx_k, q_weight, k_weight, dq_weight, dk_weight, freq, positions, workspace)
    need = 0
    if workspace is None and (dq_weight is not None or dk_weight is not None):
        need = qk_norm_rope_workspace_bytes(B, Hq, Hk, N, d)
    ws, ws_bytes, keep = _scratch(need, workspace, dev)
    t = q.dtype
    st = _call_on(dev, lib.leet_attn_qk_norm_rope_backward, _heads_view(dout_q, "dout_q", q.shape, t),
               _heads_view(q, "q", q.shape, t), _heads_view(dx_q, "dx_q", q.shape, t), Hq,
               _heads_view(dout_k, "dout_k", k.shape, t), _heads_view(k, "k", k.shape, t),
               _heads_view(dx_k, "dx_k", k.shape, t), Hk, _ptr(q_weight), _ptr(k_weight), _ptr(dq_weight),
               _ptr(dk_weight), weight_dtype, eps, _rotation(freq, layout, positions, pos0, scale, B, N), ws, ws_bytes,
               B, N, d, _dtype_code(q))
    if st != LEET_OK:
        raise LeetAttnError(st, "leet_attn_qk_norm_rope_backward")
    return dx_q, dx_k, dq_weight, dk_weight


def _gate_code(gate: torch.Tensor, x_dtype: torch.dtype) -> int:
    if gate.dtype != x_dtype and gate.dtype != torch.float32:
        raise TypeError("gate must have the type of x or be float32")
    return _dtype_code(gate)


def _scan_sequences(shape, offsets: Optional[torch.Tensor]) -> int:
    """Number of sequences of a [B, N, C] call."""
    if len(shape) != 3:
        raise ValueError("x must be [B, N, C]")
    if offsets is None:
        return shape[0]
    if offsets.dtype != torch.int32 or offsets.dim() != 1 or offsets.numel() < 1 or not offsets.is_contiguous():
        raise ValueError("offsets must be a contiguous int32 tensor [sequences + 1]")
    if shape[0] != 1:
        raise ValueError("packed sequences need B = 1")
    return offsets.numel() - 1


def _scan_states(S: int, C: int, **states) -> None:
    for name, s in states.items():
        if s is not None and (s.dtype != torch.float32 or tuple(s.shape) != (S, C) or not s.is_contiguous()):
            raise ValueError(f"{name} must be contiguous float32 [{S}, {C}]")


def gated_scan_workspace_bytes(B: int, N: int, C: int, backward: bool = False) -> int:
    return int(lib.leet_attn_gated_scan_workspace_bytes(B, N, C, 1 if backward else 0))


def leet_attn_gated_scan(x: torch.Tensor, gate: torch.Tensor, mode: int = GATE_LOG, out: Optional[torch.Tensor] = None,
                         state_in: Optional[torch.Tensor] = None, state_out: Optional[torch.Tensor] = None,
                         offsets: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None):
    """Gated linear recurrence ``h_t = a_t h_{t-1} + b_t`` in every channel of x, gate [B, N, C]; returns h in x's type.

    ``mode``: what the gate is (GATE_DECAY a itself, GATE_LOG its logarithm, GATE_SIGMOID its logit with b = (1 - a) x).
    States are float32 [B, C]; with ``offsets`` (int32 [S + 1], B = 1: packed sequences) [S, C].  Autograd sees nothing
    of it (``leet_attn_gated_scan_backward``)."""
    S = _scan_sequences(x.shape, offsets)
    B, N, C = x.shape
    _sizes("leet_attn_gated_scan", B, N, C, S)
    _scan_states(S, C, state_in=state_in, state_out=state_out)
    if out is None:
        out = _new_dense(x)
    dev = _on(x, gate, out, state_in, state_out, offsets, workspace)
    t = x.dtype
    need = gated_scan_workspace_bytes(B, N, C) if workspace is None else 0
    ws, ws_bytes, keep = _scratch(need, workspace, dev)
    st = _call_on(dev, lib.leet_attn_gated_scan, _rows_view(x, "x", x.shape, t), _rows_view(gate, "gate", x.shape, gate.dtype),
               _rows_view(out, "out", x.shape, t), _ptr(state_in), _ptr(state_out), _ptr(offsets), S, ws, ws_bytes,
               B, N, C, _dtype_code(x), _gate_code(gate, t), mode)
    if st != LEET_OK:
        raise LeetAttnError(st, "leet_attn_gated_scan")
    return out


def leet_attn_gated_scan_backward(dh: torch.Tensor, x: Optional[torch.Tensor], gate: torch.Tensor, h: torch.Tensor,
                                  mode: int = GATE_LOG, dx: Optional[torch.Tensor] = None,
                                  dgate: Optional[torch.Tensor] = None, state_in: Optional[torch.Tensor] = None,
                                  dstate_out: Optional[torch.Tensor] = None, dstate_in: Optional[torch.Tensor] = None,
                                  offsets: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None):
    """Gradients of ``leet_attn_gated_scan``: (dx, dgate), and dstate_in where given.

    ``h`` is the forward call's output, ``dh`` its gradient, ``dstate_out`` that of state_out (None: zero); ``x`` is
    read with GATE_SIGMOID only and may be None otherwise."""
    S = _scan_sequences(h.shape, offsets)
    B, N, C = h.shape
    _sizes("leet_attn_gated_scan_backward", B, N, C, S)
    _scan_states(S, C, state_in=state_in, dstate_out=dstate_out, dstate_in=dstate_in)
    if mode == GATE_SIGMOID and x is None:
        raise ValueError("GATE_SIGMOID needs x")
    if dx is None:
        dx = _new_dense(h)
    if dgate is None:
        dgate = _new_dense(gate)
    dev = _on(dh, x, gate, h, dx, dgate, state_in, dstate_out, dstate_in, offsets, workspace)
    t, g = h.dtype, gate.dtype
    need = gated_scan_workspace_bytes(B, N, C, True) if workspace is None else 0
    ws, ws_bytes, keep = _scratch(need, workspace, dev)
    st = _call_on(dev, lib.leet_attn_gated_scan_backward, _rows_view(dh, "dh", h.shape, t),
               None if x is None else _rows_view(x, "x", h.shape, t), _rows_view(gate, "gate", h.shape, g),
               _rows_view(h, "h", h.shape, t), _rows_view(dx, "dx", h.shape, t), _rows_view(dgate, "dgate", h.shape, g),
               _ptr(state_in), _ptr(dstate_out), _ptr(dstate_in), _ptr(offsets), S, ws, ws_bytes, B, N, C,
               _dtype_code(h), _gate_code(gate, t), mode)
    if st != LEET_OK:
        raise LeetAttnError(st, "leet_attn_gated_scan_backward")
    return dx, dgate


def leet_attn_gated_scan_step(x: torch.Tensor, gate: torch.Tensor, state: torch.Tensor, mode: int = GATE_LOG,
                              out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """One token of every sequence: x, gate [B, C]; ``state`` (float32 [B, C]) is updated in place, ``out`` is it in x's type."""
    if x.dim() != 2:
        raise ValueError("x must be [B, C]")
    B, C = x.shape
    _sizes("leet_attn_gated_scan_step", B, C)
    _scan_states(B, C, state=state)
    if out is None:
        out = _new_dense(x)
    dev = _on(x, gate, out, state)
    st = _call_on(dev, lib.leet_attn_gated_scan_step, _rows_view(x, "x", x.shape, x.dtype),
               _rows_view(gate, "gate", x.shape, gate.dtype), _rows_view(out, "out", x.shape, x.dtype), _ptr(state), B, C,
               _dtype_code(x), _gate_code(gate, x.dtype), mode)
    if st != LEET_OK:
        raise LeetAttnError(st, "leet_attn_gated_scan_step")
    return out
