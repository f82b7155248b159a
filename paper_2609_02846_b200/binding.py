"""ctypes binding of ``libue5m3.so``: same names as the C ABI, argument marshalling only.

Every function takes torch CUDA tensors, passes their device pointers and the current CUDA stream
to the library and returns torch tensors that wrap the caller-visible outputs.  Nothing is computed
here.  The library is required: a missing or unloadable ``libue5m3.so`` raises at first use.
"""
from __future__ import annotations

import ctypes as C
import math
import os
from array import array
from dataclasses import dataclass
from typing import Optional

import torch

F32, BF16 = 0, 1
LAYOUT_1D_ROW, LAYOUT_1D_COL, LAYOUT_2D = 0, 1, 2
BLOCK_32 = 0x100            # OR into a layout: the block-size control (one scale per 32 elements)
ROUND_RNE, ROUND_SR = 0, 1
SCALES_ROWMAJOR, SCALES_TILED = 0, 1
SCALE_1D, SCALE_1D_TILED, SCALE_2D = 0, 1, 2
FPROP, DGRAD, WGRAD = 0, 1, 2

SYMBOLS = ("ue5m3_sample_amax", "ue5m3_quantize", "ue5m3_quantize_dual", "ue5m3_quantize_current", "ue5m3_gemm",
           "ue5m3_gemm_probe_matched", "ue5m3_gemm_stall_selftest", "ue5m3_scales_bytes", "ue5m3_unswizzle_scales",
           "ue5m3_last_device_status", "ue5m3_status_string", "ue5m3_layer_norm", "ue5m3_layer_norm_backward_workspace_bytes",
           "ue5m3_layer_norm_backward", "ue5m3_dropout_add", "ue5m3_attention_workspace_bytes", "ue5m3_attention",
           "ue5m3_attention_backward_workspace_bytes", "ue5m3_attention_backward", "ue5m3_block_stall_selftest", "ue5m3_rotary",
           "ue5m3_qk_norm_rotary", "ue5m3_qk_norm_rotary_backward_workspace_bytes", "ue5m3_qk_norm_rotary_backward", "ue5m3_adamw",
           "ue5m3_attention_sinks", "ue5m3_attention_sinks_backward_workspace_bytes", "ue5m3_attention_sinks_backward")

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libue5m3.so")
_lib = None


class _Heads(C.Structure):                  # ue5m3_heads
    _fields_ = [("data", C.c_void_p), ("batch_stride", C.c_int64), ("token_stride", C.c_int64), ("head_stride", C.c_int64)]


class _AttentionShape(C.Structure):         # ue5m3_attention_shape
    _fields_ = [("batch", C.c_int64), ("q_len", C.c_int64), ("k_len", C.c_int64), ("heads", C.c_int64), ("kv_heads", C.c_int64),
                ("head_dim", C.c_int64), ("window_left", C.c_int64), ("k_lens", C.c_void_p), ("scale", C.c_float), ("dtype", C.c_int),
                ("causal", C.c_int)]


class _RotaryShape(C.Structure):            # ue5m3_rotary_shape
    _fields_ = [("batch", C.c_int64), ("tokens", C.c_int64), ("heads", C.c_int64), ("kv_heads", C.c_int64), ("head_dim", C.c_int64),
                ("rotary_dim", C.c_int64), ("frequencies", C.c_void_p), ("positions", C.c_void_p), ("position_stride", C.c_int64),
                ("first_position", C.c_int64), ("position_bytes", C.c_int), ("interleaved", C.c_int), ("amplitude", C.c_float),
                ("dtype", C.c_int)]


class _AdamwStep(C.Structure):              # ue5m3_adamw_step
    _fields_ = [("step", C.c_int64), ("lr", C.c_double), ("beta1", C.c_double), ("beta2", C.c_double), ("eps", C.c_double),
                ("weight_decay", C.c_double), ("grad_scale", C.c_void_p), ("clock", C.c_void_p), ("seed", C.c_uint64),
                ("state_bits", C.c_int)]


class Ue5m3Error(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)}")


def library_path() -> str:
    return _LIB_PATH


def _load() -> C.CDLL:
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise FileNotFoundError(
                f"{_LIB_PATH} is missing: build it with `python -m paper_2609_02846_b200.build` "
                "(there is no fallback implementation)")
        L = C.CDLL(_LIB_PATH)
        i64, u64, vp, ci, f32 = C.c_int64, C.c_uint64, C.c_void_p, C.c_int, C.c_float
        L.ue5m3_sample_amax.restype = ci
        L.ue5m3_sample_amax.argtypes = [vp, ci, i64, i64, i64, vp, vp]
        L.ue5m3_quantize.restype = ci
        L.ue5m3_quantize.argtypes = [vp, ci, i64, i64, i64, ci, ci, vp, f32, u64, vp, vp, vp, vp, vp, vp, ci, vp]
        L.ue5m3_quantize_current.restype = ci
        L.ue5m3_quantize_current.argtypes = [vp, ci, i64, i64, i64, ci, ci, vp, f32, u64, vp, vp, vp, vp, vp, vp, ci, vp]
        L.ue5m3_quantize_dual.restype = ci
        L.ue5m3_quantize_dual.argtypes = [vp, ci, i64, i64, i64, ci, vp, f32, f32, u64, u64, vp, vp, vp, vp, vp, vp, vp, vp, ci, vp]
        L.ue5m3_gemm.restype = ci
        L.ue5m3_gemm.argtypes = [ci, i64, i64, i64, vp, vp, ci, vp, vp, vp, ci, vp, vp, ci, i64, vp]
        L.ue5m3_gemm_static.restype = ci
        L.ue5m3_gemm_static.argtypes = [ci, i64, i64, i64, vp, vp, ci, vp, vp, vp, ci, vp, vp, ci, i64, vp]
        L.ue5m3_gemm_fp16.restype = ci
        L.ue5m3_gemm_fp16.argtypes = [ci, i64, i64, i64, vp, vp, ci, vp, vp, vp, ci, vp, vp, ci, i64, vp]
        L.ue5m3_gemm_native_workspace_bytes.restype = C.c_size_t
        L.ue5m3_gemm_native_workspace_bytes.argtypes = [i64, i64, i64, ci, ci]
        L.ue5m3_gemm_native.restype = ci
        L.ue5m3_gemm_native.argtypes = [ci, i64, i64, i64, vp, vp, ci, vp, vp, vp, ci, vp, vp, ci, i64, vp, vp]
        L.ue5m3_gemm_probe_matched.restype = ci
        L.ue5m3_gemm_probe_matched.argtypes = [ci, i64, i64, i64, vp, vp, ci, vp, vp, vp, ci, vp, ci, ci, vp, ci, i64, vp]
        L.ue5m3_gemm_stall_selftest.restype = ci
        L.ue5m3_gemm_stall_selftest.argtypes = [ci, i64, i64, i64, vp, vp, ci, vp, vp, vp, ci, vp, vp, ci, i64, i64, vp]
        L.ue5m3_scales_bytes.restype = C.c_size_t
        L.ue5m3_scales_bytes.argtypes = [i64, i64, ci, ci]
        L.ue5m3_unswizzle_scales.restype = ci
        L.ue5m3_unswizzle_scales.argtypes = [vp, vp, i64, i64, vp]
        L.ue5m3_last_device_status.restype = ci
        L.ue5m3_last_device_status.argtypes = []
        L.ue5m3_layer_norm.restype = ci
        L.ue5m3_layer_norm.argtypes = [vp, ci, i64, i64, i64, vp, vp, ci, f32, vp, i64, vp, vp, vp]
        L.ue5m3_layer_norm_backward_workspace_bytes.restype = C.c_size_t
        L.ue5m3_layer_norm_backward_workspace_bytes.argtypes = [i64, i64]
        L.ue5m3_layer_norm_backward.restype = ci
        L.ue5m3_layer_norm_backward.argtypes = [vp, i64, vp, ci, i64, i64, i64, vp, ci, vp, vp, vp, i64, vp, vp, vp, vp]
        L.ue5m3_dropout_add.restype = ci
        L.ue5m3_dropout_add.argtypes = [vp, i64, vp, i64, ci, i64, i64, f32, u64, vp, i64, vp]
        shape, heads = C.POINTER(_AttentionShape), C.POINTER(_Heads)
        L.ue5m3_attention.restype = ci
        L.ue5m3_attention.argtypes = [shape, heads, heads, heads, heads, vp, vp, vp]
        L.ue5m3_attention_workspace_bytes.restype = C.c_size_t
        L.ue5m3_attention_workspace_bytes.argtypes = [shape]
        L.ue5m3_attention_backward_workspace_bytes.restype = C.c_size_t
        L.ue5m3_attention_backward_workspace_bytes.argtypes = [shape]
        L.ue5m3_attention_backward.restype = ci
        L.ue5m3_attention_backward.argtypes = [shape, heads, heads, heads, heads, heads, vp, heads, heads, heads, vp, vp]
        L.ue5m3_attention_sinks.restype = ci
        L.ue5m3_attention_sinks.argtypes = [shape, i64, heads, heads, heads, heads, vp, vp, vp]
        L.ue5m3_attention_sinks_backward_workspace_bytes.restype = C.c_size_t
        L.ue5m3_attention_sinks_backward_workspace_bytes.argtypes = [shape, i64]
        L.ue5m3_attention_sinks_backward.restype = ci
        L.ue5m3_attention_sinks_backward.argtypes = [shape, i64, heads, heads, heads, heads, heads, vp, heads, heads, heads, vp, vp]
        turn = C.POINTER(_RotaryShape)
        L.ue5m3_rotary.restype = ci
        L.ue5m3_rotary.argtypes = [turn, ci, heads, heads, heads, heads, vp]
        L.ue5m3_qk_norm_rotary.restype = ci
        L.ue5m3_qk_norm_rotary.argtypes = [turn, heads, heads, vp, vp, ci, f32, heads, heads, vp]
        L.ue5m3_qk_norm_rotary_backward_workspace_bytes.restype = C.c_size_t
        L.ue5m3_qk_norm_rotary_backward_workspace_bytes.argtypes = [turn]
        L.ue5m3_qk_norm_rotary_backward.restype = ci
        L.ue5m3_qk_norm_rotary_backward.argtypes = [turn, heads, heads, heads, heads, vp, vp, ci, f32, heads, heads, vp, vp, vp, vp]
        L.ue5m3_adamw.restype = ci
        L.ue5m3_adamw.argtypes = [vp, i64, C.POINTER(_AdamwStep), vp]
        L.ue5m3_block_stall_selftest.restype = ci
        L.ue5m3_block_stall_selftest.argtypes = [ci, vp, C.c_size_t, i64, vp]
        L.ue5m3_status_string.restype = C.c_char_p
        L.ue5m3_status_string.argtypes = [ci]
        _lib = L
    return _lib


def status_string(status: int) -> str:
    return _load().ue5m3_status_string(int(status)).decode()


def _check(status: int, where: str) -> None:
    if status != 0:
        raise Ue5m3Error(status, where)


def _dtype_code_of(dtype: torch.dtype) -> int:
    if dtype == torch.float32:
        return F32
    if dtype == torch.bfloat16:
        return BF16
    raise TypeError(f"unsupported dtype {dtype}: the library takes float32 or bfloat16")


def _dtype_code(t: torch.Tensor) -> int:
    return _dtype_code_of(t.dtype)


def _dev_ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("the library takes device tensors only")
    return C.c_void_p(t.data_ptr())


def _stream(t: torch.Tensor):
    return C.c_void_p(torch.cuda.current_stream(t.device).cuda_stream)


def _matrix(x: torch.Tensor):
    if x.dim() != 2 or x.stride(1) != 1:
        raise ValueError("expected a 2-D tensor whose rows are contiguous")
    return x.shape[0], x.shape[1], x.stride(0)


# ---------------------------------------------------------------------------------------------
def sample_amax(x: torch.Tensor, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """max |x| as a 1-element float32 device tensor (no host synchronisation)."""
    rows, cols, ld = _matrix(x)
    if out is None:
        out = torch.empty(1, dtype=torch.float32, device=x.device)
    with torch.cuda.device(x.device):
        _check(_load().ue5m3_sample_amax(_dev_ptr(x), _dtype_code(x), rows, cols, ld, _dev_ptr(out), _stream(x)),
               "ue5m3_sample_amax")
    return out


def scales_bytes(rows: int, cols: int, layout: int, scale_layout: int = SCALES_ROWMAJOR) -> int:
    return int(_load().ue5m3_scales_bytes(rows, cols, layout, scale_layout))


@dataclass
class QuantizedOperand:
    """A K-major GEMM operand [R, Kc]: packed E2M1 payload, UE5M3 scales, tensor decode factor."""
    payload: torch.Tensor                 # uint8 [R, Kc/2]
    scales: torch.Tensor                  # uint8, row-major [R, Kc/16] / [R/16, Kc/16], or flat tiled buffer
    decode: torch.Tensor                  # float32 [1]
    scale_mode: int                       # SCALE_1D, SCALE_1D_TILED or SCALE_2D
    payload_t: Optional[torch.Tensor] = None   # 2D only: the same codes for the transpose [Kc, R/2]
    scales_t: Optional[torch.Tensor] = None    # 2D only: [Kc/16, R/16]

    @property
    def R(self) -> int:
        return self.payload.shape[0]

    @property
    def Kc(self) -> int:
        return self.payload.shape[1] * 2

    def transposed(self) -> "QuantizedOperand":
        if self.payload_t is None:
            raise ValueError("this operand was quantized without its transposed copy")
        return QuantizedOperand(self.payload_t, self.scales_t, self.decode, SCALE_2D, self.payload, self.scales)


def _alloc_operand(x: torch.Tensor, layout: int, want_transpose: bool, scale_layout: int) -> QuantizedOperand:
    """Output buffers of one quantization of `x`."""
    rows, cols, _ = _matrix(x)
    dev = x.device
    u8 = dict(dtype=torch.uint8, device=dev)
    nbytes = scales_bytes(rows, cols, layout, scale_layout)
    if nbytes == 0:
        _check(2, "ue5m3_quantize (rows and cols must be positive multiples of 16)")
    if layout == LAYOUT_1D_ROW:
        payload = torch.empty((rows, cols // 2), **u8)
        sshape = (rows, cols // 16)
    elif layout == LAYOUT_1D_COL:
        payload = torch.empty((cols, rows // 2), **u8)
        sshape = (cols, rows // 16)
    else:
        payload = torch.empty((rows, cols // 2), **u8)
        sshape = (rows // 16, cols // 16)
    scales = torch.zeros(nbytes, **u8) if scale_layout == SCALES_TILED else torch.empty(sshape, **u8)
    payload_t = scales_t = None
    if layout == LAYOUT_2D and want_transpose:
        payload_t = torch.empty((cols, rows // 2), **u8)
        scales_t = torch.empty((cols // 16, rows // 16), **u8)
    mode = SCALE_2D if layout == LAYOUT_2D else (SCALE_1D_TILED if scale_layout == SCALES_TILED else SCALE_1D)
    return QuantizedOperand(payload, scales, torch.empty(1, dtype=torch.float32, device=dev), mode, payload_t, scales_t)


def quantize(x: torch.Tensor, layout: int, rounding: int, amax_held: torch.Tensor, target_T: float = 448.0,
             seed: int = 0, want_transpose: bool = False, stats: Optional[torch.Tensor] = None,
             scale_layout: int = SCALES_ROWMAJOR, out: Optional[QuantizedOperand] = None,
             block: int = 16) -> QuantizedOperand:
    """ue5m3_quantize.  `stats` (int64[4], device) is accumulated into when given.  `block = 32` selects the
    block-size control (one scale per 32 elements, stored in every 16-element slot it covers)."""
    if block not in (16, 32):
        raise ValueError("block must be 16 or 32")
    rows, cols, ld = _matrix(x)
    dev = x.device
    if out is None:
        out = _alloc_operand(x, layout, want_transpose, scale_layout)
    if stats is not None and (stats.dtype != torch.int64 or stats.numel() != 4):
        raise ValueError("stats must be an int64 tensor with 4 elements")
    with torch.cuda.device(dev):
        _check(_load().ue5m3_quantize(
            _dev_ptr(x), _dtype_code(x), rows, cols, ld, layout | (BLOCK_32 if block == 32 else 0), rounding,
            _dev_ptr(amax_held), C.c_float(target_T), C.c_uint64(int(seed) & (2 ** 64 - 1)),
            _dev_ptr(out.payload), _dev_ptr(out.scales), _dev_ptr(out.payload_t), _dev_ptr(out.scales_t),
            _dev_ptr(out.decode), _dev_ptr(stats), scale_layout, _stream(x)), "ue5m3_quantize")
    return out


def quantize_current(x: torch.Tensor, layout: int, rounding: int, target_T: float = 448.0, seed: int = 0,
                     want_transpose: bool = False, stats: Optional[torch.Tensor] = None,
                     scale_layout: int = SCALES_ROWMAJOR, amax_out: Optional[torch.Tensor] = None,
                     out: Optional[QuantizedOperand] = None, block: int = 16):
    """ue5m3_quantize_current: the per-batch (D = 1) reference policy.  Returns (operand, amax) where amax is the
    tensor maximum the operand was scaled by (device float32[1]).  `layout` is one of the three LAYOUT_* values;
    `block = 32` selects the block-size control as in `quantize`."""
    if block not in (16, 32):
        raise ValueError("block must be 16 or 32")
    if layout not in (LAYOUT_1D_ROW, LAYOUT_1D_COL, LAYOUT_2D):
        raise ValueError("layout must be LAYOUT_1D_ROW, LAYOUT_1D_COL or LAYOUT_2D (pass block=32 for the block-size control)")
    if amax_out is None:
        amax_out = torch.empty(1, dtype=torch.float32, device=x.device)
    if out is None:
        out = _alloc_operand(x, layout, want_transpose, scale_layout)
    rows, cols, ld = _matrix(x)
    with torch.cuda.device(x.device):
        _check(_load().ue5m3_quantize_current(
            _dev_ptr(x), _dtype_code(x), rows, cols, ld, layout | (BLOCK_32 if block == 32 else 0), rounding, _dev_ptr(amax_out),
            C.c_float(target_T), C.c_uint64(int(seed) & (2 ** 64 - 1)),
            _dev_ptr(out.payload), _dev_ptr(out.scales), _dev_ptr(out.payload_t), _dev_ptr(out.scales_t),
            _dev_ptr(out.decode), _dev_ptr(stats), scale_layout, _stream(x)), "ue5m3_quantize_current")
    return out, amax_out


def quantize_dual(x: torch.Tensor, rounding: int, amax_held: torch.Tensor, target_T_row: float = 448.0,
                  target_T_col: float = 448.0, seed_row: int = 0, seed_col: int = 0,
                  stats_row: Optional[torch.Tensor] = None, stats_col: Optional[torch.Tensor] = None,
                  scale_layout: int = SCALES_ROWMAJOR,
                  out: Optional[tuple] = None) -> tuple:
    """ue5m3_quantize_dual: the 1D_ROW and the 1D_COL quantization of `x` from one read.  Returns (row, col)
    operands, each identical to what `quantize` produces for that layout, target and seed."""
    rows, cols, ld = _matrix(x)
    dev = x.device
    u8 = dict(dtype=torch.uint8, device=dev)
    if out is None:
        ops = []
        for layout, (R, K) in ((LAYOUT_1D_ROW, (rows, cols)), (LAYOUT_1D_COL, (cols, rows))):
            nbytes = scales_bytes(rows, cols, layout, scale_layout)
            if nbytes == 0:
                _check(2, "ue5m3_quantize_dual (rows and cols must be positive multiples of 16)")
            scales = torch.zeros(nbytes, **u8) if scale_layout == SCALES_TILED else torch.empty((R, K // 16), **u8)
            ops.append(QuantizedOperand(torch.empty((R, K // 2), **u8), scales, torch.empty(1, dtype=torch.float32, device=dev),
                                        SCALE_1D_TILED if scale_layout == SCALES_TILED else SCALE_1D))
        out = tuple(ops)
    row, col = out
    for st in (stats_row, stats_col):
        if st is not None and (st.dtype != torch.int64 or st.numel() != 4):
            raise ValueError("stats must be int64 tensors with 4 elements")
    with torch.cuda.device(dev):
        _check(_load().ue5m3_quantize_dual(
            _dev_ptr(x), _dtype_code(x), rows, cols, ld, rounding, _dev_ptr(amax_held),
            C.c_float(target_T_row), C.c_float(target_T_col),
            C.c_uint64(int(seed_row) & (2 ** 64 - 1)), C.c_uint64(int(seed_col) & (2 ** 64 - 1)),
            _dev_ptr(row.payload), _dev_ptr(row.scales), _dev_ptr(col.payload), _dev_ptr(col.scales),
            _dev_ptr(row.decode), _dev_ptr(col.decode), _dev_ptr(stats_row), _dev_ptr(stats_col),
            scale_layout, _stream(x)), "ue5m3_quantize_dual")
    return out


def unswizzle_scales(tiled: torch.Tensor, R: int, kblocks: int) -> torch.Tensor:
    out = torch.empty((R, kblocks), dtype=torch.uint8, device=tiled.device)
    with torch.cuda.device(tiled.device):
        _check(_load().ue5m3_unswizzle_scales(_dev_ptr(tiled), _dev_ptr(out), R, kblocks, _stream(tiled)),
               "ue5m3_unswizzle_scales")
    return out


def gemm(op: int, a: QuantizedOperand, b: QuantizedOperand, out_dtype: torch.dtype = torch.bfloat16,
         out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """C[Mo, No] = d_A d_B * A[Mo, Kc] B[No, Kc]^T on the quantized operands (ue5m3_gemm)."""
    Mo, No, Kc = a.R, b.R, a.Kc
    if b.Kc != Kc:
        raise ValueError(f"contraction sizes differ: {Kc} vs {b.Kc}")
    if out is None:
        out = torch.empty((Mo, No), dtype=out_dtype, device=a.payload.device)
    with torch.cuda.device(out.device):
        _check(_load().ue5m3_gemm(op, Mo, No, Kc,
                                  _dev_ptr(a.payload), _dev_ptr(a.scales), a.scale_mode, _dev_ptr(a.decode),
                                  _dev_ptr(b.payload), _dev_ptr(b.scales), b.scale_mode, _dev_ptr(b.decode),
                                  _dev_ptr(out), _dtype_code(out), out.stride(0), _stream(out)), "ue5m3_gemm")
    return out


def gemm_static(op: int, a: QuantizedOperand, b: QuantizedOperand, out_dtype: torch.dtype = torch.bfloat16,
                out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """`gemm` with the library's file-scope workspace instead of its allocated one (ue5m3_gemm_static): nothing is
    allocated by the call; calls that may overlap in time must be ordered by the caller."""
    Mo, No, Kc = a.R, b.R, a.Kc
    if b.Kc != Kc:
        raise ValueError(f"contraction sizes differ: {Kc} vs {b.Kc}")
    if out is None:
        out = torch.empty((Mo, No), dtype=out_dtype, device=a.payload.device)
    with torch.cuda.device(out.device):
        _check(_load().ue5m3_gemm_static(op, Mo, No, Kc,
                                         _dev_ptr(a.payload), _dev_ptr(a.scales), a.scale_mode, _dev_ptr(a.decode),
                                         _dev_ptr(b.payload), _dev_ptr(b.scales), b.scale_mode, _dev_ptr(b.decode),
                                         _dev_ptr(out), _dtype_code(out), out.stride(0), _stream(out)), "ue5m3_gemm_static")
    return out


def scale_window(cmin: int, cmax: int) -> Optional[int]:
    """The rule by which ue5m3_gemm decides between its two kernels, restated on the host: the shift k with
    8 <= c - 8k <= 126 for all non-zero codes cmin..cmax of a scale row (then UE5M3 code c and UE4M3 code c - 8k denote
    values that differ by exactly 2^(k - 8)), or None when the row has no such window."""
    if cmin < 8 or cmax > 0xF7 or cmin > cmax:
        return None
    k_lo = (cmax - 126 + 7) >> 3 if cmax > 126 else 0   # the smallest shift that brings cmax down to 126
    k_hi = (cmin - 8) >> 3                              # the largest one that keeps cmin at 8 or above
    if k_lo > k_hi:
        return None
    return 2 if k_lo <= 2 <= k_hi else k_lo             # rows agree on 2 where they can


def gemm_fp16(op: int, a: QuantizedOperand, b: QuantizedOperand, out_dtype: torch.dtype = torch.bfloat16,
              out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The product of `gemm`, always through the FP16 reconstruction kernel (ue5m3_gemm_fp16)."""
    Mo, No, Kc = a.R, b.R, a.Kc
    if b.Kc != Kc:
        raise ValueError(f"contraction sizes differ: {Kc} vs {b.Kc}")
    if out is None:
        out = torch.empty((Mo, No), dtype=out_dtype, device=a.payload.device)
    with torch.cuda.device(out.device):
        _check(_load().ue5m3_gemm_fp16(op, Mo, No, Kc,
                                       _dev_ptr(a.payload), _dev_ptr(a.scales), a.scale_mode, _dev_ptr(a.decode),
                                       _dev_ptr(b.payload), _dev_ptr(b.scales), b.scale_mode, _dev_ptr(b.decode),
                                       _dev_ptr(out), _dtype_code(out), out.stride(0), _stream(out)), "ue5m3_gemm_fp16")
    return out


def gemm_native_workspace(a: QuantizedOperand, b: QuantizedOperand) -> torch.Tensor:
    """A workspace of the size ue5m3_gemm_native wants for these operands (uint8, device)."""
    n = _load().ue5m3_gemm_native_workspace_bytes(a.R, b.R, a.Kc, a.scale_mode, b.scale_mode)
    return torch.empty(max(int(n), 16), dtype=torch.uint8, device=a.payload.device)     # 0: a Kc the call will refuse


def native_windows(workspace: torch.Tensor, a: QuantizedOperand, b: QuantizedOperand):
    """Reads a workspace back: (all rows have windows, k of A's scale rows, k of B's scale rows) as numpy arrays."""
    ra = a.R // 16 if a.scale_mode == SCALE_2D else a.R
    rb = b.R // 16 if b.scale_mode == SCALE_2D else b.R
    off_b = 16 + ((ra + 15) // 16) * 16
    w = workspace[:off_b + rb].cpu().numpy()          # the shifted scales that follow are the kernel's own business
    return int(w[:4].view("int32")[0]) == 0, w[16:16 + ra].copy(), w[off_b:off_b + rb].copy()


def gemm_native(op: int, a: QuantizedOperand, b: QuantizedOperand, out_dtype: torch.dtype = torch.bfloat16,
                out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The product of `gemm` on the tensor core's FP4 path (ue5m3_gemm_native).  `workspace` (see gemm_native_workspace)
    receives the window shift of every scale row; `out` is left untouched when some row has no UE4M3 window."""
    Mo, No, Kc = a.R, b.R, a.Kc
    if b.Kc != Kc:
        raise ValueError(f"contraction sizes differ: {Kc} vs {b.Kc}")
    if out is None:
        out = torch.empty((Mo, No), dtype=out_dtype, device=a.payload.device)
    if workspace is None:
        workspace = gemm_native_workspace(a, b)
    with torch.cuda.device(out.device):
        _check(_load().ue5m3_gemm_native(op, Mo, No, Kc,
                                         _dev_ptr(a.payload), _dev_ptr(a.scales), a.scale_mode, _dev_ptr(a.decode),
                                         _dev_ptr(b.payload), _dev_ptr(b.scales), b.scale_mode, _dev_ptr(b.decode),
                                         _dev_ptr(out), _dtype_code(out), out.stride(0), _dev_ptr(workspace), _stream(out)),
               "ue5m3_gemm_native")
    return out


def gemm_probe_matched(op: int, a: QuantizedOperand, b: QuantizedOperand, out_dtype: torch.dtype = torch.bfloat16,
                       out: Optional[torch.Tensor] = None, cross_rounding: int = 0,
                       grid_denominator: int = 1024) -> torch.Tensor:
    """The same product under the output model of Section 6.2: 64-product partials rounded to nearest even,
    cross-group additions toward zero, 1/grid_denominator grid, scale product last (ue5m3_gemm_probe_matched)."""
    Mo, No, Kc = a.R, b.R, a.Kc
    if b.Kc != Kc:
        raise ValueError(f"contraction sizes differ: {Kc} vs {b.Kc}")
    if out is None:
        out = torch.empty((Mo, No), dtype=out_dtype, device=a.payload.device)
    with torch.cuda.device(out.device):
        _check(_load().ue5m3_gemm_probe_matched(op, Mo, No, Kc,
                                                _dev_ptr(a.payload), _dev_ptr(a.scales), a.scale_mode, _dev_ptr(a.decode),
                                                _dev_ptr(b.payload), _dev_ptr(b.scales), b.scale_mode, _dev_ptr(b.decode),
                                                int(cross_rounding), int(grid_denominator),
                                                _dev_ptr(out), _dtype_code(out), out.stride(0), _stream(out)),
               "ue5m3_gemm_probe_matched")
    return out


def gemm_stall_selftest(which: int, a: QuantizedOperand, b: QuantizedOperand, out: torch.Tensor,
                        wait_limit_cycles: int = 2_000_000) -> None:
    """ue5m3_gemm_stall_selftest: launches the chosen GEMM kernel (0: FP16 kernel of ue5m3_gemm, 1: ue5m3_gemm_probe_matched,
    2: native FP4 kernel of ue5m3_gemm) with its
    copy producer switched off and every wait bounded by `wait_limit_cycles`; `out` is left untouched and
    `last_device_status()` then reports the timeout once."""
    with torch.cuda.device(out.device):
        _check(_load().ue5m3_gemm_stall_selftest(int(which), a.R, b.R, a.Kc,
                                                 _dev_ptr(a.payload), _dev_ptr(a.scales), a.scale_mode, _dev_ptr(a.decode),
                                                 _dev_ptr(b.payload), _dev_ptr(b.scales), b.scale_mode, _dev_ptr(b.decode),
                                                 _dev_ptr(out), _dtype_code(out), out.stride(0), int(wait_limit_cycles),
                                                 _stream(out)), "ue5m3_gemm_stall_selftest")


def last_device_status() -> int:
    return int(_load().ue5m3_last_device_status())


# ---------------------------------------------------------------------------------------------
# The operators between the quantized linears.  Small calls are bound by what the host does, so these wrappers ask torch for as
# little as they can: sizes and strides once as tuples, outputs through new_empty, no device switch when the device is current.
def _call(fn, where: str, x: torch.Tensor, *args) -> None:
    """fn(*args, stream) on x's device and torch's current stream there."""
    if not x.is_cuda:
        raise ValueError("the library takes device tensors only")
    index = x.get_device()
    if index == torch.cuda.current_device():
        status = fn(*args, torch._C._cuda_getCurrentRawStream(index))
    else:
        with torch.cuda.device(index):
            status = fn(*args, torch._C._cuda_getCurrentRawStream(index))
    if status:
        raise Ue5m3Error(status, where)


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _differs(t: torch.Tensor, shape, like: torch.Tensor) -> bool:
    return t.shape != shape or t.dtype != like.dtype or t.get_device() != like.get_device()


def _unlike(t: torch.Tensor, shape, like: torch.Tensor) -> ValueError:
    return ValueError(f"expected a tensor like [{tuple(shape)}, {like.dtype}, {like.device}], got [{tuple(t.shape)}, {t.dtype}, {t.device}]")


def _rows(x: torch.Tensor, like: Optional[torch.Tensor] = None):
    """(rows, cols, leading dimension) of a 2-D tensor with contiguous rows; `like`: its shape, type and device are required."""
    if like is not None and _differs(x, like.shape, like):
        raise _unlike(x, like.shape, like)
    if x.dim() != 2:
        raise ValueError("expected a 2-D tensor whose rows are contiguous")
    (rows, cols), (ld, one) = x.shape, x.stride()
    if one != 1 and cols > 1:
        raise ValueError("expected a 2-D tensor whose rows are contiguous")
    return rows, cols, ld if rows > 1 else cols


def _vector(t: Optional[torch.Tensor], n: int, like: torch.Tensor, dtype=None):
    if t is not None and (t.dim() != 1 or t.shape[0] != n or (n > 1 and t.stride(0) != 1) or t.get_device() != like.get_device()
                          or (dtype is not None and t.dtype != dtype)):
        raise ValueError(f"expected a contiguous vector of {n} values{'' if dtype is None else f' of {dtype}'} on {like.device}")


def layer_norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None, eps: float = 1e-5,
               out: Optional[torch.Tensor] = None) -> tuple:
    """ue5m3_layer_norm: (y, mean, rstd) of the rows of `x` [rows, cols] (float32 or bfloat16); weight and bias [cols], float32 or
    bfloat16, may be None.  mean and rstd (float32 [rows]) are what `layer_norm_backward` takes."""
    rows, cols, ldx = _rows(x)
    param = weight if weight is not None else bias
    _vector(weight, cols, x)
    _vector(bias, cols, x, None if param is None else param.dtype)
    if out is None:
        out, ldy = x.new_empty((rows, cols)), cols
    else:
        ldy = _rows(out, x)[2]
    mean, rstd = x.new_empty(rows, dtype=torch.float32), x.new_empty(rows, dtype=torch.float32)
    _call(_load().ue5m3_layer_norm, "ue5m3_layer_norm", x, x.data_ptr(), _dtype_code(x), rows, cols, ldx, _ptr(weight), _ptr(bias),
          F32 if param is None else _dtype_code(param), eps, out.data_ptr(), ldy, mean.data_ptr(), rstd.data_ptr())
    return out, mean, rstd


def layer_norm_backward(dy: torch.Tensor, x: torch.Tensor, weight: Optional[torch.Tensor], mean: torch.Tensor, rstd: torch.Tensor,
                        want_weight: bool = True, want_bias: bool = True, out: Optional[torch.Tensor] = None,
                        bias_dtype: Optional[torch.dtype] = None) -> tuple:
    """ue5m3_layer_norm_backward: (dx, dweight, dbias).  dweight is None without a weight or when not wanted, dbias when not
    wanted; both have the weight's type.  Without a weight dbias has the type `bias_dtype` (x's by default)."""
    rows, cols, ldx = _rows(x)
    lddy = _rows(dy, x)[2]
    _vector(weight, cols, x)
    _vector(mean, rows, x, torch.float32)
    _vector(rstd, rows, x, torch.float32)
    if out is None:
        out, lddx = x.new_empty((rows, cols)), cols
    else:
        lddx = _rows(out, x)[2]
    param = weight.dtype if weight is not None else x.dtype if bias_dtype is None else bias_dtype
    if bias_dtype is not None and bias_dtype != param:
        raise ValueError(f"weight and bias have one type: {param} and {bias_dtype}")
    param_code = _dtype_code_of(param)
    lib = _load()
    dw = x.new_empty(cols, dtype=param) if want_weight and weight is not None else None
    db = x.new_empty(cols, dtype=param) if want_bias else None
    ws = None
    if dw is not None or db is not None:
        ws = x.new_empty(lib.ue5m3_layer_norm_backward_workspace_bytes(rows, cols), dtype=torch.uint8)
    _call(lib.ue5m3_layer_norm_backward, "ue5m3_layer_norm_backward", x, dy.data_ptr(), lddy, x.data_ptr(), _dtype_code(x), rows, cols, ldx,
          _ptr(weight), param_code, mean.data_ptr(), rstd.data_ptr(), out.data_ptr(), lddx, _ptr(dw), _ptr(db), _ptr(ws))
    return out, dw, db


def dropout_add(x: torch.Tensor, p: float, seed: int, residual: Optional[torch.Tensor] = None,
                out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """ue5m3_dropout_add: residual + dropout(x) for `x` [rows, cols]; the draws depend on the seed and the element's index only.
    The gradient of x is this call on dy with the same p and seed and no residual."""
    rows, cols, ldx = _rows(x)
    ldr = 0 if residual is None else _rows(residual, x)[2]
    if out is None:
        out, ldy = x.new_empty((rows, cols)), cols
    else:
        ldy = _rows(out, x)[2]
    _call(_load().ue5m3_dropout_add, "ue5m3_dropout_add", x, x.data_ptr(), ldx, _ptr(residual), ldr, _dtype_code(x), rows, cols, p,
          int(seed) & (2 ** 64 - 1), out.data_ptr(), ldy)
    return out


def _heads(t: torch.Tensor, shape, like: torch.Tensor) -> _Heads:
    if t.shape != shape or (t is not like and _differs(t, shape, like)):       # (`like` itself may stand where another shape is wanted)
        raise _unlike(t, shape, like)
    batch, token, head, one = t.stride()
    if one != 1 and shape[3] > 1:
        raise ValueError("expected tensors [batch, tokens, heads, head_dim] whose last dimension is contiguous")
    return _Heads(t.data_ptr(), batch, token, head)


def _attention_shape(q, k, causal, window_left, k_lens, scale) -> _AttentionShape:
    if q.dim() != 4 or k.dim() != 4:
        raise ValueError("expected tensors [batch, tokens, heads, head_dim]")
    (B, Lq, H, D), (Bk, Lk, Hk, Dk) = q.shape, k.shape
    if Bk != B or Dk != D:
        raise ValueError(f"q {tuple(q.shape)} and k {tuple(k.shape)} differ in batch or head dimension")
    if k_lens is not None and (k_lens.dim() != 1 or k_lens.shape[0] != B or k_lens.dtype != torch.int32 or not k_lens.is_contiguous()
                               or k_lens.get_device() != q.get_device()):
        raise ValueError("k_lens must be a contiguous int32 tensor with one length per sequence, on the queries' device")
    return _AttentionShape(B, Lq, Lk, H, Hk, D, int(window_left), _ptr(k_lens), D ** -0.5 if scale is None else float(scale),
                           _dtype_code(q), 1 if causal else 0)


def attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, causal: bool = False, window_left: int = -1,
              k_lens: Optional[torch.Tensor] = None, scale: Optional[float] = None, out: Optional[torch.Tensor] = None, sinks: int = 0) -> tuple:
    """ue5m3_attention (ue5m3_attention_sinks with `sinks`: the first keys, up to 128, that stay visible behind the window): (o, lse) for q [batch, tokens, heads, head_dim] and k, v [batch, keys, kv_heads, head_dim], bfloat16.  Any
    strides with a contiguous last dimension (views of a fused projection); `window_left` = keys a query sees before its own
    position (-1: all), `k_lens` int32 [batch] = valid keys of each sequence, `scale` defaults to head_dim ** -0.5.  Query i stands at
    position i + keys - tokens of every sequence, whatever its k_lens (right-padded batches).  `out` may be q; any other overlap with
    an input is refused."""
    shape = _attention_shape(q, k, causal, window_left, k_lens, scale)
    if out is None:
        out = q.new_empty(q.shape)
    lse = q.new_empty((shape.batch, shape.heads, shape.q_len), dtype=torch.float32)
    lib = _load()
    need = lib.ue5m3_attention_workspace_bytes(shape)
    ws = q.new_empty(need, dtype=torch.uint8) if need else None
    args = _heads(q, q.shape, q), _heads(k, k.shape, q), _heads(v, k.shape, q), _heads(out, q.shape, q), lse.data_ptr(), _ptr(ws)
    if sinks:
        _call(lib.ue5m3_attention_sinks, "ue5m3_attention_sinks", q, shape, sinks, *args)
    else:
        _call(lib.ue5m3_attention, "ue5m3_attention", q, shape, *args)
    return out, lse


def attention_backward(dout: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, o: torch.Tensor, lse: torch.Tensor,
                       causal: bool = False, window_left: int = -1, k_lens: Optional[torch.Tensor] = None,
                       scale: Optional[float] = None, out: Optional[tuple] = None, sinks: int = 0) -> tuple:
    """ue5m3_attention_backward (ue5m3_attention_sinks_backward with `sinks`): (dq, dk, dv) from what `attention` returned (o, lse) and the gradient of o; the other arguments as
    in that call.  `out`: three tensors to write to (any strides with a contiguous last dimension, e.g. views of one fused
    gradient) that overlap neither one another nor dout, q, k, v."""
    shape = _attention_shape(q, k, causal, window_left, k_lens, scale)
    qs, ks = q.shape, k.shape
    if lse.shape != (shape.batch, shape.heads, shape.q_len) or lse.dtype != torch.float32 or not lse.is_contiguous() or lse.get_device() != q.get_device():
        raise ValueError("lse must be the contiguous float32 [batch, heads, tokens] tensor that attention returned")
    dq, dk, dv = (q.new_empty(qs), k.new_empty(ks), k.new_empty(ks)) if out is None else out
    lib = _load()
    need = lib.ue5m3_attention_sinks_backward_workspace_bytes(shape, sinks) if sinks else lib.ue5m3_attention_backward_workspace_bytes(shape)
    ws = q.new_empty(need, dtype=torch.uint8)
    args = _heads(dout, qs, q), _heads(q, qs, q), _heads(k, ks, q), _heads(v, ks, q), _heads(o, qs, q), lse.data_ptr(), _heads(dq, qs, q), \
        _heads(dk, ks, q), _heads(dv, ks, q), ws.data_ptr()
    if sinks:
        _call(lib.ue5m3_attention_sinks_backward, "ue5m3_attention_sinks_backward", q, shape, sinks, *args)
    else:
        _call(lib.ue5m3_attention_backward, "ue5m3_attention_backward", q, shape, *args)
    return dq, dk, dv


def rotary_frequencies(rotary_dim: int, base: float = 10000.0, scaling: Optional[str] = None, factor: float = 1.0,
                       trained_length: Optional[int] = None, fast: float = 32.0, slow: float = 1.0, device="cuda") -> tuple:
    """(frequencies, amplitude) for the rotary calls: base^(-2 i / rotary_dim) radians per position, a float64 tensor [rotary_dim / 2], and
    1.0.  For contexts `factor` times longer than the trained one, `scaling`:
      "linear"  every frequency divided by the factor (positions shrunk);
      "base"    a larger base, by which the slowest pair turns `factor` times slower and the fastest as before;
      "parts"   pairs that turn at most `slow` times within `trained_length` positions are divided by the factor, those that turn `fast`
                times or more stay, a linear ramp in between; the amplitude is 0.1 ln(factor) + 1."""
    if rotary_dim < 2 or rotary_dim % 2:
        raise ValueError(f"rotary_dim = {rotary_dim}: a positive even number is wanted")
    if not base > 0 or not factor >= 1:
        raise ValueError(f"base {base} has to be positive and factor {factor} at least 1")
    if scaling not in (None, "linear", "base", "parts"):
        raise ValueError(f"unknown scaling {scaling!r}: None, 'linear', 'base' or 'parts'")
    if scaling == "base" and rotary_dim > 2:
        base = base * factor ** (rotary_dim / (rotary_dim - 2))
    f = torch.tensor([base ** (-2.0 * i / rotary_dim) for i in range(rotary_dim // 2)], dtype=torch.float64)
    amplitude = 1.0
    if scaling == "linear":
        f = f / factor
    elif scaling == "parts":
        if not trained_length or not fast > slow:
            raise ValueError("scaling 'parts' wants the trained_length and fast > slow")
        keep = ((trained_length * f / (2 * math.pi) - slow) / (fast - slow)).clamp(0, 1)
        f = f * keep + f / factor * (1 - keep)
        amplitude = 0.1 * math.log(factor) + 1.0
    return f.to(device), amplitude


def _rotary_shape(q, k, frequencies, positions, interleaved, amplitude) -> _RotaryShape:
    if q.dim() != 4 or (k is not None and k.dim() != 4):
        raise ValueError("expected tensors [batch, tokens, heads, head_dim]")
    B, L, H, D = q.shape
    Hk = 0
    if k is not None:
        Bk, Lk, Hk, Dk = k.shape
        if Bk != B or Lk != L or Dk != D:
            raise ValueError(f"q {tuple(q.shape)} and k {tuple(k.shape)} differ in more than the heads")
    if frequencies.dim() != 1 or frequencies.dtype != torch.float64 or not frequencies.is_contiguous() or frequencies.get_device() != q.get_device():
        raise ValueError("frequencies must be a contiguous float64 vector on the queries' device (see rotary_frequencies)")
    first, stride, size, at = 0, 0, 0, None
    if isinstance(positions, int):
        first = positions
    elif positions is not None:
        if positions.dtype not in (torch.int32, torch.int64) or positions.get_device() != q.get_device() or positions.dim() not in (1, 2) or \
                positions.shape[-1] != L or (L > 1 and positions.stride(-1) != 1) or (positions.dim() == 2 and positions.shape[0] not in (1, B)):
            raise ValueError(f"positions must be an int32 or int64 tensor [{L}] or [{B}, {L}] with contiguous tokens on the queries' device")
        at, size = positions.data_ptr(), positions.element_size()
        stride = positions.stride(0) if positions.dim() == 2 and positions.shape[0] > 1 else 0
    return _RotaryShape(B, L, H, Hk, D, 2 * frequencies.shape[0], frequencies.data_ptr(), at, stride, first, size, 1 if interleaved else 0,
                        amplitude, _dtype_code(q))


def _pair(t: tuple, q: torch.Tensor, k: Optional[torch.Tensor]) -> tuple:
    """C descriptions of two tensors like q and k."""
    return _heads(t[0], q.shape, q), None if k is None else _heads(t[1], k.shape, q)


def _out_pair(q: torch.Tensor, k: Optional[torch.Tensor], out: Optional[tuple]) -> tuple:
    """((q's, k's output), their C descriptions): new contiguous tensors unless given."""
    if out is not None:
        return out, _pair(out, q, k)
    shape = q.shape
    _, L, H, D = shape
    a = q.new_empty(shape)
    if k is None:
        return (a, None), (_Heads(a.data_ptr(), L * H * D, H * D, D), None)
    shape = k.shape
    b, n = k.new_empty(shape), shape[2] * D
    return (a, b), (_Heads(a.data_ptr(), L * H * D, H * D, D), _Heads(b.data_ptr(), L * n, n, D))


def rotary(q: torch.Tensor, k: Optional[torch.Tensor], frequencies: torch.Tensor, positions=None, interleaved: bool = False,
           amplitude: float = 1.0, inverse: bool = False, out: Optional[tuple] = None) -> tuple:
    """ue5m3_rotary: (q, k) with the first 2 * len(frequencies) values of every head's row turned by position * frequency.  q [batch, tokens,
    heads, head_dim], k [batch, tokens, kv_heads, head_dim] or None, float32 or bfloat16, any strides with a contiguous last dimension;
    `frequencies` float64 (see rotary_frequencies).  `positions`: None (the tokens' indices), the first token's position, or an int32 / int64
    tensor [tokens] or [batch, tokens].  `inverse` turns back, which is the gradient.  `out` may be (q, k)."""
    shape = _rotary_shape(q, k, frequencies, positions, interleaved, amplitude)
    out, to = _out_pair(q, k, out)
    _call(_load().ue5m3_rotary, "ue5m3_rotary", q, shape, 1 if inverse else 0, *_pair((q, k), q, k), *to)
    return out


def _norm_weights(q, q_weight, k_weight):
    """The weights' type code."""
    one = q_weight if q_weight is not None else k_weight
    dtype = None if one is None else one.dtype
    for w in (q_weight, k_weight):
        _vector(w, q.shape[-1], q, dtype)
    return F32 if one is None else _dtype_code_of(dtype)


def qk_norm_rotary(q: torch.Tensor, k: Optional[torch.Tensor], q_weight: Optional[torch.Tensor], k_weight: Optional[torch.Tensor],
                   frequencies: torch.Tensor, positions=None, interleaved: bool = False, amplitude: float = 1.0, eps: float = 1e-6,
                   out: Optional[tuple] = None) -> tuple:
    """ue5m3_qk_norm_rotary: (q, k) with every head's row divided by its root mean square, times the weight [head_dim] (float32 or bfloat16,
    None: 1), and turned as by `rotary`, whose other arguments these are."""
    shape = _rotary_shape(q, k, frequencies, positions, interleaved, amplitude)
    code = _norm_weights(q, q_weight, k_weight)
    out, to = _out_pair(q, k, out)
    _call(_load().ue5m3_qk_norm_rotary, "ue5m3_qk_norm_rotary", q, shape, *_pair((q, k), q, k), _ptr(q_weight), _ptr(k_weight), code, eps, *to)
    return out


def qk_norm_rotary_backward(dq: torch.Tensor, dk: Optional[torch.Tensor], q: torch.Tensor, k: Optional[torch.Tensor],
                            q_weight: Optional[torch.Tensor], k_weight: Optional[torch.Tensor], frequencies: torch.Tensor, positions=None,
                            interleaved: bool = False, amplitude: float = 1.0, eps: float = 1e-6, want_weights: bool = True,
                            out: Optional[tuple] = None) -> tuple:
    """ue5m3_qk_norm_rotary_backward: (dq, dk, dq_weight, dk_weight) from the gradients of what `qk_norm_rotary` returned and its arguments.
    A weight's gradient has the weight's type; it is None without the weight or when not wanted.  `out`: where dq and dk go (may be the
    upstream gradients)."""
    shape = _rotary_shape(q, k, frequencies, positions, interleaved, amplitude)
    code = _norm_weights(q, q_weight, k_weight)
    out, to = _out_pair(q, k, out)
    dqw = q_weight.new_empty(q_weight.shape) if want_weights and q_weight is not None else None
    dkw = k_weight.new_empty(k_weight.shape) if want_weights and k_weight is not None else None
    lib = _load()
    ws = None
    if dqw is not None or dkw is not None:
        ws = q.new_empty(lib.ue5m3_qk_norm_rotary_backward_workspace_bytes(shape), dtype=torch.uint8)
    _call(lib.ue5m3_qk_norm_rotary_backward, "ue5m3_qk_norm_rotary_backward", q, shape, *_pair((dq, dk), q, k), *_pair((q, k), q, k),
          _ptr(q_weight), _ptr(k_weight), code, eps, *to, _ptr(dqw), _ptr(dkw), _ptr(ws))
    return *out, dqw, dkw


ADAMW_BLOCK = 256           # elements that share a scale of 8-bit moments
_NUMBERS = {torch.float32: F32, torch.bfloat16: BF16}
ADAMW_CLOCK_BYTES = 32


def adamw(params, grads, m, v, step: int = 1, lr: float = 1e-3, betas: tuple = (0.9, 0.999), eps: float = 1e-8, weight_decay: float = 0.01,
          master=None, m_scale=None, v_scale=None, grad_scale: Optional[torch.Tensor] = None, seed: int = 0,
          clock: Optional[torch.Tensor] = None, streams=None) -> None:
    """ue5m3_adamw: one AdamW step over lists of contiguous tensors on one device, in place.  params and grads float32 or bfloat16; `master`: float32
    copies of the params (a list, entries may be None) that take the step instead and are rounded into them.  Moments m and v: float32, or uint8
    with `m_scale` and `v_scale` (float32, one for every ADAMW_BLOCK elements; all zeros before the first step), rounded by draws of (seed, stream, step,
    element), where `streams` (default: the places in the lists) tell the tensors apart.  `step` counts from 1; `clock` (ADAMW_CLOCK_BYTES zero bytes, uint8 or int64)
    counts on the device instead, for steps captured into a graph.  `grad_scale`: float32 tensor of one value that the gradients are multiplied by; where it
    is not finite nothing is written."""
    count = len(params)
    eight = m_scale is not None
    if not (len(grads) == len(m) == len(v) == count) or any(x is not None and len(x) != count for x in (master, m_scale, v_scale, streams)) or \
            eight != (v_scale is not None):
        raise ValueError("params, grads and their states are lists of the same length (m_scale and v_scale both or neither)")
    if count == 0:
        return
    device = params[0].get_device()
    state = torch.uint8 if eight else torch.float32

    def column(ts, sizes, types, what) -> list:
        """Addresses of a list of tensors, each contiguous, of its size and one of the types, on the first one's device."""
        at = [t.data_ptr() for t, n in zip(ts, sizes) if t.dtype in types and t.numel() == n and t.is_contiguous() and t.get_device() == device]
        if len(at) != count:
            for i, (t, n) in enumerate(zip(ts, sizes)):
                if len(types) > 1:
                    _dtype_code(t)
                if t.dtype not in types or t.numel() != n or not t.is_contiguous() or t.get_device() != device:
                    raise ValueError(f"{what}[{i}]: expected a contiguous tensor of {n} values of {types} on {params[0].device}, got [{tuple(t.shape)}, {t.dtype}, {t.device}]")
        return at

    sizes, none = [p.numel() for p in params], [0] * count
    first = column(params, sizes, _NUMBERS, "params")
    if len(set(first)) != count and len({x for x, n in zip(first, sizes) if n}) != sum(n > 0 for n in sizes):
        raise ValueError("a tensor stands in params twice")
    at_grads = column(grads, sizes, _NUMBERS, "grads")
    if [g.shape for g in grads] != [p.shape for p in params]:
        raise ValueError("params and grads have different shapes")
    copies = none
    if master is not None:
        some = [i for i, t in enumerate(master) if t is not None]
        if len(some) == count:
            copies = column(master, sizes, (torch.float32,), "master")
        else:
            copies = list(none)
            for i in some:
                t = master[i]
                if t.dtype is not torch.float32 or t.numel() != sizes[i] or not t.is_contiguous() or t.get_device() != device:
                    raise ValueError(f"master[{i}]: expected a contiguous tensor of {sizes[i]} float32 on {params[0].device}, got [{tuple(t.shape)}, {t.dtype}, {t.device}]")
                copies[i] = t.data_ptr()
    scales = none, none
    if eight:
        blocks = [-(-n // ADAMW_BLOCK) for n in sizes]
        scales = column(m_scale, blocks, (torch.float32,), "m_scale"), column(v_scale, blocks, (torch.float32,), "v_scale")
    kinds = [(x & 0xFFFFFFFF) | _NUMBERS[p.dtype] << 32 | _NUMBERS[g.dtype] << 40 for x, p, g in zip(range(count) if streams is None else streams, params, grads)]
    rows = zip(first, at_grads, copies, column(m, sizes, (state,), "m"), column(v, sizes, (state,), "v"), *scales, sizes, kinds)
    flat = array("q", [x for row in rows for x in row])
    for t, what in ((grad_scale, "grad_scale"), (clock, "clock")):
        if t is not None and t.get_device() != device:
            raise ValueError(f"{what} is on {t.device}, the params on {params[0].device}")
    if grad_scale is not None and (grad_scale.dtype != torch.float32 or grad_scale.numel() != 1):
        raise ValueError("grad_scale must be a float32 tensor of one value")
    if clock is not None and (clock.numel() * clock.element_size() < ADAMW_CLOCK_BYTES or not clock.is_contiguous()):
        raise ValueError(f"clock must hold {ADAMW_CLOCK_BYTES} bytes")
    how = _AdamwStep(step, lr, betas[0], betas[1], eps, weight_decay, _ptr(grad_scale), _ptr(clock), int(seed) & (2 ** 64 - 1), 8 if eight else 32)
    _call(_load().ue5m3_adamw, "ue5m3_adamw", params[0], flat.buffer_info()[0], count, how)


def block_stall_selftest(which: int, buffer: torch.Tensor, wait_limit_cycles: int = 2_000_000) -> None:
    """ue5m3_block_stall_selftest: launches a small attention (0), attention with few queries (1), attention backward (2), layer
    norm (3) or layer norm backward (4) with its copies switched off and every wait bounded by `wait_limit_cycles`; `last_device_status()` then reports the timeout once."""
    _call(_load().ue5m3_block_stall_selftest, "ue5m3_block_stall_selftest", buffer, int(which), buffer.data_ptr(),
          buffer.numel() * buffer.element_size(), int(wait_limit_cycles))


# ---------------------------------------------------------------------------------------------
class AmaxCache:
    """Sample-and-hold tensor reference of one operand: the maximum is re-sampled when the cache is
    empty or `interval` steps old and held in between (not a window maximum).  The held value stays
    on the device, so holding costs nothing and refreshing costs one ue5m3_sample_amax launch."""

    def __init__(self, interval: int = 50):
        self.interval = int(interval)
        self.last_refresh: Optional[int] = None
        self.held: Optional[torch.Tensor] = None

    def refreshes_at(self, step: int) -> bool:
        return self.last_refresh is None or step - self.last_refresh >= self.interval

    def get(self, x: torch.Tensor, step: int) -> torch.Tensor:
        if self.refreshes_at(step):
            self.held = sample_amax(x, self.held)
            self.last_refresh = step
        return self.held


def _multiply(op: int, a: QuantizedOperand, b: QuantizedOperand, out_dtype: torch.dtype, grid_denominator: Optional[int]):
    """`gemm`, or `gemm_probe_matched` with the given grid when `grid_denominator` is not None."""
    if grid_denominator is None:
        return gemm(op, a, b, out_dtype)
    return gemm_probe_matched(op, a, b, out_dtype, grid_denominator=grid_denominator)


def linear_forward(x: torch.Tensor, w: torch.Tensor, amax_x: torch.Tensor, amax_w: torch.Tensor,
                   target_T: float = 448.0, out_dtype: torch.dtype = torch.bfloat16,
                   scale_layout: int = SCALES_ROWMAJOR, grid_denominator: Optional[int] = None):
    """Y = X W^T: quantize X (1D along K, RNE) and W (2D tiles, RNE, with transposed copy), multiply.
    Returns (Y, qx, qw); qw carries the transposed view the backward pass needs.  `grid_denominator` not None
    selects the Section 6.2 output model for the product (0 = that model without its grid step)."""
    qx = quantize(x, LAYOUT_1D_ROW, ROUND_RNE, amax_x, target_T, scale_layout=scale_layout)
    qw = quantize(w, LAYOUT_2D, ROUND_RNE, amax_w, target_T, want_transpose=True)
    return _multiply(FPROP, qx, qw, out_dtype, grid_denominator), qx, qw


def linear_backward(dy: torch.Tensor, x: torch.Tensor, qw: QuantizedOperand, amax_dy: torch.Tensor,
                    amax_x: torch.Tensor, seed: int, target_T: float = 448.0, target_T_wgrad_dy: float = 448.0,
                    out_dtype: torch.dtype = torch.bfloat16, scale_layout: int = SCALES_ROWMAJOR,
                    grid_denominator: Optional[int] = None, grad_rounding: int = ROUND_SR):
    """dX = dY W and dW = dY^T X.  dY is rounded stochastically by default, once per GEMM with seeds 4*seed and
    4*seed + 1 (`grad_rounding = ROUND_RNE` gives the nearest-even control); the saved activation X is
    re-quantized along the token dimension with RNE."""
    qdy = quantize(dy, LAYOUT_1D_ROW, grad_rounding, amax_dy, target_T, seed=4 * seed, scale_layout=scale_layout)
    dx = _multiply(DGRAD, qdy, qw.transposed(), out_dtype, grid_denominator)
    qdy_t = quantize(dy, LAYOUT_1D_COL, grad_rounding, amax_dy, target_T_wgrad_dy, seed=4 * seed + 1, scale_layout=scale_layout)
    qx_t = quantize(x, LAYOUT_1D_COL, ROUND_RNE, amax_x, target_T, scale_layout=scale_layout)
    dw = _multiply(WGRAD, qdy_t, qx_t, out_dtype, grid_denominator)
    return dx, dw
