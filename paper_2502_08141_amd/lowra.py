"""Thin Python binding of the C-ABI HIP library (include/lowra.h): argument marshalling only.

Functions carry the names of the C entry points.  Tensors are torch CUDA (ROCm) tensors used as
device memory; every step of the path runs in the library's kernels on torch's current stream.
There is no CPU fallback: a missing library or a failing call raises.
"""
from __future__ import annotations

import ctypes as C
import dataclasses
import importlib.util
import os

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "liblowra_hip.so")
CALL_PATH = os.path.join(_HERE, "_lowra_call.so")
_lib = None
_call = None        # csrc/call.cpp: the calls made once per layer, natively for plain tensors; None from it: go on here

OK, INVALID_ARG, UNSUPPORTED, MISALIGNED, WORKSPACE_TOO_SMALL, HIP_ERROR, OUT_OF_MEMORY = range(7)
STATIC_SCRATCH_BYTES, STATIC_ARRAY_BYTES = 4 << 20, 36 << 20
OP_LINEAR_FWD, OP_LINEAR_BWD_INPUT, OP_ADAPTER_GRADS, OP_LOFTQ_INIT = 0, 1, 2, 3
OUT_BF16, OUT_FP32 = 0, 1
PATH_AUTO, PATH_GEMV, PATH_GEMM, PATH_GEMV_GENERAL = 0, 1, 2, 3
SCALE_FP32, SCALE_BF16 = 0, 1
ACT_NONE, ACT_RELU, ACT_GELU, ACT_GELU_TANH, ACT_SILU = 0, 1, 2, 3, 4
ACTS = {"none": ACT_NONE, "relu": ACT_RELU, "gelu": ACT_GELU, "gelu_tanh": ACT_GELU_TANH, "silu": ACT_SILU}
NORM_LAYER, NORM_RMS = 0, 1
ROPE_HALF, ROPE_INTERLEAVED = 0, 1
ROPE_SCALE_NONE, ROPE_SCALE_LINEAR, ROPE_SCALE_BASE, ROPE_SCALE_TURNS, ROPE_SCALE_INDEX = 0, 1, 2, 3, 4
ROPE_SCALINGS = {"none": ROPE_SCALE_NONE, "linear": ROPE_SCALE_LINEAR, "base": ROPE_SCALE_BASE, "turns": ROPE_SCALE_TURNS, "index": ROPE_SCALE_INDEX}

SYMBOLS = [
    "lowra_status_string", "lowra_plan_rows", "lowra_layout_create", "lowra_layout_destroy", "lowra_layout_set_scale_dtype",
    "lowra_packed_bytes", "lowra_workspace_bytes", "lowra_quantize", "lowra_quantize_batch", "lowra_dequantize",
    "lowra_linear_fwd", "lowra_linear_fwd_static", "lowra_linear_bwd_input", "lowra_set_linear_path", "lowra_set_fwd_tiling", "lowra_plan_fwd_tiling", "lowra_set_mid_tiling",
    "lowra_plan_mid_tiling", "lowra_plan_small_fwd", "lowra_set_kernel_timer",
    "lowra_learn_tables", "lowra_average_thresholds", "lowra_channel_mse", "lowra_assign_precisions",
    "lowra_adapter_grads", "lowra_linear_side_product", "lowra_adapter_grads_from_side", "lowra_loftq_init",
    "lowra_fwd_batch_workspace_bytes", "lowra_fwd_batch_create", "lowra_fwd_batch_run", "lowra_fwd_batch_destroy",
    "lowra_bwd_batch_workspace_bytes", "lowra_bwd_batch_create", "lowra_bwd_batch_run", "lowra_bwd_batch_destroy",
    "lowra_linear_fwd_act", "lowra_linear_bwd_input_act", "lowra_act_bwd", "lowra_act_bwd_workspace_bytes",
    "lowra_muon_batch_workspace_bytes", "lowra_muon_batch_create", "lowra_muon_batch_run", "lowra_muon_batch_destroy",
    "lowra_norm_fwd", "lowra_norm_bwd", "lowra_norm_bwd_workspace_bytes", "lowra_rope", "lowra_rope_frequencies",
    "lowra_vocab_loss", "lowra_vocab_loss_workspace_bytes",
    "lowra_adamw_batch_create", "lowra_adamw_batch_run", "lowra_adamw_batch_destroy", "lowra_adamw_state",
    "lowra_measure_copy", "lowra_measure_read", "lowra_measure_mfma", "lowra_measure_mfma_random",
]


class FwdItem(C.Structure):
    """lowra_fwd_item: one matrix of a batched small-token forward (device pointers)."""
    _fields_ = [("layout", C.c_void_p), ("packed", C.c_void_p), ("absmax", C.c_void_p), ("x", C.c_void_p),
                ("A", C.c_void_p), ("B", C.c_void_p), ("y", C.c_void_p)]


class FwdEpilogue(C.Structure):
    """lowra_fwd_epilogue (device pointers)."""
    _fields_ = [("act", C.c_int), ("bias", C.c_void_p), ("mul", C.c_void_p), ("residual", C.c_void_p), ("z", C.c_void_p)]


class BwdEpilogue(C.Structure):
    """lowra_bwd_epilogue (device pointers)."""
    _fields_ = [("act", C.c_int), ("z", C.c_void_p), ("mul", C.c_void_p), ("residual", C.c_void_p), ("dmul", C.c_void_p)]


class MuonItemRecord(C.Structure):
    """lowra_muon_item (device pointers)."""
    _fields_ = [("rows", C.c_int), ("cols", C.c_int), ("scale", C.c_float)] + [(n, C.c_void_p) for n in (
        "grad", "momentum", "momentum_out", "weight", "weight_out", "weight_bf16", "update")]


class MuonStep(C.Structure):
    """lowra_muon_step."""
    _fields_ = [("lr", C.c_float), ("momentum", C.c_float), ("nesterov", C.c_int), ("weight_decay", C.c_float), ("steps", C.c_int),
                ("a", C.c_float), ("b", C.c_float), ("c", C.c_float), ("eps", C.c_float)]


class RopeTensor(C.Structure):
    """lowra_rope_tensor (device pointers, strides in elements)."""
    _fields_ = [("x", C.c_void_p), ("y", C.c_void_p), ("heads", C.c_int)] + [(n, C.c_int64) for n in (
        "x_token_stride", "x_head_stride", "y_token_stride", "y_head_stride")]


class AdamWItemRecord(C.Structure):
    """lowra_adamw_item (device pointers)."""
    _fields_ = [("count", C.c_int64), ("state_bits", C.c_int), ("lr_scale", C.c_float), ("decay_scale", C.c_float)] + [(n, C.c_void_p) for n in (
        "grad", "m", "v", "m_absmax", "v_absmax", "weight", "m_out", "v_out", "m_absmax_out", "v_absmax_out", "weight_out", "weight_bf16")]


class AdamWStep(C.Structure):
    """lowra_adamw_step."""
    _fields_ = [(n, C.c_double) for n in ("lr", "beta_one", "beta_two", "eps", "weight_decay")] + [("step", C.c_int64)]


class LowraError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} (status {status})")


def lib() -> C.CDLL:
    """Load liblowra_hip.so (built by paper_2502_08141_amd.build); raises if it is not there."""
    global _lib, _call
    if _lib is None:
        for path in (LIB_PATH, CALL_PATH):
            if not os.path.exists(path):
                raise FileNotFoundError(f"{path} is missing: run `python -m paper_2502_08141_amd.build` first")
        L = C.CDLL(LIB_PATH)
        vp, u8p, f32p, u16p = C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p
        L.lowra_status_string.restype = C.c_char_p
        L.lowra_status_string.argtypes = [C.c_int]
        L.lowra_plan_rows.argtypes = [C.c_int, C.c_int, C.c_int, C.c_void_p, C.c_void_p]
        L.lowra_layout_create.argtypes = [C.c_int, C.c_int, C.c_int, C.c_void_p, C.c_void_p, C.c_int,
                                          C.c_void_p, C.POINTER(C.c_void_p)]
        L.lowra_layout_destroy.restype = None
        L.lowra_layout_destroy.argtypes = [vp]
        L.lowra_packed_bytes.restype = C.c_size_t
        L.lowra_packed_bytes.argtypes = [vp]
        L.lowra_workspace_bytes.restype = C.c_size_t
        L.lowra_workspace_bytes.argtypes = [vp, C.c_int, C.c_int, C.c_int]
        L.lowra_layout_set_scale_dtype.argtypes = [vp, C.c_int]
        L.lowra_quantize.argtypes = [vp, f32p, f32p, u8p, f32p, vp]
        L.lowra_quantize_batch.argtypes = [C.c_int, vp, vp, vp, vp, vp, vp]
        L.lowra_dequantize.argtypes = [vp, u8p, f32p, f32p, C.c_int, vp, vp]
        lin = [vp, u8p, f32p, f32p, u16p, C.c_int, u16p, u16p, C.c_int, C.c_float, u16p, vp, C.c_size_t, vp]
        L.lowra_linear_fwd.argtypes = lin
        L.lowra_linear_bwd_input.argtypes = lin
        L.lowra_linear_fwd_static.argtypes = lin[:11] + [vp]
        L.lowra_linear_fwd_act.argtypes = lin[:10] + [vp] + lin[10:]
        L.lowra_linear_bwd_input_act.argtypes = lin[:10] + [vp] + lin[10:]
        L.lowra_act_bwd_workspace_bytes.restype = C.c_size_t
        L.lowra_act_bwd_workspace_bytes.argtypes = [C.c_int, C.c_int]
        L.lowra_act_bwd.argtypes = [C.c_int, C.c_int, C.c_int, u16p, u16p, u16p, u16p, u16p, f32p, vp, C.c_size_t, vp]
        L.lowra_learn_tables.argtypes = [vp, f32p, f32p, f32p, C.c_int, f32p, f32p, f32p, vp]
        L.lowra_average_thresholds.argtypes = [vp, f32p, vp]
        L.lowra_adapter_grads.argtypes = [vp, u16p, u16p, C.c_int, u16p, u16p, C.c_int, C.c_float, f32p, f32p, vp, C.c_size_t, vp]
        L.lowra_linear_side_product.argtypes = [vp, C.c_int, C.c_int, C.c_int, vp]
        L.lowra_linear_side_product.restype = C.c_void_p
        L.lowra_adapter_grads_from_side.argtypes = [vp, u16p, u16p, C.c_int, C.c_int, u16p, u16p, f32p, f32p, vp, C.c_size_t, vp]
        L.lowra_loftq_init.argtypes = [vp, f32p, f32p, f32p, C.c_int, C.c_int, C.c_int, u16p, u8p, f32p, u16p, u16p, vp, C.c_size_t, vp]
        L.lowra_fwd_batch_workspace_bytes.restype = C.c_size_t
        L.lowra_fwd_batch_workspace_bytes.argtypes = [C.c_int, C.c_void_p, C.c_int]
        L.lowra_fwd_batch_create.argtypes = [C.c_int, C.c_void_p, f32p, C.c_int, C.c_int, C.c_float, vp, C.c_size_t, C.c_void_p]
        L.lowra_fwd_batch_run.argtypes = [vp, vp]
        L.lowra_fwd_batch_destroy.restype = None
        L.lowra_fwd_batch_destroy.argtypes = [vp]
        L.lowra_bwd_batch_workspace_bytes.restype = C.c_size_t
        L.lowra_bwd_batch_workspace_bytes.argtypes = [C.c_int, C.c_void_p, C.c_int, C.c_int]
        L.lowra_bwd_batch_create.argtypes = [C.c_int, C.c_void_p, f32p, C.c_int, C.c_int, C.c_float, vp, C.c_size_t, C.c_void_p]
        L.lowra_bwd_batch_run.argtypes = [vp, vp]
        L.lowra_bwd_batch_destroy.restype = None
        L.lowra_bwd_batch_destroy.argtypes = [vp]
        L.lowra_muon_batch_workspace_bytes.restype = C.c_size_t
        L.lowra_muon_batch_workspace_bytes.argtypes = [C.c_int, C.c_void_p]
        L.lowra_muon_batch_create.argtypes = [C.c_int, C.c_void_p, vp, C.c_size_t, C.c_void_p]
        L.lowra_muon_batch_run.argtypes = [vp, vp, vp]
        L.lowra_muon_batch_destroy.restype = None
        L.lowra_muon_batch_destroy.argtypes = [vp]
        L.lowra_norm_fwd.argtypes = [C.c_int] * 3 + [u16p] * 3 + [C.c_float, u16p, vp]
        L.lowra_norm_bwd_workspace_bytes.restype = C.c_size_t
        L.lowra_norm_bwd_workspace_bytes.argtypes = [C.c_int, C.c_int]
        L.lowra_norm_bwd.argtypes = [C.c_int] * 3 + [u16p] * 3 + [C.c_float, u16p, u16p, f32p, f32p, vp, C.c_size_t, vp]
        L.lowra_rope_frequencies.argtypes = [C.c_int, C.c_double, C.c_int, C.c_double, C.c_int, C.c_double, C.c_double, vp]
        L.lowra_rope.argtypes = [C.c_int, vp] + [C.c_int] * 4 + [vp, vp, C.c_float, C.c_int, vp]
        L.lowra_vocab_loss_workspace_bytes.restype = C.c_size_t
        L.lowra_vocab_loss_workspace_bytes.argtypes = [C.c_int] * 4
        L.lowra_vocab_loss.argtypes = [C.c_int] * 3 + [u16p, u16p, vp, f32p, f32p, f32p, u16p, vp, C.c_size_t, vp]
        L.lowra_adamw_batch_create.argtypes = [C.c_int, vp, vp]
        L.lowra_adamw_batch_run.argtypes = [vp, vp, f32p, vp]
        L.lowra_adamw_batch_destroy.restype = None
        L.lowra_adamw_batch_destroy.argtypes = [vp]
        L.lowra_adamw_state.argtypes = [C.c_int64, C.c_int, vp, f32p, f32p, vp]
        L.lowra_channel_mse.argtypes = [C.c_int, C.c_int, f32p, f32p, f32p, f32p, vp]
        L.lowra_assign_precisions.argtypes = [C.c_int, C.c_void_p, C.c_void_p, C.c_double, C.c_void_p]
        L.lowra_measure_copy.argtypes = [vp, vp, C.c_size_t, vp]
        L.lowra_measure_read.argtypes = [vp, C.c_size_t, vp, vp]
        L.lowra_measure_mfma.argtypes = [C.c_int, C.c_int, vp, C.POINTER(C.c_double), vp]
        L.lowra_measure_mfma_random.argtypes = [C.c_int, C.c_int, vp, C.POINTER(C.c_double), vp]
        L.lowra_set_linear_path.argtypes = [C.c_int]
        L.lowra_set_fwd_tiling.argtypes = [C.c_int, C.c_int, C.c_int]
        L.lowra_plan_fwd_tiling.argtypes = [C.c_int, C.c_int, C.c_int, C.POINTER(C.c_int), C.POINTER(C.c_int), C.POINTER(C.c_int)]
        L.lowra_set_mid_tiling.argtypes = [C.c_int, C.c_int]
        L.lowra_plan_mid_tiling.argtypes = [C.c_int] * 6 + [C.POINTER(C.c_int)] * 2
        L.lowra_plan_small_fwd.argtypes = [C.c_int] * 5 + [C.POINTER(C.c_int)] * 3
        L.lowra_set_kernel_timer.argtypes = [vp, vp]
        spec = importlib.util.spec_from_file_location("_lowra_call", CALL_PATH)
        call = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(call)
        call.init(*(C.cast(f, C.c_void_p).value for f in (L.lowra_linear_fwd, L.lowra_linear_bwd_input, L.lowra_linear_side_product,
                                                          L.lowra_adapter_grads, L.lowra_adapter_grads_from_side, L.lowra_dequantize)))
        call.init_act(*(C.cast(f, C.c_void_p).value for f in (L.lowra_linear_fwd_act, L.lowra_linear_bwd_input_act, L.lowra_act_bwd)))
        call.init_step(*(C.cast(f, C.c_void_p).value for f in (L.lowra_norm_fwd, L.lowra_norm_bwd, L.lowra_rope, L.lowra_vocab_loss)))
        _lib, _call = L, call
    return _lib


def status_string(st: int) -> str:
    return lib().lowra_status_string(int(st)).decode()


def _check(st: int, where: str):
    if st != OK:
        raise LowraError(st, where)


def _stream() -> int:
    """Raw handle of the current device's current stream (torch.cuda.current_stream() builds a Python object: 1.5 us)."""
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _ptr(t) -> int:
    return 0 if t is None else t.data_ptr()


def _dev(t: torch.Tensor, dtype, name: str):
    if not (t.dtype is dtype and t.is_cuda and t.is_contiguous()):
        raise TypeError(f"{name}: need a contiguous {dtype} device tensor")
    return t


def lowra_plan_rows(K: int, bits) -> np.ndarray:
    """Host only: byte offset of every channel's row in the packed buffer, int64 [N+1]."""
    bits = np.ascontiguousarray(bits, dtype=np.uint8)
    off = np.zeros(bits.size + 1, dtype=np.int64)
    _check(lib().lowra_plan_rows(bits.size, int(K), 64, bits.ctypes.data, off.ctypes.data), "lowra_plan_rows")
    return off


class Layout:
    """Owner of a lowra_layout handle (lowra_layout_create / lowra_layout_destroy)."""

    def __init__(self, K: int, bits, codebook_id, codebook_bits, group: int = 64):
        self.bits = np.ascontiguousarray(bits, dtype=np.uint8)
        self.cb = np.ascontiguousarray(codebook_id, dtype=np.int32)
        self.cb_bits = np.ascontiguousarray(codebook_bits, dtype=np.uint8)
        if self.cb.shape != self.bits.shape:
            raise ValueError("bits and codebook_id must have the same length")
        self.N, self.K, self.C = int(self.bits.size), int(K), int(self.cb_bits.size)
        h = C.c_void_p()
        st = lib().lowra_layout_create(self.N, self.K, int(group), self.bits.ctypes.data, self.cb.ctypes.data,
                                       self.C, self.cb_bits.ctypes.data, C.byref(h))
        _check(st, "lowra_layout_create")
        self.handle = h
        self.packed_bytes = int(lib().lowra_packed_bytes(h))
        self.scale_dtype = torch.float32
        self._describe()

    def _describe(self):
        """What the native calls read of a layout (csrc/call.cpp); None once it is closed."""
        self.native = (self.handle.value, self.N, self.K, self.C, self.packed_bytes, self.scale_dtype is torch.bfloat16) if self.handle else None

    def set_scale_dtype(self, dtype):
        """torch.float32 (default) or torch.bfloat16: the type of the stored group scales (lowra_layout_set_scale_dtype)."""
        code = {torch.float32: SCALE_FP32, torch.bfloat16: SCALE_BF16}[dtype]
        _check(lib().lowra_layout_set_scale_dtype(self.handle, code), "lowra_layout_set_scale_dtype")
        self.scale_dtype = dtype
        self._describe()
        return self

    def workspace_bytes(self, op: int, M: int, r: int) -> int:
        return int(lib().lowra_workspace_bytes(self.handle, int(op), int(M), int(r)))

    def close(self):
        if getattr(self, "handle", None):
            lib().lowra_layout_destroy(self.handle)
            self.handle, self.packed_bytes, self.native = None, 0, None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


lowra_layout_create = Layout


def lowra_quantize(layout: Layout, W, thresholds, packed=None, absmax=None):
    """W [N,K] fp32, thresholds [C,16] fp32 -> (packed uint8 [packed_bytes], absmax fp32 [N,K/64])."""
    _dev(W, torch.float32, "W"); _dev(thresholds, torch.float32, "thresholds")
    if tuple(W.shape) != (layout.N, layout.K) or tuple(thresholds.shape) != (layout.C, 16):
        raise ValueError("shape mismatch")
    if packed is None:
        packed = torch.empty(layout.packed_bytes, dtype=torch.uint8, device=W.device)
    if absmax is None:
        absmax = torch.empty((layout.N, layout.K // 64), dtype=layout.scale_dtype, device=W.device)
    _dev(packed, torch.uint8, "packed"); _dev(absmax, layout.scale_dtype, "absmax")
    if packed.numel() != layout.packed_bytes or absmax.numel() != layout.N * (layout.K // 64):
        raise ValueError("output size mismatch")
    _check(lib().lowra_quantize(layout.handle, _ptr(W), _ptr(thresholds), _ptr(packed), _ptr(absmax), _stream()),
           "lowra_quantize")
    return packed, absmax


def lowra_quantize_batch(layouts, Ws, thresholds, packed=None, absmax=None):
    """The matrices of a list in as few launches as possible: lists of what lowra_quantize takes -> (list of packed, list of absmax)."""
    n = len(layouts)
    if len(Ws) != n or len(thresholds) != n:
        raise ValueError("list lengths differ")
    packed = [None] * n if packed is None else list(packed)
    absmax = [None] * n if absmax is None else list(absmax)
    if len(packed) != n or len(absmax) != n:
        raise ValueError("list lengths differ")
    for i, (lay, W, thr) in enumerate(zip(layouts, Ws, thresholds)):
        _dev(W, torch.float32, "W"); _dev(thr, torch.float32, "thresholds")
        if tuple(W.shape) != (lay.N, lay.K) or tuple(thr.shape) != (lay.C, 16):
            raise ValueError("shape mismatch")
        if packed[i] is None:
            packed[i] = torch.empty(lay.packed_bytes, dtype=torch.uint8, device=W.device)
        if absmax[i] is None:
            absmax[i] = torch.empty((lay.N, lay.K // 64), dtype=lay.scale_dtype, device=W.device)
        _dev(packed[i], torch.uint8, "packed"); _dev(absmax[i], lay.scale_dtype, "absmax")
        if packed[i].numel() != lay.packed_bytes or absmax[i].numel() != lay.N * (lay.K // 64):
            raise ValueError("output size mismatch")
    arr = lambda values: (C.c_void_p * n)(*values)
    _check(lib().lowra_quantize_batch(n, arr([lay.handle for lay in layouts]), arr([_ptr(W) for W in Ws]),
                                      arr([_ptr(t) for t in thresholds]), arr([_ptr(p) for p in packed]),
                                      arr([_ptr(a) for a in absmax]), _stream()), "lowra_quantize_batch")
    return packed, absmax


def _state(layout, packed, absmax, mappings):
    _dev(packed, torch.uint8, "packed"); _dev(absmax, layout.scale_dtype, "absmax"); _dev(mappings, torch.float32, "mappings")
    if packed.numel() != layout.packed_bytes or absmax.numel() != layout.N * (layout.K // 64) or \
            tuple(mappings.shape) != (layout.C, 16):
        raise ValueError("quantized state does not match the layout")


def _native(result, where: str):
    """What a native call returned, unless it is a status."""
    if result.__class__ is int:
        raise LowraError(result, where)
    return result


def lowra_dequantize(layout: Layout, packed, absmax, mappings, out_dtype=torch.bfloat16, out=None):
    """-> What [N,K] in bf16 (default) or fp32."""
    if out is None and out_dtype is torch.bfloat16 and layout.__class__ is Layout:
        res = _call.dequantize(layout.native, packed, absmax, mappings)
        if res is not None:
            return _native(res, "lowra_dequantize")
    _state(layout, packed, absmax, mappings)
    code = {torch.bfloat16: OUT_BF16, torch.float32: OUT_FP32}[out_dtype]
    if out is None:
        out = torch.empty((layout.N, layout.K), dtype=out_dtype, device=packed.device)
    _dev(out, out_dtype, "out")
    if out.numel() != layout.N * layout.K:
        raise ValueError("output size mismatch")
    _check(lib().lowra_dequantize(layout.handle, _ptr(packed), _ptr(absmax), _ptr(mappings), code, _ptr(out), _stream()),
           "lowra_dequantize")
    return out


def _linear(fn, name, op, layout, packed, absmax, mappings, act, act_cols, out_cols, A, B, s, out, workspace):
    _state(layout, packed, absmax, mappings)
    _dev(act, torch.bfloat16, "activation")
    if act.dim() != 2 or act.shape[1] != act_cols:
        raise ValueError("activation shape mismatch")
    M = int(act.shape[0])
    r = 0
    if A is not None and B is not None and A.shape[0] > 0:
        _dev(A, torch.bfloat16, "A"); _dev(B, torch.bfloat16, "B")
        r = int(A.shape[0])
        if tuple(A.shape) != (r, layout.K) or tuple(B.shape) != (layout.N, r):
            raise ValueError("LoRA operand shape mismatch")
    else:
        A = B = None
    if out is None:
        out = torch.empty((M, out_cols), dtype=torch.bfloat16, device=act.device)
    _dev(out, torch.bfloat16, "out")
    if tuple(out.shape) != (M, out_cols):
        raise ValueError("output shape mismatch")
    if workspace is None:                                     # (a caller's own is checked by the library)
        need = layout.workspace_bytes(op, M, r)
        if need:
            workspace = torch.empty(need, dtype=torch.uint8, device=act.device)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(fn(layout.handle, packed.data_ptr(), absmax.data_ptr(), mappings.data_ptr(), act.data_ptr(), M, _ptr(A), _ptr(B), r,
              s, out.data_ptr(), _ptr(workspace), ws_bytes, _stream()), name)
    return out


def lowra_linear_fwd(layout: Layout, packed, absmax, mappings, x, A, B, s, y=None, workspace=None):
    """y [M,N] bf16 = x What^T + s (x A^T) B^T."""
    if y is None and workspace is not None and layout.__class__ is Layout:
        res = _call.linear(0, layout.native, packed, absmax, mappings, x, A, B, s, workspace)
        if res is not None:
            return _native(res, "lowra_linear_fwd")
    return _linear(lib().lowra_linear_fwd, "lowra_linear_fwd", OP_LINEAR_FWD, layout, packed, absmax, mappings,
                   x, layout.K, layout.N, A, B, s, y, workspace)


def lowra_linear_fwd_static(layout: Layout, packed, absmax, mappings, x, A, B, s, y):
    """lowra_linear_fwd without a workspace argument (the library's static scratch); `y` [M,N] bf16 is the
    caller's: nothing is allocated here or in the library."""
    _state(layout, packed, absmax, mappings)
    _dev(x, torch.bfloat16, "x"); _dev(y, torch.bfloat16, "y")
    M = int(x.shape[0])
    if tuple(x.shape) != (M, layout.K) or tuple(y.shape) != (M, layout.N):
        raise ValueError("shape mismatch")
    r = 0
    if A is not None and B is not None and A.shape[0] > 0:
        _dev(A, torch.bfloat16, "A"); _dev(B, torch.bfloat16, "B")
        r = int(A.shape[0])
        if tuple(A.shape) != (r, layout.K) or tuple(B.shape) != (layout.N, r):
            raise ValueError("LoRA operand shape mismatch")
    else:
        A = B = None
    _check(lib().lowra_linear_fwd_static(layout.handle, _ptr(packed), _ptr(absmax), _ptr(mappings), _ptr(x), M, _ptr(A),
                                         _ptr(B), r, C.c_float(s), _ptr(y), _stream()), "lowra_linear_fwd_static")
    return y


def lowra_linear_bwd_input(layout: Layout, packed, absmax, mappings, dY, A, B, s, dX=None, workspace=None):
    """dX [M,K] bf16 = dY What + s (dY B) A."""
    if dX is None and workspace is not None and layout.__class__ is Layout:
        res = _call.linear(1, layout.native, packed, absmax, mappings, dY, A, B, s, workspace)
        if res is not None:
            return _native(res, "lowra_linear_bwd_input")
    return _linear(lib().lowra_linear_bwd_input, "lowra_linear_bwd_input", OP_LINEAR_BWD_INPUT, layout, packed,
                   absmax, mappings, dY, layout.N, layout.K, A, B, s, dX, workspace)


def _here(device, *tensors):
    """`device` is the current one, and the tensors are on it."""
    if device.index != torch.cuda.current_device() or any(t.device != device for t in tensors):
        raise ValueError("tensors on another device than the current one")


def _operand(t, shape, name: str, device):
    """An optional bf16 operand of an epilogue."""
    if t is not None:
        _dev(t, torch.bfloat16, name)
        if tuple(t.shape) != shape:
            raise ValueError(f"{name}: shape mismatch")
        if t.device != device:
            raise ValueError(f"{name}: on another device")
    return t


def _linear_act(fn, name, op, layout, packed, absmax, mappings, act_in, cols_in, cols, A, B, s, epilogue, out, workspace):
    """What the two linear calls with an epilogue share: `epilogue(M)` checks the operands and gives their record."""
    _state(layout, packed, absmax, mappings)
    _dev(act_in, torch.bfloat16, "activation")
    if act_in.dim() != 2 or act_in.shape[1] != cols_in:
        raise ValueError("activation shape mismatch")
    _here(act_in.device, packed, absmax, mappings)
    M, r = int(act_in.shape[0]), 0
    if M > 0x7fffffff:
        raise ValueError("too many tokens")
    if A is not None and B is not None and A.shape[0] > 0:
        _dev(A, torch.bfloat16, "A"); _dev(B, torch.bfloat16, "B")
        r = int(A.shape[0])
        if tuple(A.shape) != (r, layout.K) or tuple(B.shape) != (layout.N, r):
            raise ValueError("LoRA operand shape mismatch")
        _here(act_in.device, A, B)
    else:
        A = B = None
    if out is None:
        out = torch.empty((M, cols), dtype=torch.bfloat16, device=act_in.device)
    _operand(out, (M, cols), "out", act_in.device)
    record, second = epilogue(M)
    if workspace is None:
        workspace = torch.empty(layout.workspace_bytes(op, M, r), dtype=torch.uint8, device=act_in.device)
    _here(act_in.device, _dev(workspace, torch.uint8, "workspace"))
    _check(fn(layout.handle, _ptr(packed), _ptr(absmax), _ptr(mappings), _ptr(act_in), M, _ptr(A), _ptr(B), r, float(s), C.addressof(record),
              _ptr(out), _ptr(workspace), workspace.numel(), _stream()), name)
    return out, second


def lowra_linear_fwd_act(layout: Layout, packed, absmax, mappings, x, A, B, s, act: int, bias=None, mul=None, residual=None, keep_z: bool = False,
                         y=None, z=None, workspace=None):
    """v = x What^T + s (x A^T) B^T + bias -> (y, z): y [M,N] bf16 = act(v) mul + residual, and z [M,N] bf16 = v with `keep_z` (or
    where `z` is given), else None.  act: ACT_*; bias [N], mul and residual [M,N] bf16."""
    if y is None and z is None and workspace is not None and layout.__class__ is Layout:
        res = _call.linear_act(0, layout.native, packed, absmax, mappings, x, A, B, s, act, bias, mul, residual, keep_z, workspace)
        if res is not None:
            return _native(res, "lowra_linear_fwd_act")

    def epilogue(M):
        kept, shape = z, (M, layout.N)
        _operand(bias, (layout.N,), "bias", x.device); _operand(mul, shape, "mul", x.device); _operand(residual, shape, "residual", x.device)
        if kept is None and keep_z:
            kept = torch.empty(shape, dtype=torch.bfloat16, device=x.device)
        _operand(kept, shape, "z", x.device)
        return FwdEpilogue(int(act), _ptr(bias), _ptr(mul), _ptr(residual), _ptr(kept)), kept

    return _linear_act(lib().lowra_linear_fwd_act, "lowra_linear_fwd_act", OP_LINEAR_FWD, layout, packed, absmax, mappings, x, layout.K, layout.N,
                       A, B, s, epilogue, y, workspace)


def lowra_linear_bwd_input_act(layout: Layout, packed, absmax, mappings, dY, A, B, s, act: int, z=None, mul=None, residual=None, dX=None, dmul=None,
                               workspace=None, mul_grad: bool = True):
    """g = dY What + s (dY B) A + residual -> (dX, dmul): dX [M,K] bf16 = g mul act'(z), and with `mul` dmul [M,K] bf16 = g act(z), else
    None: the gradients of z and mul of the layer's input act(z) mul.  z, mul, residual: [M,K] bf16; without `mul_grad` (mul is frozen)
    there is no dmul."""
    if dX is None and dmul is None and mul_grad and workspace is not None and layout.__class__ is Layout:
        res = _call.linear_act(1, layout.native, packed, absmax, mappings, dY, A, B, s, act, z, mul, residual, False, workspace)
        if res is not None:
            return _native(res, "lowra_linear_bwd_input_act")

    def epilogue(M):
        second, shape = dmul, (M, layout.K)
        for t, n in ((z, "z"), (mul, "mul"), (residual, "residual")):
            _operand(t, shape, n, dY.device)
        if second is None and mul is not None and mul_grad:
            second = torch.empty(shape, dtype=torch.bfloat16, device=dY.device)
        _operand(second, shape, "dmul", dY.device)
        return BwdEpilogue(int(act), _ptr(z), _ptr(mul), _ptr(residual), _ptr(second)), second

    return _linear_act(lib().lowra_linear_bwd_input_act, "lowra_linear_bwd_input_act", OP_LINEAR_BWD_INPUT, layout, packed, absmax, mappings, dY,
                       layout.N, layout.K, A, B, s, epilogue, dX, workspace)


def lowra_act_bwd_workspace_bytes(M: int, N: int) -> int:
    return int(lib().lowra_act_bwd_workspace_bytes(int(M), int(N)))


def lowra_act_bwd(dY, act: int, z=None, mul=None, bias_grad: bool = False, workspace=None, dZ=None, dmul=None, db=None, mul_grad: bool = True):
    """dY [M,N] bf16, the gradient of act(z) mul -> (dZ, dmul, db): dZ bf16 = dY mul act'(z) (None where it would be dY), dmul bf16 =
    dY act(z) (None without `mul`, or without `mul_grad`: mul is frozen), db fp32 [N] = the sum of dZ over the tokens (None without
    `bias_grad`).  What is given of dZ (dY itself, for one), dmul and db is written there."""
    if dZ is None and dmul is None and db is None and mul_grad and workspace is not None and _lib is not None:
        res = _call.act_bwd(dY, act, z, mul, bias_grad, workspace)
        if res is not None:
            return _native(res, "lowra_act_bwd")
    _dev(dY, torch.bfloat16, "dY")
    if dY.dim() != 2:
        raise ValueError("dY: shape mismatch")
    _here(dY.device)
    shape, act = tuple(dY.shape), int(act)
    M, N = shape
    if max(shape) > 0x7fffffff:
        raise ValueError("dY: too large")
    _operand(z, shape, "z", dY.device); _operand(mul, shape, "mul", dY.device)
    if dZ is None and (act != ACT_NONE or mul is not None):
        dZ = torch.empty_like(dY)
    if dmul is None and mul is not None and mul_grad:
        dmul = torch.empty_like(dY)
    _operand(dZ, shape, "dZ", dY.device); _operand(dmul, shape, "dmul", dY.device)
    if db is not None:
        _here(dY.device, _dev(db, torch.float32, "db"))
        if tuple(db.shape) != (N,):
            raise ValueError("db: shape mismatch")
    elif bias_grad:
        db = torch.empty(N, dtype=torch.float32, device=dY.device)
    if workspace is None:
        workspace = torch.empty(lowra_act_bwd_workspace_bytes(M, N) if db is not None else 0, dtype=torch.uint8, device=dY.device)
    _here(dY.device, _dev(workspace, torch.uint8, "workspace"))
    _check(lib().lowra_act_bwd(M, N, act, _ptr(dY), _ptr(z), _ptr(mul), _ptr(dZ), _ptr(dmul), _ptr(db), _ptr(workspace), workspace.numel(), _stream()),
           "lowra_act_bwd")
    return dZ, dmul, db


def lowra_learn_tables(layout: Layout, W, init_thresholds, init_mappings, iterations: int = 2):
    """W [N,K] fp32, init tables [C,16] fp32 -> (thresholds [N,16], mappings [N,16], mse [N,iterations+1]), all fp32."""
    _dev(W, torch.float32, "W"); _dev(init_thresholds, torch.float32, "init_thresholds"); _dev(init_mappings, torch.float32, "init_mappings")
    if tuple(W.shape) != (layout.N, layout.K) or tuple(init_thresholds.shape) != (layout.C, 16) or \
            tuple(init_mappings.shape) != (layout.C, 16):
        raise ValueError("shape mismatch")
    thr = torch.empty((layout.N, 16), dtype=torch.float32, device=W.device)
    mp = torch.empty((layout.N, 16), dtype=torch.float32, device=W.device)
    mse = torch.empty((layout.N, int(iterations) + 1), dtype=torch.float32, device=W.device)
    _check(lib().lowra_learn_tables(layout.handle, _ptr(W), _ptr(init_thresholds), _ptr(init_mappings), int(iterations),
                                    _ptr(thr), _ptr(mp), _ptr(mse), _stream()), "lowra_learn_tables")
    return thr, mp, mse


def lowra_average_thresholds(layout: Layout, thresholds):
    """In place on thresholds [N,16] fp32: per width, the mean over the channels of that width."""
    _dev(thresholds, torch.float32, "thresholds")
    if tuple(thresholds.shape) != (layout.N, 16):
        raise ValueError("shape mismatch")
    _check(lib().lowra_average_thresholds(layout.handle, _ptr(thresholds), _stream()), "lowra_average_thresholds")
    return thresholds


def lowra_adapter_grads(layout: Layout, x, dY, A, B, s, workspace=None):
    """x [M,K], dY [M,N], A [r,K], B [N,r] bf16 -> (dA fp32 [r,K], dB fp32 [N,r])."""
    if workspace is not None and layout.__class__ is Layout:
        res = _call.grads(layout.native, x, dY, A, B, s, workspace)
        if res is not None:
            return _native(res, "lowra_adapter_grads")
    for t, nme in ((x, "x"), (dY, "dY"), (A, "A"), (B, "B")):
        _dev(t, torch.bfloat16, nme)
    M, r = int(x.shape[0]), int(A.shape[0])
    if tuple(x.shape) != (M, layout.K) or tuple(dY.shape) != (M, layout.N) or tuple(A.shape) != (r, layout.K) or \
            tuple(B.shape) != (layout.N, r):
        raise ValueError("shape mismatch")
    if workspace is None:
        workspace = torch.empty(max(layout.workspace_bytes(OP_ADAPTER_GRADS, M, r), 16), dtype=torch.uint8, device=x.device)
    dA = torch.empty((r, layout.K), dtype=torch.float32, device=x.device)
    dB = torch.empty((layout.N, r), dtype=torch.float32, device=x.device)
    _check(lib().lowra_adapter_grads(layout.handle, _ptr(x), _ptr(dY), M, _ptr(A), _ptr(B), r, float(s), _ptr(dA), _ptr(dB),
                                     _ptr(workspace), workspace.numel(), _stream()), "lowra_adapter_grads")
    return dA, dB


def lowra_linear_side_product(layout: Layout, op: int, M: int, r: int, workspace):
    """The rank-r intermediate a finished linear call left in `workspace`: a bf16 [M,64] view of it, or None."""
    if layout.__class__ is Layout:
        res = _call.side_product(layout.native, op, M, r, workspace)
        if res is not None:
            return res[0]
    _dev(workspace, torch.uint8, "workspace")
    p = lib().lowra_linear_side_product(layout.handle, int(op), int(M), int(r), _ptr(workspace))
    if not p:
        return None
    off = int(p) - workspace.data_ptr()
    return workspace[off:off + M * 64 * 2].view(torch.bfloat16).view(M, 64)


def lowra_adapter_grads_from_side(layout: Layout, x, dY, r, st, su, workspace=None):
    """x [M,K], dY [M,N], st = s x A^T, su = s dY B (bf16 [M,64], from lowra_linear_side_product) -> (dA fp32 [r,K], dB fp32 [N,r])."""
    if workspace is not None and layout.__class__ is Layout:
        res = _call.grads_from_side(layout.native, x, dY, r, st, su, workspace)
        if res is not None:
            return _native(res, "lowra_adapter_grads_from_side")
    for t, nme in ((x, "x"), (dY, "dY"), (st, "st"), (su, "su")):
        _dev(t, torch.bfloat16, nme)
    M, r = int(x.shape[0]), int(r)
    if tuple(x.shape) != (M, layout.K) or tuple(dY.shape) != (M, layout.N) or tuple(st.shape) != (M, 64) or tuple(su.shape) != (M, 64):
        raise ValueError("shape mismatch")
    if workspace is None:
        workspace = torch.empty(max(layout.workspace_bytes(OP_ADAPTER_GRADS, M, r), 16), dtype=torch.uint8, device=x.device)
    dA = torch.empty((r, layout.K), dtype=torch.float32, device=x.device)
    dB = torch.empty((layout.N, r), dtype=torch.float32, device=x.device)
    _check(lib().lowra_adapter_grads_from_side(layout.handle, _ptr(x), _ptr(dY), M, r, _ptr(st), _ptr(su), _ptr(dA), _ptr(dB),
                                               _ptr(workspace), workspace.numel(), _stream()), "lowra_adapter_grads_from_side")
    return dA, dB


def lowra_loftq_init(layout: Layout, W, thresholds, mappings, r, omega, steps=5, power_iterations=16, workspace=None):
    """W fp32 [N,K], omega bf16 [r,K] (random start) -> (packed, absmax, A bf16 [r,K], B bf16 [N,r])."""
    _dev(W, torch.float32, "W"); _dev(thresholds, torch.float32, "thresholds"); _dev(mappings, torch.float32, "mappings")
    if tuple(W.shape) != (layout.N, layout.K):
        raise ValueError("W shape mismatch")
    r = int(r)
    if r > 0:
        _dev(omega, torch.bfloat16, "omega")
        if tuple(omega.shape) != (r, layout.K):
            raise ValueError("omega shape mismatch")
    need = layout.workspace_bytes(OP_LOFTQ_INIT, 0, r) if r > 0 else 0
    if workspace is None:
        workspace = torch.empty(max(need, 16), dtype=torch.uint8, device=W.device)
    packed = torch.empty(max(layout.packed_bytes, 1), dtype=torch.uint8, device=W.device)[:layout.packed_bytes]
    absmax = torch.empty((layout.N, layout.K // 64), dtype=torch.float32, device=W.device)
    A = torch.empty((r, layout.K), dtype=torch.bfloat16, device=W.device)
    B = torch.empty((layout.N, r), dtype=torch.bfloat16, device=W.device)
    _check(lib().lowra_loftq_init(layout.handle, _ptr(W), _ptr(thresholds), _ptr(mappings), r, int(steps), int(power_iterations),
                                  _ptr(omega) if r > 0 else C.c_void_p(0), _ptr(packed), _ptr(absmax), _ptr(A), _ptr(B),
                                  _ptr(workspace), workspace.numel(), _stream()), "lowra_loftq_init")
    return packed, absmax, A, B


class FwdBatch:
    """Several small-token forwards (M <= 16) as one run.  `items`: list of (layout, packed, absmax, x, A, B)
    with A = B = None when r == 0; the outputs y[i] ([M, N_i] bf16) are allocated here.  Every tensor is kept
    alive by the object: the library holds their addresses."""

    def __init__(self, items, mappings, s, workspace=None):
        if not items:
            raise ValueError("empty batch")
        _dev(mappings, torch.float32, "mappings")
        M = int(items[0][3].shape[0])
        r = 0 if items[0][4] is None else int(items[0][4].shape[0])
        self.y, self._keep = [], [mappings]
        arr = (FwdItem * len(items))()
        for i, (layout, packed, absmax, x, A, B) in enumerate(items):
            _dev(packed, torch.uint8, "packed"); _dev(absmax, layout.scale_dtype, "absmax"); _dev(x, torch.bfloat16, "x")
            if tuple(x.shape) != (M, layout.K) or packed.numel() != layout.packed_bytes or absmax.numel() != layout.N * (layout.K // 64):
                raise ValueError(f"item {i}: shape mismatch")
            if r:
                _dev(A, torch.bfloat16, "A"); _dev(B, torch.bfloat16, "B")
                if tuple(A.shape) != (r, layout.K) or tuple(B.shape) != (layout.N, r):
                    raise ValueError(f"item {i}: LoRA shape mismatch")
            y = torch.empty((M, layout.N), dtype=torch.bfloat16, device=x.device)
            arr[i] = FwdItem(layout.handle.value if isinstance(layout.handle, C.c_void_p) else layout.handle,
                             packed.data_ptr(), absmax.data_ptr(), x.data_ptr(),
                             A.data_ptr() if r else 0, B.data_ptr() if r else 0, y.data_ptr())
            self.y.append(y)
            self._keep += [layout, packed, absmax, x, A, B]
        need = int(lib().lowra_fwd_batch_workspace_bytes(len(items), C.addressof(arr), r))
        if workspace is None:
            workspace = torch.empty(max(need, 16), dtype=torch.uint8, device=mappings.device)
        self._keep.append(workspace)
        self.handle = C.c_void_p()
        _check(lib().lowra_fwd_batch_create(len(items), C.addressof(arr), _ptr(mappings), M, r, float(s), _ptr(workspace),
                                            workspace.numel(), C.addressof(self.handle)), "lowra_fwd_batch_create")

    def run(self):
        _check(lib().lowra_fwd_batch_run(self.handle, _stream()), "lowra_fwd_batch_run")
        return self.y

    def close(self):
        if self.handle:
            lib().lowra_fwd_batch_destroy(self.handle)
            self.handle = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class BwdBatch:
    """Several small-token input gradients (M <= 16) as one run.  `items`: list of (layout, packed, absmax, dY, A, B)
    with A = B = None when r == 0; the outputs dX[i] ([M, K_i] bf16) are allocated here.  Every tensor is kept
    alive by the object: the library holds their addresses."""

    def __init__(self, items, mappings, s, workspace=None):
        if not items:
            raise ValueError("empty batch")
        _dev(mappings, torch.float32, "mappings")
        M = int(items[0][3].shape[0])
        r = 0 if items[0][4] is None else int(items[0][4].shape[0])
        self.dX, self._keep = [], [mappings]
        arr = (FwdItem * len(items))()          # same record: layout, packed, absmax, activations in, A, B, out
        for i, (layout, packed, absmax, dY, A, B) in enumerate(items):
            _dev(packed, torch.uint8, "packed"); _dev(absmax, layout.scale_dtype, "absmax"); _dev(dY, torch.bfloat16, "dY")
            if tuple(dY.shape) != (M, layout.N) or packed.numel() != layout.packed_bytes or absmax.numel() != layout.N * (layout.K // 64):
                raise ValueError(f"item {i}: shape mismatch")
            if r:
                _dev(A, torch.bfloat16, "A"); _dev(B, torch.bfloat16, "B")
                if tuple(A.shape) != (r, layout.K) or tuple(B.shape) != (layout.N, r):
                    raise ValueError(f"item {i}: LoRA shape mismatch")
            dX = torch.empty((M, layout.K), dtype=torch.bfloat16, device=dY.device)
            arr[i] = FwdItem(layout.handle.value if isinstance(layout.handle, C.c_void_p) else layout.handle,
                             packed.data_ptr(), absmax.data_ptr(), dY.data_ptr(),
                             A.data_ptr() if r else 0, B.data_ptr() if r else 0, dX.data_ptr())
            self.dX.append(dX)
            self._keep += [layout, packed, absmax, dY, A, B]
        need = int(lib().lowra_bwd_batch_workspace_bytes(len(items), C.addressof(arr), M, r))
        if workspace is None:
            workspace = torch.empty(max(need, 16), dtype=torch.uint8, device=mappings.device)
        self._keep.append(workspace)
        self.handle = C.c_void_p()
        _check(lib().lowra_bwd_batch_create(len(items), C.addressof(arr), _ptr(mappings), M, r, float(s), _ptr(workspace),
                                            workspace.numel(), C.addressof(self.handle)), "lowra_bwd_batch_create")

    def run(self):
        _check(lib().lowra_bwd_batch_run(self.handle, _stream()), "lowra_bwd_batch_run")
        return self.dX

    def close(self):
        if self.handle:
            lib().lowra_bwd_batch_destroy(self.handle)
            self.handle = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


@dataclasses.dataclass
class MuonItem:
    """One matrix of a MuonBatch: fp32 device tensors [rows, cols] (weight_bf16: bf16), the short side at most 64.  `momentum_out` and
    `weight_out` are the tensors themselves where they are not given (in place); without `weight` the batch writes `update` only."""
    grad: torch.Tensor
    momentum: torch.Tensor
    weight: torch.Tensor | None = None
    weight_bf16: torch.Tensor | None = None
    update: torch.Tensor | None = None
    scale: float = 1.0
    momentum_out: torch.Tensor | None = None
    weight_out: torch.Tensor | None = None


class MuonBatch:
    """The optimiser step on a list of MuonItem with the update orthogonalised by Newton-Schulz products (lowra_muon_batch_*).  Every
    tensor is kept alive by the object: the library holds their addresses."""

    def __init__(self, items, workspace=None):
        self.handle = C.c_void_p()
        if not items:
            raise ValueError("empty batch")
        device = items[0].grad.device
        arr = (MuonItemRecord * len(items))()
        self._keep = []
        for i, it in enumerate(items):
            mo = it.momentum if it.momentum_out is None else it.momentum_out
            wo = it.weight if it.weight_out is None else it.weight_out
            fields = (("grad", it.grad, torch.float32), ("momentum", it.momentum, torch.float32), ("momentum_out", mo, torch.float32),
                      ("weight", it.weight, torch.float32), ("weight_out", wo, torch.float32), ("weight_bf16", it.weight_bf16, torch.bfloat16),
                      ("update", it.update, torch.float32))
            for name, t, dtype in fields:
                if t is None and name not in ("grad", "momentum"):
                    continue
                _dev(t, dtype, name)
                if t.dim() != 2 or t.shape != it.grad.shape or t.device != device:
                    raise ValueError(f"item {i}: {name}: shape or device mismatch")
            if max(it.grad.shape) > 0x7fffffff:
                raise ValueError(f"item {i}: too large")
            arr[i] = MuonItemRecord(int(it.grad.shape[0]), int(it.grad.shape[1]), float(it.scale), *(_ptr(t) for _, t, _ in fields))
            self._keep += [t for _, t, _ in fields]
        _here(device)
        need = int(lib().lowra_muon_batch_workspace_bytes(len(items), C.addressof(arr)))
        if workspace is None:
            workspace = torch.empty(max(need, 16), dtype=torch.uint8, device=device)
        _here(device, _dev(workspace, torch.uint8, "workspace"))
        self._keep.append(workspace)
        _check(lib().lowra_muon_batch_create(len(items), C.addressof(arr), _ptr(workspace), workspace.numel(), C.addressof(self.handle)),
               "lowra_muon_batch_create")

    def run(self, lr: float, momentum: float = 0.95, nesterov: bool = True, weight_decay: float = 0.0, steps: int = 5,
            coefficients=(3.4445, -4.7750, 2.0315), eps: float = 1e-7):
        step = MuonStep(lr, momentum, nesterov, weight_decay, steps, *coefficients, eps)
        _check(lib().lowra_muon_batch_run(self.handle, C.addressof(step), _stream()), "lowra_muon_batch_run")

    def close(self):
        if self.handle:
            lib().lowra_muon_batch_destroy(self.handle)
            self.handle = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _rows(t, name: str):
    """A contiguous bf16 device tensor of rows, at most 2^31 - 1 each way, on the current device -> its shape."""
    _dev(t, torch.bfloat16, name)
    if t.dim() != 2 or max(t.shape) > 0x7fffffff:
        raise ValueError(f"{name}: shape mismatch")
    _here(t.device)
    return int(t.shape[0]), int(t.shape[1])


def _typed(t, dtype, shape, name: str, device):
    """An optional tensor of this type, shape and device."""
    if t is not None:
        _here(device, _dev(t, dtype, name))
        if tuple(t.shape) != shape:
            raise ValueError(f"{name}: shape mismatch")
    return t


def lowra_norm_fwd(x, weight=None, bias=None, kind: int = NORM_LAYER, eps: float = 1e-5, y=None):
    """y [M,N] bf16 = (x - mean) / sqrt(mean((x - mean)^2) + eps) weight + bias over the rows of x [M,N] bf16; NORM_RMS: mean = 0.  weight, bias:
    [N] bf16 or None; y may be x."""
    if y is None and _lib is not None:
        res = _call.norm_fwd(x, weight, bias, kind, eps)
        if res is not None:
            return _native(res, "lowra_norm_fwd")
    M, N = _rows(x, "x")
    _operand(weight, (N,), "weight", x.device); _operand(bias, (N,), "bias", x.device)
    if y is None:
        y = torch.empty_like(x)
    _operand(y, (M, N), "y", x.device)
    _check(lib().lowra_norm_fwd(M, N, int(kind), _ptr(x), _ptr(weight), _ptr(bias), float(eps), _ptr(y), _stream()), "lowra_norm_fwd")
    return y


def lowra_norm_bwd_workspace_bytes(M: int, N: int) -> int:
    return int(lib().lowra_norm_bwd_workspace_bytes(int(M), int(N)))


def lowra_norm_bwd(dY, x, weight=None, kind: int = NORM_LAYER, eps: float = 1e-5, residual=None, input_grad: bool = True, weight_grad: bool = False,
                   bias_grad: bool = False, dX=None, dweight=None, dbias=None, workspace=None):
    """The way back of lowra_norm_fwd for dY [M,N] bf16 -> (dX, dweight, dbias): dX bf16 with `residual` [M,N] bf16 added (None without `input_grad`),
    dweight and dbias fp32 [N] (None without `weight_grad`, `bias_grad`).  What is given of the three is written there; dX may be residual."""
    if dX is None and dweight is None and dbias is None and workspace is not None and _lib is not None:
        res = _call.norm_bwd(dY, x, weight, kind, eps, residual, input_grad, weight_grad, bias_grad, workspace)
        if res is not None:
            return _native(res, "lowra_norm_bwd")
    M, N = _rows(dY, "dY")
    device = dY.device
    _operand(x, (M, N), "x", device); _operand(weight, (N,), "weight", device); _operand(residual, (M, N), "residual", device)
    if x is None:
        raise ValueError("x is missing")
    if dX is None and input_grad:
        dX = torch.empty_like(dY)
    _operand(dX, (M, N), "dX", device)
    if dweight is None and weight_grad:
        dweight = torch.empty(N, dtype=torch.float32, device=device)
    if dbias is None and bias_grad:
        dbias = torch.empty(N, dtype=torch.float32, device=device)
    _typed(dweight, torch.float32, (N,), "dweight", device); _typed(dbias, torch.float32, (N,), "dbias", device)
    if workspace is None:
        workspace = torch.empty(lowra_norm_bwd_workspace_bytes(M, N) if dweight is not None or dbias is not None else 0, dtype=torch.uint8, device=device)
    _here(device, _dev(workspace, torch.uint8, "workspace"))
    _check(lib().lowra_norm_bwd(M, N, int(kind), _ptr(dY), _ptr(x), _ptr(weight), float(eps), _ptr(residual), _ptr(dX), _ptr(dweight), _ptr(dbias),
                                _ptr(workspace), workspace.numel(), _stream()), "lowra_norm_bwd")
    return dX, dweight, dbias


def lowra_rope_frequencies(rot: int, base: float = 10000.0, scaling: int = ROPE_SCALE_NONE, factor: float = 1.0, original: int = 0, low: float = 1.0,
                           high: float = 8.0, device="cuda"):
    """The plan of lowra_rope for `rot` columns: the pairs' frequencies base^(-2 j / rot), stretched as `scaling` (ROPE_SCALE_*) says, as an int64
    tensor [rot/2] of 2^-64 turns a position on `device`."""
    turns = np.zeros(max(int(rot) // 2, 1), np.uint64)
    _check(lib().lowra_rope_frequencies(int(rot), float(base), int(scaling), float(factor), int(original), float(low), float(high), turns.ctypes.data),
           "lowra_rope_frequencies")
    return torch.from_numpy(turns.view(np.int64)).to(device)


def lowra_rope(x, positions, turns, layout: int = ROPE_HALF, inverse: bool = False, magnitude: float = 1.0, out=None):
    """Rotary positions of x [M, heads, D] bf16, or of a list of up to four of those (queries and keys) with the same M and D, by positions [M]
    int32 and the plan `turns` (lowra_rope_frequencies), whose length says how many columns are turned.  Tokens and heads may have any stride, the
    columns are contiguous.  `out`: where to write, of the same shapes (x itself: in place); new tensors without it.  `inverse`: the way back."""
    if out is None and _lib is not None:
        res = _call.rope(x, positions, turns, layout, inverse, magnitude)
        if res is not None:
            return _native(res, "lowra_rope")
    many = isinstance(x, (list, tuple))
    xs = list(x) if many else [x]
    if not xs or len(xs) > 4:
        raise ValueError("one to four tensors")
    for t in xs:
        if not (isinstance(t, torch.Tensor) and t.dtype is torch.bfloat16 and t.is_cuda and t.dim() == 3 and (t.stride(2) == 1 or t.shape[2] == 1)):
            raise TypeError("x: need bf16 device tensors [tokens, heads, columns] with contiguous columns")
    M, D, device = int(xs[0].shape[0]), int(xs[0].shape[2]), xs[0].device
    _here(device, *xs, _dev(positions, torch.int32, "positions"), _dev(turns, torch.int64, "turns"))
    if max(M, D) > 0x7fffffff or tuple(positions.shape) != (M,) or turns.dim() != 1:
        raise ValueError("positions or turns: shape mismatch")
    if out is None:
        ys = [torch.empty(t.shape, dtype=torch.bfloat16, device=device) for t in xs]
    else:
        ys = list(out) if isinstance(out, (list, tuple)) else [out]
    if len(ys) != len(xs):
        raise ValueError("out: as many tensors as x")
    arr = (RopeTensor * len(xs))()
    for i, (a, b) in enumerate(zip(xs, ys)):
        if not (b.dtype is torch.bfloat16 and b.is_cuda and b.dim() == 3 and (b.stride(2) == 1 or b.shape[2] == 1)):
            raise TypeError("out: need bf16 device tensors [tokens, heads, columns] with contiguous columns")
        if a.shape != b.shape or a.shape[0] != M or a.shape[2] != D or b.device != device:
            raise ValueError("shape or device mismatch")
        arr[i] = RopeTensor(a.data_ptr(), b.data_ptr(), int(a.shape[1]), a.stride(0), a.stride(1), b.stride(0), b.stride(1))
    _check(lib().lowra_rope(len(xs), C.addressof(arr), M, D, 2 * int(turns.shape[0]), int(layout), _ptr(positions), _ptr(turns), float(magnitude), int(bool(inverse)),
                            _stream()), "lowra_rope")
    return ys if many else ys[0]


def lowra_vocab_loss_workspace_bytes(M: int, V: int, K: int, grad: bool = True) -> int:
    return int(lib().lowra_vocab_loss_workspace_bytes(int(M), int(V), int(K), int(bool(grad))))


def lowra_vocab_loss(h, W, targets, weights=None, grad: bool = True, loss=None, lse=None, dH=None, workspace=None):
    """Cross entropy of h [M,K] bf16 through the frozen head W [V,K] bf16 against targets [M] int32 (outside 0..V-1: no target, loss 0) ->
    (loss fp32 [M], lse fp32 [M], dH bf16 [M,K]): dH is the gradient of the sum of weights loss with respect to h (weights: [M] fp32, None: ones), None
    without `grad`.  targets and weights may begin anywhere (`labels[1:]`): what is not 16-byte aligned is copied first."""
    if loss is None and lse is None and dH is None and workspace is not None and _lib is not None:
        res = _call.vocab_loss(h, W, targets, weights, grad, workspace)
        if res is not None:
            return _native(res, "lowra_vocab_loss")
    M, K = _rows(h, "h")
    V, _ = _rows(W, "W")
    device = h.device
    _here(device, W, _dev(targets, torch.int32, "targets"))
    if W.shape[1] != K or tuple(targets.shape) != (M,):
        raise ValueError("shape mismatch")
    _typed(weights, torch.float32, (M,), "weights", device)
    # the library takes 16-byte aligned ones; labels[1:] beside h[:-1] are not
    targets, weights = (t.clone() if t is not None and t.data_ptr() & 15 else t for t in (targets, weights))
    loss = torch.empty(M, dtype=torch.float32, device=device) if loss is None else loss
    lse = torch.empty(M, dtype=torch.float32, device=device) if lse is None else lse
    _typed(loss, torch.float32, (M,), "loss", device); _typed(lse, torch.float32, (M,), "lse", device)
    if dH is None and grad:
        dH = torch.empty_like(h)
    _operand(dH, (M, K), "dH", device)
    if workspace is None:
        workspace = torch.empty(lowra_vocab_loss_workspace_bytes(M, V, K, dH is not None), dtype=torch.uint8, device=device)
    _here(device, _dev(workspace, torch.uint8, "workspace"))
    _check(lib().lowra_vocab_loss(M, V, K, _ptr(h), _ptr(W), _ptr(targets), _ptr(weights), _ptr(loss), _ptr(lse), _ptr(dH), _ptr(workspace), workspace.numel(),
                                  _stream()), "lowra_vocab_loss")
    return loss, lse, dH


@dataclasses.dataclass
class AdamWItem:
    """One tensor of an AdamWBatch: grad and weight fp32 device tensors of any one shape; m and v fp32 (32-bit states), or m int8 and v uint8 with
    m_absmax and v_absmax fp32 [ceil(elements / 64)] (8-bit states).  The outputs are the tensors themselves where they are not given (in place); weight_bf16: a
    bf16 copy of the new weights."""
    grad: torch.Tensor
    m: torch.Tensor
    v: torch.Tensor
    weight: torch.Tensor
    m_absmax: torch.Tensor | None = None
    v_absmax: torch.Tensor | None = None
    weight_bf16: torch.Tensor | None = None
    lr_scale: float = 1.0
    decay_scale: float = 1.0
    m_out: torch.Tensor | None = None
    v_out: torch.Tensor | None = None
    m_absmax_out: torch.Tensor | None = None
    v_absmax_out: torch.Tensor | None = None
    weight_out: torch.Tensor | None = None


class AdamWBatch:
    """The AdamW step on a list of AdamWItem (lowra_adamw_batch_*).  Every tensor is kept alive by the object: the library holds their addresses."""

    def __init__(self, items):
        self.handle = C.c_void_p()
        if not items:
            raise ValueError("empty batch")
        self.device = device = items[0].grad.device
        arr = (AdamWItemRecord * len(items))()
        self._keep = []
        for i, it in enumerate(items):
            count, shape = it.grad.numel(), it.grad.shape
            eight = it.m.dtype is torch.int8
            groups = torch.Size([(count + 63) // 64])
            own = lambda name: getattr(it, name) if getattr(it, name + "_out") is None else getattr(it, name + "_out")
            fields = [("grad", it.grad, torch.float32, shape), ("m", it.m, torch.int8 if eight else torch.float32, shape),
                      ("v", it.v, torch.uint8 if eight else torch.float32, shape), ("m_absmax", it.m_absmax, torch.float32, groups),
                      ("v_absmax", it.v_absmax, torch.float32, groups), ("weight", it.weight, torch.float32, shape)]
            fields += [(n + "_out", own(n), *next(f[2:] for f in fields if f[0] == n)) for n in ("m", "v", "m_absmax", "v_absmax", "weight")]
            fields.append(("weight_bf16", it.weight_bf16, torch.bfloat16, shape))
            for name, t, dtype, want in fields:
                if t is None and (name == "weight_bf16" or ("absmax" in name and not eight)):
                    continue
                _dev(t, dtype, name)
                if t.shape != want or t.device != device:
                    raise ValueError(f"item {i}: {name}: shape or device mismatch")
            if not eight and any(t is not None for name, t, _, _ in fields if "absmax" in name):
                raise ValueError(f"item {i}: absmax with 32-bit states")
            by = {name: _ptr(t) for name, t, _, _ in fields}
            arr[i] = AdamWItemRecord(count=count, state_bits=8 if eight else 32, lr_scale=float(it.lr_scale), decay_scale=float(it.decay_scale), **by)
            self._keep += [t for _, t, _, _ in fields]
        _here(device)
        _check(lib().lowra_adamw_batch_create(len(items), C.addressof(arr), C.addressof(self.handle)), "lowra_adamw_batch_create")

    def run(self, lr: float, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay: float = 0.01, step: int = 1, grad_scale=None):
        """One step, number `step` from 1; grad_scale: a device tensor of one fp32, a factor of all gradients."""
        if grad_scale is not None:
            _here(self.device, _dev(grad_scale, torch.float32, "grad_scale"))
            if grad_scale.numel() != 1:
                raise ValueError("grad_scale: need one element")
        s = AdamWStep(lr, betas[0], betas[1], eps, weight_decay, step)
        _check(lib().lowra_adamw_batch_run(self.handle, C.addressof(s), _ptr(grad_scale), _stream()), "lowra_adamw_batch_run")

    def close(self):
        if self.handle:
            lib().lowra_adamw_batch_destroy(self.handle)
            self.handle = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def lowra_adamw_state(codes, absmax, out=None):
    """What 8-bit states of an AdamWItem stand for: codes int8 (m) or uint8 (v) of any shape, absmax fp32 [ceil(elements / 64)] -> fp32 of that shape."""
    if codes.dtype not in (torch.int8, torch.uint8):
        raise TypeError("codes: need int8 or uint8")
    _here(codes.device, _dev(codes, codes.dtype, "codes"))
    _typed(absmax, torch.float32, ((codes.numel() + 63) // 64,), "absmax", codes.device)
    if out is None:
        out = torch.empty(codes.shape, dtype=torch.float32, device=codes.device)
    _typed(out, torch.float32, tuple(codes.shape), "out", codes.device)
    _check(lib().lowra_adamw_state(codes.numel(), int(codes.dtype is torch.int8), _ptr(codes), _ptr(absmax), _ptr(out), _stream()), "lowra_adamw_state")
    return out


def lowra_channel_mse(W, thresholds3, mappings3):
    """W [N,K] fp32, tables [3,16] fp32 (rows: 1, 2, 4 bits) -> mse fp32 [N,3]."""
    _dev(W, torch.float32, "W"); _dev(thresholds3, torch.float32, "thresholds3"); _dev(mappings3, torch.float32, "mappings3")
    if W.dim() != 2 or tuple(thresholds3.shape) != (3, 16) or tuple(mappings3.shape) != (3, 16):
        raise ValueError("shape mismatch")
    N, K = W.shape
    mse = torch.empty((N, 3), dtype=torch.float32, device=W.device)
    _check(lib().lowra_channel_mse(int(N), int(K), _ptr(W), _ptr(thresholds3), _ptr(mappings3), _ptr(mse), _stream()),
           "lowra_channel_mse")
    return mse


def lowra_assign_precisions(channel_params, mse, budget_bits_per_param: float) -> np.ndarray:
    """Host only: greedy budgeted assignment. channel_params int64 [N], mse fp32 [N,3] -> bits uint8 [N]."""
    params = np.ascontiguousarray(channel_params, dtype=np.int64)
    mse = np.ascontiguousarray(mse, dtype=np.float32)
    if mse.shape != (params.size, 3):
        raise ValueError("shape mismatch")
    bits = np.zeros(params.size, dtype=np.uint8)
    _check(lib().lowra_assign_precisions(int(params.size), params.ctypes.data, mse.ctypes.data, float(budget_bits_per_param),
                                         bits.ctypes.data), "lowra_assign_precisions")
    return bits


def lowra_set_linear_path(path: int):
    _check(lib().lowra_set_linear_path(int(path)), "lowra_set_linear_path")


def lowra_plan_fwd_tiling(N: int, M: int, compute_units: int = 256):
    """(rows_a, rows_b, cols_a) the forward GEMM's planner picks (host only)."""
    ra, rb, ca = C.c_int(), C.c_int(), C.c_int()
    _check(lib().lowra_plan_fwd_tiling(int(N), int(M), int(compute_units), C.byref(ra), C.byref(rb), C.byref(ca)), "lowra_plan_fwd_tiling")
    return ra.value, rb.value, ca.value


def lowra_set_fwd_tiling(rows_a: int = 0, rows_b: int = 0, cols_a: int = 0):
    _check(lib().lowra_set_fwd_tiling(int(rows_a), int(rows_b), int(cols_a)), "lowra_set_fwd_tiling")


def lowra_set_mid_tiling(rows: int = 0, splits: int = 0):
    _check(lib().lowra_set_mid_tiling(int(rows), int(splits)), "lowra_set_mid_tiling")


def lowra_plan_mid_tiling(op: int, N: int, K: int, M: int, has_4bit: bool, codebooks: int):
    """(rows, splits) of a linear call's mid-token GEMM, (0, 0) where another kernel takes it (host only)."""
    rows, splits = C.c_int(), C.c_int()
    _check(lib().lowra_plan_mid_tiling(int(op), int(N), int(K), int(M), int(has_4bit), int(codebooks), C.byref(rows), C.byref(splits)),
           "lowra_plan_mid_tiling")
    return rows.value, splits.value


def lowra_plan_small_fwd(N: int, K: int, M: int, r: int, batch_strips: int = 0):
    """(wavefronts, rounds, fused) of the general small-token forward (host only)."""
    w, n, f = C.c_int(), C.c_int(), C.c_int()
    _check(lib().lowra_plan_small_fwd(int(N), int(K), int(M), int(r), int(batch_strips), C.byref(w), C.byref(n), C.byref(f)), "lowra_plan_small_fwd")
    return w.value, n.value, bool(f.value)


def lowra_set_kernel_timer(start_event=None, stop_event=None):
    """Measurement hook: raw hipEvent_t handles (ints) recorded around the dominant kernel of linear calls."""
    _check(lib().lowra_set_kernel_timer(C.c_void_p(start_event or 0), C.c_void_p(stop_event or 0)),
           "lowra_set_kernel_timer")


def lowra_measure_copy(dst, src):
    """Measurement kernel: dst = src (uint8 device tensors of equal size, a multiple of 16 bytes)."""
    _check(lib().lowra_measure_copy(_ptr(dst), _ptr(src), C.c_size_t(src.numel() * src.element_size()), _stream()), "lowra_measure_copy")


def lowra_measure_read(src, out4):
    """Measurement kernel: stream src once."""
    _check(lib().lowra_measure_read(_ptr(src), C.c_size_t(src.numel() * src.element_size()), _ptr(out4), _stream()), "lowra_measure_read")


def lowra_measure_mfma(workgroups: int, iterations: int, out4, random_operands: bool = False) -> float:
    """Measurement kernel: a loop of independent bf16 MFMAs on registers (constant operands, or pseudo-random ones
    that change with every instruction); returns its flop count."""
    fl = C.c_double(0.0)
    fn = lib().lowra_measure_mfma_random if random_operands else lib().lowra_measure_mfma
    _check(fn(int(workgroups), int(iterations), _ptr(out4), C.byref(fl), _stream()), "lowra_measure_mfma")
    return float(fl.value)
