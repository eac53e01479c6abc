"""Python binding of libentropack.so (argument marshalling only).

Every step of encoding runs in the library's C++ encoder and every step of
decoding runs in its HIP kernels; this module converts numpy arrays and torch
device tensors to pointers and back.  PyTorch is used only for device memory
and streams.  The library must be built first (``__graft_entry__.build()``);
if it is missing, loading raises instead of falling back to anything else.
"""
from __future__ import annotations

import ctypes as C
import os
import weakref

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libentropack.so")

# ---- constants (mirror include/entropack.h) -------------------------------------
OK, ERR_ARG, ERR_FORMAT, ERR_UNSUPPORTED, ERR_NOMEM, ERR_HIP, ERR_CORRUPT = 0, -1, -2, -3, -4, -5, -6
BF16, FP16, FP32, FP8_E4M3, INT8, FP8_E5M2, UINT8, COORD2_I32 = 1, 2, 3, 4, 5, 6, 7, 100
CONT_DIRECT, CONT_FP8_ROW, CONT_INT8_ROW, CONT_FP8E5M2_ROW, CONT_UINT8_TENSOR = 0, 1, 2, 3, 4
STATUS_PAYLOAD_OVERRUN, STATUS_BAD_FINAL_STATE, STATUS_BAD_END_OFFSET = 1, 2, 4
STATUS_NO_PAGES, STATUS_TABLE_FULL, STATUS_SLOTS_FULL = 8, 16, 32
SCALE_BLOCK, SCALE_ROW_BLOCK, SCALE_ROW = 1, 2, 3
NORM_NONE, NORM_RMS, NORM_LAYER = 0, 1, 2
ACT_SILU, ACT_GELU, ACT_GELU_TANH = 1, 2, 3
ROPE_PLAIN, ROPE_LINEAR, ROPE_BASE, ROPE_TURNS, ROPE_INDEX = 0, 1, 2, 3, 4
ROPE_HALF, ROPE_PAIRS = 1, 2

ITEMSIZE = {BF16: 2, FP16: 2, FP32: 4, FP8_E4M3: 1, INT8: 1, FP8_E5M2: 1, UINT8: 1, COORD2_I32: 4}


class EncodeParams(C.Structure):
    _fields_ = [("target_bpp", C.c_double), ("tile_vectors", C.c_int32),
                ("prob_bits", C.c_int32), ("search_steps", C.c_int32),
                ("container", C.c_int32), ("scale_lo", C.c_double), ("scale_hi", C.c_double),
                ("sample_vectors", C.c_int64), ("state_credit_bits", C.c_double),
                ("nthreads", C.c_int32), ("rdo_candidates", C.c_int32),
                ("rdo_sweeps", C.c_int32), ("reserved", C.c_int32)]


class EncodeStats(C.Structure):
    _fields_ = [("scale", C.c_double), ("rate_estimate_sample", C.c_double),
                ("rate_stored", C.c_double), ("code_length_bits", C.c_double),
                ("erel_coded", C.c_double), ("erel_original", C.c_double),
                ("mean_state_bits", C.c_double), ("bytes", C.c_uint64),
                ("payload_bits", C.c_uint64), ("prob_bits", C.c_uint32),
                ("n_tiles", C.c_uint32), ("max_alphabet", C.c_uint32),
                ("sample_rows", C.c_uint32), ("escalations", C.c_uint32),
                ("coarsenings", C.c_uint32), ("rdo_rows_moved", C.c_uint32),
                ("reserved", C.c_uint32)]


class Blob(C.Structure):
    _fields_ = [("data", C.POINTER(C.c_uint8)), ("size", C.c_uint64)]


class TensorInfo(C.Structure):
    _fields_ = [("rows", C.c_uint32), ("cols", C.c_uint32), ("prob_bits", C.c_uint32),
                ("tile_vectors", C.c_uint32), ("n_tiles", C.c_uint32),
                ("container", C.c_uint32), ("table_bytes", C.c_uint32),
                ("payload_words", C.c_uint32), ("total_bytes", C.c_uint64),
                ("off_tables", C.c_uint64), ("off_sigma", C.c_uint64),
                ("off_delta", C.c_uint64), ("off_states", C.c_uint64),
                ("off_offsets", C.c_uint64), ("off_payload", C.c_uint64),
                ("max_alphabet", C.c_uint32), ("coord2_min", C.c_int32),
                ("coord2_max", C.c_int32), ("max_abs_weight", C.c_float),
                ("path", C.c_uint32), ("sum_alphabet", C.c_uint32),
                ("table_off", C.c_uint32 * 16), ("table_min", C.c_int32 * 16),
                ("table_A", C.c_uint32 * 16), ("coset_f0", C.c_uint32),
                ("coset_f1", C.c_uint32)]


class Layer(C.Structure):
    _fields_ = [("info", TensorInfo), ("d_blob", C.c_void_p), ("d_out", C.c_void_p),
                ("d_dequant", C.c_void_p), ("out_dtype", C.c_int32), ("reserved", C.c_int32)]


class Stack(C.Structure):
    _fields_ = [("d_workspace", C.c_void_p), ("n_layers", C.c_int32), ("path", C.c_uint32),
                ("total_tasks", C.c_uint32), ("lds_bytes", C.c_uint32),
                ("reserved", C.c_uint32 * 4)]


class Kv8Cache(C.Structure):
    _fields_ = [("d_k", C.c_void_p), ("d_v", C.c_void_p), ("d_k_scale", C.c_void_p),
                ("d_v_scale", C.c_void_p), ("n_pages", C.c_int64), ("kv_heads", C.c_int32),
                ("page_tokens", C.c_int32), ("head_dim", C.c_int32), ("dtype", C.c_int32)]


class Kv8Attn(C.Structure):
    _fields_ = [("d_q", C.c_void_p), ("d_out", C.c_void_p), ("d_lse", C.c_void_p),
                ("d_cu_q", C.c_void_p), ("d_len", C.c_void_p), ("d_table", C.c_void_p),
                ("table_ld", C.c_int64), ("n_req", C.c_int64), ("total_q", C.c_int64),
                ("q_row", C.c_int64), ("out_row", C.c_int64), ("q_heads", C.c_int32),
                ("dtype", C.c_int32), ("causal", C.c_int32), ("window", C.c_int32),
                ("max_q", C.c_int32), ("max_len", C.c_int32), ("scale", C.c_float),
                ("reserved", C.c_int32)]


class NormCall(C.Structure):
    _fields_ = [("d_x", C.c_void_p), ("d_res", C.c_void_p), ("d_res_out", C.c_void_p),
                ("d_y", C.c_void_p), ("d_y_scale", C.c_void_p), ("d_post_w", C.c_void_p),
                ("d_post_b", C.c_void_p), ("d_gate", C.c_void_p), ("d_w", C.c_void_p),
                ("d_b", C.c_void_p), ("m", C.c_int64), ("n", C.c_int64), ("x_row", C.c_int64),
                ("res_row", C.c_int64), ("res_out_row", C.c_int64), ("y_row", C.c_int64),
                ("group_rows", C.c_int64), ("gate_ld", C.c_int64), ("w_ld", C.c_int64),
                ("b_ld", C.c_int64), ("x_dtype", C.c_int32), ("res_dtype", C.c_int32),
                ("w_dtype", C.c_int32), ("y_dtype", C.c_int32), ("post", C.c_int32),
                ("pre", C.c_int32), ("w_plus_one", C.c_int32), ("alpha", C.c_float),
                ("eps", C.c_float), ("reserved", C.c_int32)]


class RopeCall(C.Structure):
    _fields_ = [("d_q", C.c_void_p), ("d_q_out", C.c_void_p), ("d_k", C.c_void_p),
                ("d_k_out", C.c_void_p), ("d_freqs", C.c_void_p), ("d_pos", C.c_void_p),
                ("d_cu", C.c_void_p), ("d_len", C.c_void_p), ("n_req", C.c_int64),
                ("n_tokens", C.c_int64), ("q_row", C.c_int64), ("q_out_row", C.c_int64),
                ("k_row", C.c_int64), ("k_out_row", C.c_int64), ("q_heads", C.c_int32),
                ("k_heads", C.c_int32), ("head_dim", C.c_int32), ("rot_first", C.c_int32),
                ("rot_dim", C.c_int32), ("layout", C.c_int32), ("dtype", C.c_int32),
                ("inverse", C.c_int32), ("amplitude", C.c_float), ("reserved", C.c_int32)]


class EntroPackError(RuntimeError):
    def __init__(self, code: int, what: str, msg: str):
        super().__init__(f"{what}: status {code}: {msg}")
        self.code = code


_lib = None


def lib():
    """The loaded native library (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with __graft_entry__.build()")
        L = C.CDLL(LIB_PATH)
        vp, u32, i32, i64, u64 = C.c_void_p, C.c_uint32, C.c_int32, C.c_int64, C.c_uint64
        L.ep_encode_params_default.argtypes = [C.POINTER(EncodeParams)]
        L.ep_encode_params_default.restype = None
        L.ep_encode_cpu.argtypes = [vp, C.c_int, i64, i64, C.POINTER(EncodeParams),
                                    C.POINTER(Blob), C.POINTER(EncodeStats)]
        L.ep_encode_gpu.argtypes = [vp, C.c_int, i64, i64, C.POINTER(EncodeParams),
                                    C.POINTER(Blob), C.POINTER(EncodeStats), vp]
        L.ep_blob_free.argtypes = [C.POINTER(Blob)]
        L.ep_blob_free.restype = None
        L.ep_blob_info.argtypes = [vp, u64, C.POINTER(TensorInfo)]
        L.ep_decode_tiles.argtypes = [C.POINTER(TensorInfo), vp, C.c_int, vp, vp, u32, u32, vp, vp]
        L.ep_decode_layers_workspace.argtypes = [C.c_int]
        L.ep_decode_layers_workspace.restype = u64
        L.ep_decode_layers.argtypes = [C.POINTER(Layer), C.c_int, vp, u64, vp, vp]
        L.ep_decode_layers_noalloc.argtypes = [C.POINTER(Layer), C.c_int, vp, vp]
        L.ep_stack_workspace.argtypes = [C.c_int]
        L.ep_stack_workspace.restype = u64
        L.ep_stack_prepare.argtypes = [C.POINTER(Layer), C.c_int, vp, u64, C.POINTER(Stack), vp]
        L.ep_stack_decode.argtypes = [C.POINTER(Stack), vp, vp]
        L.ep_gemm_i8_nt.argtypes = [vp, vp, vp, i64, i64, i64, vp]
        L.ep_decode_matmul_i8.argtypes = [C.POINTER(TensorInfo), vp, vp, C.c_int, vp, vp, vp, vp]
        L.ep_decode_gemm_i8.argtypes = [C.POINTER(TensorInfo), vp, vp, i64, vp, vp, vp, u64, vp, vp]
        L.ep_decode_gemm_i8_prepared.argtypes = [C.POINTER(TensorInfo), vp, vp, i64, vp, vp, vp, u64,
                                                 vp, vp]
        L.ep_decode_gemm_i8_prepare.argtypes = [C.POINTER(TensorInfo), vp, vp, u64, vp]
        L.ep_decode_gemm_bf16.argtypes = [C.POINTER(TensorInfo), vp, vp, i64, vp, vp, vp, u64, vp, vp]
        L.ep_decode_gemm_bf16_prepared.argtypes = [C.POINTER(TensorInfo), vp, vp, i64, vp, vp, vp, u64,
                                                   vp, vp]
        L.ep_decode_gemm_bf16_prepare.argtypes = [C.POINTER(TensorInfo), vp, vp, u64, vp]
        L.ep_decode_gemm_bf16_workspace.argtypes = [C.POINTER(TensorInfo)]
        L.ep_decode_gemm_bf16_workspace.restype = u64
        L.ep_decode_gemm_i8_workspace.argtypes = [C.POINTER(TensorInfo)]
        L.ep_decode_gemm_i8_workspace.restype = u64
        L.ep_quant_fp8_block.argtypes = [vp, C.c_int, i64, i64, i64, C.c_int, vp, vp, vp]
        L.ep_gemm_fp8_block.argtypes = [vp, vp, vp, C.c_int, vp, C.c_int, vp, C.c_int, i64, i64, i64, vp]
        L.ep_kv8_slots.argtypes = [vp, vp, i64, C.c_int, vp, vp, vp, i64, vp, vp, vp, i64, vp, vp, vp]
        L.ep_kv8_append.argtypes = [C.POINTER(Kv8Cache), vp, vp, C.c_int, i64, i64, vp, i64, vp]
        L.ep_kv8_attention_workspace.argtypes = [C.POINTER(Kv8Cache), C.POINTER(Kv8Attn)]
        L.ep_kv8_attention_workspace.restype = u64
        L.ep_kv8_attention.argtypes = [C.POINTER(Kv8Cache), C.POINTER(Kv8Attn), vp, u64, vp]
        L.ep_quant_i8_row.argtypes = [vp, C.c_int, i64, i64, i64, vp, vp, vp]
        L.ep_gemm_i8_scaled.argtypes = [vp, vp, vp, vp, vp, vp, C.c_int, i64, i64, i64, vp, u64, vp]
        L.ep_gemm_i8_scaled_workspace.argtypes = [i64, i64, i64]
        L.ep_gemm_i8_scaled_workspace.restype = u64
        L.ep_norm.argtypes = [C.POINTER(NormCall), vp]
        L.ep_glu.argtypes = [vp, vp, C.c_int, i64, i64, i64, i64, C.c_int, vp, C.c_int, vp, vp]
        L.ep_rope_freqs.argtypes = [C.c_int, C.c_double, C.c_int, C.c_double, C.c_double, C.c_double,
                                    C.c_double, vp]
        L.ep_rope.argtypes = [C.POINTER(RopeCall), vp]
        L.ep_last_error.restype = C.c_char_p
        _lib = L
    return _lib


EXPORTS = ["ep_encode_params_default", "ep_encode_cpu", "ep_encode_gpu", "ep_blob_free", "ep_blob_info",
           "ep_decode_tiles", "ep_decode_layers_workspace", "ep_decode_layers",
           "ep_decode_layers_noalloc",
           "ep_stack_workspace", "ep_stack_prepare", "ep_stack_decode", "ep_gemm_i8_nt",
           "ep_decode_matmul_i8", "ep_decode_gemm_i8", "ep_decode_gemm_i8_workspace",
           "ep_decode_gemm_i8_prepare", "ep_decode_gemm_i8_prepared",
           "ep_decode_gemm_bf16", "ep_decode_gemm_bf16_workspace", "ep_decode_gemm_bf16_prepare",
           "ep_decode_gemm_bf16_prepared",
           "ep_quant_fp8_block", "ep_gemm_fp8_block", "ep_kv8_slots", "ep_kv8_append",
           "ep_kv8_attention_workspace", "ep_kv8_attention",
           "ep_quant_i8_row", "ep_gemm_i8_scaled", "ep_gemm_i8_scaled_workspace", "ep_norm", "ep_glu",
           "ep_rope_freqs", "ep_rope",
           "ep_last_error"]


def _check(rc: int, what: str):
    if rc != OK:
        raise EntroPackError(rc, what, lib().ep_last_error().decode())


def default_params(target_bpp: float, **kw) -> EncodeParams:
    p = EncodeParams()
    lib().ep_encode_params_default(C.byref(p))
    p.target_bpp = float(target_bpp)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def _blob_array(out: Blob) -> np.ndarray:
    """The blob the library allocated, as a uint8 numpy array over the same memory (no
    copy); ep_blob_free releases it once no array refers to that memory any more."""
    addr = C.cast(out.data, C.c_void_p).value
    buf = (C.c_uint8 * out.size).from_address(addr)
    weakref.finalize(buf, _free_blob, addr, out.size)
    return np.frombuffer(buf, dtype=np.uint8)


def _free_blob(addr: int, size: int) -> None:
    b = Blob(C.cast(addr, C.POINTER(C.c_uint8)), size)
    lib().ep_blob_free(C.byref(b))


def encode(w: np.ndarray, target_bpp: float, dtype: int | None = None, **kw):
    """Encode an R x C matrix (uint16 BF16 bits, or float32; FP16 bits with dtype=FP16).
    Returns (blob as a uint8 numpy array over the library's memory, no copy; stats dict)."""
    w = np.ascontiguousarray(w)
    if dtype is None:
        dtype = FP32 if w.dtype == np.float32 else BF16
    p = default_params(target_bpp, **kw)
    out = Blob()
    st = EncodeStats()
    _check(lib().ep_encode_cpu(w.ctypes.data_as(C.c_void_p), dtype, w.shape[0], w.shape[1],
                               C.byref(p), C.byref(out), C.byref(st)), "ep_encode_cpu")
    return _blob_array(out), {k: getattr(st, k) for k, _ in EncodeStats._fields_}


def encode_gpu(d_w: int, rows: int, cols: int, target_bpp: float, dtype: int = BF16,
               stream: int = 0, **kw):
    """Encode an R x C device matrix (pointer d_w: BF16/FP16 bits or FP32) with the GPU
    encoder.  Returns (blob as a uint8 numpy array, stats dict), as encode()."""
    p = default_params(target_bpp, **kw)
    out = Blob()
    st = EncodeStats()
    _check(lib().ep_encode_gpu(d_w, dtype, rows, cols, C.byref(p), C.byref(out), C.byref(st),
                               stream or None), "ep_encode_gpu")
    return _blob_array(out), {k: getattr(st, k) for k, _ in EncodeStats._fields_}


def blob_info(blob: np.ndarray) -> TensorInfo:
    info = TensorInfo()
    b = np.ascontiguousarray(blob, dtype=np.uint8)
    _check(lib().ep_blob_info(b.ctypes.data_as(C.c_void_p), b.size, C.byref(info)), "ep_blob_info")
    return info


def decode_tiles(info: TensorInfo, d_blob: int, out_dtype: int, d_out: int, d_dequant: int = 0,
                 tile_begin: int = 0, tile_end: int | None = None, d_status: int = 0,
                 stream: int = 0):
    """Raw entry point: all buffers are device addresses (ints)."""
    if tile_end is None:
        tile_end = info.n_tiles
    _check(lib().ep_decode_tiles(C.byref(info), d_blob, out_dtype, d_out, d_dequant or None,
                                 tile_begin, tile_end, d_status or None, stream or None),
           "ep_decode_tiles")


def decode_layers_workspace(n: int) -> int:
    return int(lib().ep_decode_layers_workspace(n))


def _layer_array(layers):
    arr = (Layer * len(layers))()
    for i, (info, blob, out, dq, dt) in enumerate(layers):
        arr[i].info = info
        arr[i].d_blob = blob
        arr[i].d_out = out
        arr[i].d_dequant = dq or None
        arr[i].out_dtype = dt
    return arr


def decode_layers(layers, d_ws: int, ws_bytes: int, d_status: int = 0, stream: int = 0):
    """layers: sequence of (TensorInfo, d_blob, d_out, d_dequant, out_dtype)."""
    arr = _layer_array(layers)
    _check(lib().ep_decode_layers(arr, len(layers), d_ws, ws_bytes, d_status or None,
                                  stream or None), "ep_decode_layers")


def decode_layers_noalloc(layers, d_status: int = 0, stream: int = 0):
    """As decode_layers, with the descriptors in the library's static device array (no
    workspace, no allocation; at most 512 layers)."""
    arr = _layer_array(layers)
    _check(lib().ep_decode_layers_noalloc(arr, len(layers), d_status or None, stream or None),
           "ep_decode_layers_noalloc")


def stack_workspace(n: int) -> int:
    return int(lib().ep_stack_workspace(n))


def stack_prepare(layers, d_ws: int, ws_bytes: int, stream: int = 0) -> Stack:
    """Write the device descriptors of `layers` once; returns the prepared stack."""
    st = Stack()
    arr = _layer_array(layers)
    _check(lib().ep_stack_prepare(arr, len(layers), d_ws, ws_bytes, C.byref(st), stream or None),
           "ep_stack_prepare")
    return st


def stack_decode(st: Stack, d_status: int = 0, stream: int = 0):
    _check(lib().ep_stack_decode(C.byref(st), d_status or None, stream or None), "ep_stack_decode")


def gemm_i8_nt(d_a: int, d_b: int, d_y: int, m: int, n: int, k: int, stream: int = 0):
    _check(lib().ep_gemm_i8_nt(d_a, d_b, d_y, m, n, k, stream or None), "ep_gemm_i8_nt")


def decode_matmul_i8(info: TensorInfo, d_blob: int, d_x: int, m: int, d_y: int, d_dequant: int = 0,
                     d_status: int = 0, stream: int = 0):
    """Y (m x R int32) = X (m x C int8) times the decoded INT8 container matrix, transposed."""
    _check(lib().ep_decode_matmul_i8(C.byref(info), d_blob, d_x, m, d_y, d_dequant or None,
                                     d_status or None, stream or None), "ep_decode_matmul_i8")


def decode_gemm_i8_workspace(info: TensorInfo) -> int:
    return int(lib().ep_decode_gemm_i8_workspace(C.byref(info)))


def decode_gemm_i8(info: TensorInfo, d_blob: int, d_x: int, m: int, d_y: int, d_ws: int,
                   ws_bytes: int, d_dequant: int = 0, d_status: int = 0, stream: int = 0):
    """Y (m x R int32) = X (m x C int8) times the decoded INT8 container matrix, transposed,
    on the matrix cores, for any m (the fused decode and MFMA product)."""
    _check(lib().ep_decode_gemm_i8(C.byref(info), d_blob, d_x, m, d_y, d_dequant or None, d_ws,
                                   ws_bytes, d_status or None, stream or None), "ep_decode_gemm_i8")


def decode_gemm_i8_prepare(info: TensorInfo, d_blob: int, d_ws: int, ws_bytes: int, stream: int = 0):
    """Build the tensor's decode tables once into the workspace (synchronous)."""
    _check(lib().ep_decode_gemm_i8_prepare(C.byref(info), d_blob, d_ws, ws_bytes, stream or None),
           "ep_decode_gemm_i8_prepare")


def decode_gemm_i8_prepared(info: TensorInfo, d_blob: int, d_x: int, m: int, d_y: int, d_ws: int,
                            ws_bytes: int, d_dequant: int = 0, d_status: int = 0, stream: int = 0):
    """decode_gemm_i8 on a workspace that decode_gemm_i8_prepare filled for this blob."""
    _check(lib().ep_decode_gemm_i8_prepared(C.byref(info), d_blob, d_x, m, d_y, d_dequant or None,
                                            d_ws, ws_bytes, d_status or None, stream or None),
           "ep_decode_gemm_i8_prepared")


def decode_gemm_bf16_workspace(info: TensorInfo) -> int:
    return int(lib().ep_decode_gemm_bf16_workspace(C.byref(info)))


def decode_gemm_bf16(info: TensorInfo, d_blob: int, d_x: int, m: int, d_y: int, d_ws: int,
                     ws_bytes: int, d_dequant: int = 0, d_status: int = 0, stream: int = 0):
    """Y (m x R fp32) = X (m x C bf16) times the tensor's bf16 decode, transposed, on the
    matrix cores, for any m (the fused decode and BF16 MFMA product)."""
    _check(lib().ep_decode_gemm_bf16(C.byref(info), d_blob, d_x, m, d_y, d_dequant or None, d_ws,
                                     ws_bytes, d_status or None, stream or None), "ep_decode_gemm_bf16")


def decode_gemm_bf16_prepare(info: TensorInfo, d_blob: int, d_ws: int, ws_bytes: int, stream: int = 0):
    """Build the tensor's decode tables once into the workspace (synchronous)."""
    _check(lib().ep_decode_gemm_bf16_prepare(C.byref(info), d_blob, d_ws, ws_bytes, stream or None),
           "ep_decode_gemm_bf16_prepare")


def decode_gemm_bf16_prepared(info: TensorInfo, d_blob: int, d_x: int, m: int, d_y: int, d_ws: int,
                              ws_bytes: int, d_dequant: int = 0, d_status: int = 0, stream: int = 0):
    """decode_gemm_bf16 on a workspace that decode_gemm_bf16_prepare filled for this blob."""
    _check(lib().ep_decode_gemm_bf16_prepared(C.byref(info), d_blob, d_x, m, d_y, d_dequant or None,
                                              d_ws, ws_bytes, d_status or None, stream or None),
           "ep_decode_gemm_bf16_prepared")


def quant_fp8_block(d_x: int, x_dtype: int, m: int, k: int, d_q: int, d_scale: int,
                    block_rows: int = 1, x_row: int | None = None, stream: int = 0):
    """X (m x k, rows x_row elements apart) to E4M3 codes and FP32 scales of its blocks of
    block_rows x 128."""
    _check(lib().ep_quant_fp8_block(d_x or None, x_dtype, m, k, k if x_row is None else x_row, block_rows,
                                    d_q or None, d_scale or None, stream or None), "ep_quant_fp8_block")


def gemm_fp8_block(d_x: int, d_x_scale: int, d_w: int, d_w_scale: int, d_y: int, m: int, n: int,
                   k: int, w_dtype: int = FP8_E4M3, w_scales: int = SCALE_BLOCK, y_dtype: int = BF16,
                   stream: int = 0):
    """Y (m x n) = X (m x k E4M3) times W (n x k FP8) transposed, with X's scales for each row
    and block of 128 and W's in layout w_scales."""
    _check(lib().ep_gemm_fp8_block(d_x or None, d_x_scale or None, d_w or None, w_dtype,
                                   d_w_scale or None, w_scales, d_y or None, y_dtype, m, n, k,
                                   stream or None), "ep_gemm_fp8_block")


def kv8_cache(d_k: int, d_v: int, d_k_scale: int, d_v_scale: int, n_pages: int, kv_heads: int,
              page_tokens: int, head_dim: int, dtype: int = FP8_E4M3) -> Kv8Cache:
    """Describe one layer's paged 8-bit cache (the arrays stay the caller's)."""
    return Kv8Cache(d_k, d_v, d_k_scale, d_v_scale, n_pages, kv_heads, page_tokens, head_dim, dtype)


def kv8_slots(d_cached: int, d_new: int, n_req: int, page_tokens: int, d_free: int, d_n_free: int,
              d_table: int, table_ld: int, d_len: int, d_cu: int, d_slots: int, n_slots: int,
              d_used: int, d_status: int = 0, stream: int = 0):
    """Pages and slots of the new tokens of n_req requests (block tables, slot map, lengths)."""
    _check(lib().ep_kv8_slots(d_cached or None, d_new or None, n_req, page_tokens, d_free or None,
                              d_n_free or None, d_table or None, table_ld, d_len or None, d_cu or None,
                              d_slots or None, n_slots, d_used or None, d_status or None,
                              stream or None), "ep_kv8_slots")


def kv8_append(cache: Kv8Cache, d_k: int, d_v: int, dtype: int, k_row: int, v_row: int, d_slots: int,
               n_tokens: int, stream: int = 0):
    """Quantise n_tokens keys and values into their slots of the cache."""
    _check(lib().ep_kv8_append(C.byref(cache), d_k or None, d_v or None, dtype, k_row, v_row,
                               d_slots or None, n_tokens, stream or None), "ep_kv8_append")


def kv8_attention_args(d_q: int, d_out: int, d_cu_q: int, d_len: int, d_table: int, table_ld: int,
                       n_req: int, total_q: int, q_heads: int, dtype: int, scale: float,
                       causal: bool = True, window: int = 0, max_q: int = 1, max_len: int = 1,
                       q_row: int = 0, out_row: int = 0, d_lse: int = 0) -> Kv8Attn:
    """Describe one attention call.  q_row and out_row are elements from one token to the next
    (0: packed rows of q_heads x head_dim)."""
    return Kv8Attn(d_q or None, d_out or None, d_lse or None, d_cu_q or None, d_len or None,
                   d_table or None, table_ld, n_req, total_q, q_row, out_row, q_heads, dtype, int(causal),
                   window, max_q, max_len, scale, 0)


def kv8_attention_workspace(cache: Kv8Cache, call: Kv8Attn) -> int:
    return int(lib().ep_kv8_attention_workspace(C.byref(cache), C.byref(call)))


def kv8_attention(cache: Kv8Cache, call: Kv8Attn, d_ws: int, ws_bytes: int, stream: int = 0):
    """Attention of call's queries over the cache."""
    _check(lib().ep_kv8_attention(C.byref(cache), C.byref(call), d_ws or None, ws_bytes,
                                  stream or None), "ep_kv8_attention")


def quant_i8_row(d_x: int, x_dtype: int, m: int, k: int, d_q: int, d_scale: int,
                 x_row: int | None = None, stream: int = 0):
    """X (m x k, rows x_row elements apart) to INT8 codes and an FP32 scale for each row."""
    _check(lib().ep_quant_i8_row(d_x or None, x_dtype, m, k, k if x_row is None else x_row, d_q or None,
                                 d_scale or None, stream or None), "ep_quant_i8_row")


def gemm_i8_scaled_workspace(m: int, n: int, k: int) -> int:
    """Bytes that gemm_i8_scaled needs for these sizes; fewer rows may need more.  1 MiB for each CU is
    enough for all."""
    return int(lib().ep_gemm_i8_scaled_workspace(m, n, k))


def gemm_i8_scaled(d_x: int, d_x_scale: int, d_w: int, d_w_scale: int, d_y: int, m: int, n: int, k: int,
                   y_dtype: int = BF16, d_bias: int = 0, d_ws: int = 0, ws_bytes: int = 0, stream: int = 0):
    """Y (m x n) = X (m x k INT8) times W (n x k INT8) transposed, with a scale for each row of both
    and an FP32 bias."""
    _check(lib().ep_gemm_i8_scaled(d_x or None, d_x_scale or None, d_w or None, d_w_scale or None,
                                   d_bias or None, d_y or None, y_dtype, m, n, k, d_ws or None, ws_bytes,
                                   stream or None), "ep_gemm_i8_scaled")


def norm_call(d_x: int, m: int, n: int, x_dtype: int = BF16, d_res: int = 0, d_res_out: int = 0,
              res_dtype: int = BF16, d_y: int = 0, y_dtype: int = BF16, d_y_scale: int = 0,
              post: int = NORM_NONE, d_post_w: int = 0, d_post_b: int = 0, d_gate: int = 0, gate_ld: int = 0,
              alpha: float = 1.0, pre: int = NORM_RMS, d_w: int = 0, d_b: int = 0, w_ld: int = 0, b_ld: int = 0,
              w_dtype: int = BF16, group_rows: int = 0, w_plus_one: bool = False, eps: float = 1e-6,
              x_row: int = 0, res_row: int = 0, res_out_row: int = 0, y_row: int = 0) -> NormCall:
    """Describe one call of norm: h = res + alpha gate N_post(x), y = N_pre(h).  Rows are n elements
    apart where their distance is 0."""
    return NormCall(d_x or None, d_res or None, d_res_out or None, d_y or None, d_y_scale or None,
                    d_post_w or None, d_post_b or None, d_gate or None, d_w or None, d_b or None, m, n,
                    x_row, res_row, res_out_row, y_row, group_rows, gate_ld, w_ld, b_ld, x_dtype, res_dtype,
                    w_dtype, y_dtype, post, pre, int(w_plus_one), alpha, eps, 0)


def norm(call: NormCall, stream: int = 0):
    """The norm after one block, the residual sum and the norm before the next."""
    _check(lib().ep_norm(C.byref(call), stream or None), "ep_norm")


def glu(d_a: int, d_b: int, x_dtype: int, m: int, n: int, act: int, d_y: int, y_dtype: int = BF16,
        d_y_scale: int = 0, a_row: int | None = None, b_row: int | None = None, stream: int = 0):
    """Y (m x n) = act(A) * B, or act(A) without B, rounded or quantised."""
    _check(lib().ep_glu(d_a or None, d_b or None, x_dtype, m, n, n if a_row is None else a_row,
                        n if b_row is None else b_row, act, d_y or None, y_dtype, d_y_scale or None,
                        stream or None), "ep_glu")


def rope_freqs(rot_dim: int, base: float = 10000.0, stretch: int = ROPE_PLAIN, factor: float = 1.0,
               trained_len: float = 0.0, low: float = 0.0, high: float = 0.0) -> np.ndarray:
    """Frequencies of rot_dim / 2 pairs as fractions of a turn in 64 bits (host array, uint64)."""
    out = np.zeros(max(0, rot_dim // 2), dtype=np.uint64)
    _check(lib().ep_rope_freqs(rot_dim, base, stretch, factor, trained_len, low, high,
                               out.ctypes.data_as(C.c_void_p)), "ep_rope_freqs")
    return out


def rope_call(d_q: int, d_q_out: int, d_freqs: int, n_tokens: int, q_heads: int, head_dim: int, dtype: int,
              d_k: int = 0, d_k_out: int = 0, k_heads: int = 0, rot_dim: int = 0, rot_first: int = 0,
              layout: int = ROPE_HALF, d_pos: int = 0, d_cu: int = 0, d_len: int = 0, n_req: int = 0,
              q_row: int = 0, q_out_row: int = 0, k_row: int = 0, k_out_row: int = 0, inverse: bool = False,
              amplitude: float = 1.0) -> RopeCall:
    """Describe one rotation of queries and keys (rot_dim 0: whole heads; rows packed where their
    distance is 0), positions in d_pos or from ep_kv8_slots' d_cu and d_len."""
    return RopeCall(d_q or None, d_q_out or None, d_k or None, d_k_out or None, d_freqs or None,
                    d_pos or None, d_cu or None, d_len or None, n_req, n_tokens, q_row, q_out_row, k_row,
                    k_out_row, q_heads, k_heads, head_dim, rot_first, rot_dim or head_dim, layout, dtype,
                    int(inverse), amplitude, 0)


def rope(call: RopeCall, stream: int = 0):
    """Rotate call's queries and keys by their positions."""
    _check(lib().ep_rope(C.byref(call), stream or None), "ep_rope")


# ---- torch conveniences (device memory and streams only) ------------------------
def _torch():
    import torch
    return torch


TORCH_DTYPE = {}


def torch_dtype(code: int):
    t = _torch()
    return {BF16: t.bfloat16, FP16: t.float16, FP32: t.float32, FP8_E4M3: t.float8_e4m3fn,
            INT8: t.int8, FP8_E5M2: t.float8_e5m2, UINT8: t.uint8, COORD2_I32: t.int32}[code]


def to_device(blob: np.ndarray, device="cuda"):
    t = _torch()
    return t.from_numpy(np.ascontiguousarray(blob, dtype=np.uint8)).to(device)


def decode(blob: np.ndarray, out_dtype: int, d_blob=None, tile_begin=0, tile_end=None,
           out=None, dequant=None, status=None, info=None):
    """Decode a blob on the current CUDA/HIP device into a new (or given) torch tensor.
    Returns (out, dequant or None, status tensor)."""
    t = _torch()
    info = info or blob_info(blob)
    if d_blob is None:
        d_blob = to_device(blob)
    if out is None:
        out = t.zeros((info.rows, info.cols), dtype=torch_dtype(out_dtype), device=d_blob.device)
    if dequant is None and info.container:
        dequant = t.zeros(info.rows, dtype=t.float32, device=d_blob.device)
    if status is None:
        status = t.zeros(1, dtype=t.int32, device=d_blob.device)
    stream = t.cuda.current_stream(d_blob.device).cuda_stream
    decode_tiles(info, d_blob.data_ptr(), out_dtype, out.data_ptr(),
                 dequant.data_ptr() if dequant is not None else 0, tile_begin, tile_end,
                 status.data_ptr(), stream)
    return out, dequant, status
