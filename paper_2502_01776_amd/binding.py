"""ctypes binding of include/svg.h: same names, argument marshalling only.

Device tensors are torch tensors (used for memory and streams only); every step of
the path runs inside the library's kernels.  There is no fallback: if the shared
object is missing, loading raises.
"""
from __future__ import annotations

import ctypes as C
import os

import numpy as np
import torch  # noqa: F401  -- must come first: the library binds to the HIP runtime torch has loaded

_HERE = os.path.dirname(os.path.abspath(__file__))
# SVG_LIBRARY_PATH selects another build of the same library (e.g. to time two builds side by side)
LIB_PATH = os.environ.get("SVG_LIBRARY_PATH") or os.path.join(_HERE, "libsvg_gfx950.so")

SVG_HEAD_SPATIAL = 0
SVG_HEAD_TEMPORAL = 1
SVG_LIST_TEMPORAL_FRAME_MAJOR = 2   # list pattern only: temporal mask without the layout transformation
SVG_NORM_NONE, SVG_NORM_RMS, SVG_NORM_LAYER = 0, 1, 2           # svg_qk_norm_rope
SVG_ROPE_INTERLEAVED, SVG_ROPE_HALF = 0, 1
SVG_FP8_Q, SVG_FP8_K, SVG_FP8_VT, SVG_FP8_SCALES = 0, 1, 2, 3   # svg_fp8_buffer_bytes
SVG_ATTN_QO_TOKEN_ORDER = 1          # svg_sparse_attn_fwd_ex: q read and o written in token order
SVG_ATTN_ELEMENT_MASK = 2            # svg_sparse_attn_fwd_ex: the pattern's element mask inside every visited tile
SVG_ATTN_KV_TOKEN_ORDER = 4          # svg_sparse_attn_fwd_ex: k, v of temporal heads stay in token order (gathered in the kernel)
SVG_BF16, SVG_F16, SVG_F32 = 0, 1, 2                            # element types of the operators around the attention
SVG_FP4_CODES, SVG_FP4_SCALES = 0, 1                            # svg_fp4_buffer_bytes
SVG_ACT_NONE, SVG_ACT_SILU, SVG_ACT_GELU_TANH = 0, 1, 2
SVG_KV4_OK, SVG_KV4_FULL, SVG_KV4_LENGTHS, SVG_KV4_PAGES = 0, 1, 2, 3      # status of svg_kv4_resize
SVG_OK = 0

EXPORTS = ("svg_strerror", "svg_version", "svg_last_hip_error", "svg_workspace_bytes", "svg_profile_plan", "svg_tile_counts",
           "svg_tile_list_build", "svg_profile_heads", "svg_profile_heads_static", "svg_layout_fwd", "svg_layout_inv",
           "svg_sparse_attn_fwd", "svg_sparse_attn_fwd_ex", "svg_dense_attn_fwd",
           "svg_layout_kv_temporal", "svg_sparse_attn_fwd_kv2",
           "svg_fp8_buffer_bytes", "svg_fp8_quantize", "svg_sparse_attn_fp8_fwd", "svg_qk_norm_rope",
           "svg_probe_mfma_bf16", "svg_probe_lds",
           "svg_gate_norm_fwd", "svg_gate_norm_workspace_bytes", "svg_gate_norm_bwd",
           "svg_fp4_buffer_bytes", "svg_fp4_quantize", "svg_fp4_dequantize",
           "svg_fp4_linear_workspace_bytes", "svg_fp4_linear", "svg_fp4_linear_quantize", "svg_fp4_linear_rows",
           "svg_kv4_bytes", "svg_kv4_resize", "svg_kv4_write", "svg_kv4_read", "svg_kv4_attn_workspace_bytes", "svg_kv4_attn_fwd")


class SvgShape(C.Structure):
    _fields_ = [("B", C.c_int32), ("H", C.c_int32), ("F", C.c_int32), ("P", C.c_int32),
                ("T", C.c_int32), ("D", C.c_int32), ("text_first", C.c_int32),
                ("w_s", C.c_int32), ("w_t", C.c_int32), ("sink_first_frame", C.c_int32),
                ("block_m", C.c_int32), ("block_n", C.c_int32), ("softmax_scale", C.c_float)]

    @property
    def N(self):
        return self.F * self.P + self.T


class SvgGateNorm(C.Structure):
    _fields_ = [("rows", C.c_int64), ("C", C.c_int32), ("groups", C.c_int32), ("stream_type", C.c_int32),
                ("branch_type", C.c_int32), ("post_norm", C.c_int32), ("pre_norm", C.c_int32),
                ("residual_scale", C.c_float), ("post_eps", C.c_float), ("eps", C.c_float), ("reserved", C.c_int32),
                ("ld_x", C.c_int64), ("ld_y", C.c_int64), ("ld_r", C.c_int64), ("ld_h", C.c_int64), ("ld_mod", C.c_int64),
                ("gate", C.c_void_p), ("scale", C.c_void_p), ("shift", C.c_void_p), ("group_ptr", C.c_void_p),
                ("post_weight", C.c_void_p), ("post_bias", C.c_void_p), ("weight", C.c_void_p), ("bias", C.c_void_p)]


class SvgGateNormGrads(C.Structure):
    _fields_ = [("ld_mod", C.c_int64), ("gate", C.c_void_p), ("scale", C.c_void_p), ("shift", C.c_void_p),
                ("post_weight", C.c_void_p), ("post_bias", C.c_void_p), ("weight", C.c_void_p), ("bias", C.c_void_p)]


class SvgTokens(C.Structure):
    _fields_ = [("B", C.c_int64), ("N", C.c_int64), ("H", C.c_int32), ("D", C.c_int32), ("stride_b", C.c_int64),
                ("stride_n", C.c_int64), ("stride_h", C.c_int64), ("type", C.c_int32), ("reserved", C.c_int32)]


class SvgKv4(C.Structure):
    _fields_ = [("B", C.c_int32), ("H", C.c_int32), ("D", C.c_int32), ("page_size", C.c_int32), ("pages", C.c_int32),
                ("max_pages", C.c_int32), ("reserved", C.c_int64), ("data", C.c_void_p), ("page_table", C.c_void_p)]


class SvgKv4Attn(C.Structure):
    _fields_ = [("softmax_scale", C.c_float), ("causal", C.c_int32), ("block", C.c_int32), ("window", C.c_int32), ("sink", C.c_int32),
                ("max_kv", C.c_int32), ("kv_len", C.c_void_p), ("q_len", C.c_void_p)]
    sequences = None          # lengths that the descriptor was made with, where they are known


class SvgError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        detail = f": {lib().svg_last_hip_error().decode()}" if status == -5 else ""
        super().__init__(f"{where}: {svg_strerror(status)} ({status}){detail}")


_lib = None


def lib():
    """The loaded shared object.  Raises FileNotFoundError if it was never built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(
                f"{LIB_PATH} not found: build it with `python -m paper_2502_01776_amd.build` "
                "(there is no CPU fallback)")
        L = C.CDLL(LIB_PATH)
        sp = C.POINTER(SvgShape)
        vp, i32p = C.c_void_p, C.POINTER(C.c_int32)
        L.svg_strerror.restype = C.c_char_p
        L.svg_strerror.argtypes = [C.c_int]
        L.svg_version.restype = C.c_char_p
        L.svg_version.argtypes = []
        L.svg_last_hip_error.restype = C.c_char_p
        L.svg_last_hip_error.argtypes = []
        L.svg_workspace_bytes.restype = C.c_size_t
        L.svg_workspace_bytes.argtypes = [sp, C.c_int32]
        L.svg_profile_plan.restype = C.c_int
        L.svg_profile_plan.argtypes = [sp, C.c_int32, i32p, i32p, i32p]
        L.svg_tile_counts.restype = C.c_int
        L.svg_tile_counts.argtypes = [sp, i32p, i32p]
        L.svg_tile_list_build.restype = C.c_int
        L.svg_tile_list_build.argtypes = [sp, C.c_int, vp, vp, C.c_int64, C.POINTER(C.c_int64)]
        L.svg_profile_heads.restype = C.c_int
        L.svg_profile_heads.argtypes = [sp, vp, vp, vp, vp, C.c_int32, vp, vp, vp, C.c_size_t, vp]
        L.svg_profile_heads_static.restype = C.c_int
        L.svg_profile_heads_static.argtypes = [sp, vp, vp, vp, vp, C.c_int32, vp, vp, vp]
        for name in ("svg_layout_fwd", "svg_layout_inv"):
            f = getattr(L, name)
            f.restype = C.c_int
            f.argtypes = [sp, vp, vp, vp, vp]
        L.svg_sparse_attn_fwd.restype = C.c_int
        L.svg_sparse_attn_fwd.argtypes = [sp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, C.c_size_t, vp]
        L.svg_sparse_attn_fwd_ex.restype = C.c_int
        L.svg_sparse_attn_fwd_ex.argtypes = [sp, vp, vp, vp, vp, vp, vp, vp, vp, vp, C.c_uint32, vp, C.c_size_t, vp]
        L.svg_layout_kv_temporal.restype = C.c_int
        L.svg_layout_kv_temporal.argtypes = [sp, vp, vp, vp, vp, vp, vp]
        L.svg_sparse_attn_fwd_kv2.restype = C.c_int
        L.svg_sparse_attn_fwd_kv2.argtypes = [sp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, C.c_uint32, vp]
        L.svg_qk_norm_rope.restype = C.c_int
        L.svg_qk_norm_rope.argtypes = [sp, vp, vp, C.c_int, vp, vp, C.c_float, vp, vp, C.c_int, vp]
        L.svg_fp8_buffer_bytes.restype = C.c_size_t
        L.svg_fp8_buffer_bytes.argtypes = [sp, C.c_int]
        L.svg_fp8_quantize.restype = C.c_int
        L.svg_fp8_quantize.argtypes = [sp, vp, vp, vp, vp, vp, vp, vp, vp, vp]
        L.svg_sparse_attn_fp8_fwd.restype = C.c_int
        L.svg_sparse_attn_fp8_fwd.argtypes = [sp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp]
        L.svg_probe_mfma_bf16.restype = C.c_int
        L.svg_probe_mfma_bf16.argtypes = [C.c_int, C.c_int32, C.c_int32, vp, vp, C.POINTER(C.c_double), vp]
        L.svg_probe_lds.restype = C.c_int
        L.svg_probe_lds.argtypes = [C.c_int, C.c_int32, C.c_int32, vp, C.c_size_t, vp]
        L.svg_dense_attn_fwd.restype = C.c_int
        L.svg_dense_attn_fwd.argtypes = [sp, vp, vp, vp, vp, vp, C.c_size_t, vp]
        gp, tp, i64 = C.POINTER(SvgGateNorm), C.POINTER(SvgTokens), C.c_int64
        L.svg_gate_norm_fwd.restype = C.c_int
        L.svg_gate_norm_fwd.argtypes = [gp, vp, vp, vp, vp, vp, vp, vp]
        L.svg_gate_norm_workspace_bytes.restype = C.c_size_t
        L.svg_gate_norm_workspace_bytes.argtypes = [gp]
        L.svg_gate_norm_bwd.restype = C.c_int
        L.svg_gate_norm_bwd.argtypes = [gp, vp, vp, vp, vp, vp, vp, C.POINTER(SvgGateNormGrads), vp, C.c_size_t, vp]
        L.svg_fp4_buffer_bytes.restype = C.c_size_t
        L.svg_fp4_buffer_bytes.argtypes = [i64, i64, C.c_int]
        L.svg_fp4_quantize.restype = C.c_int
        L.svg_fp4_quantize.argtypes = [tp, vp, C.c_int, vp, vp, vp]
        L.svg_fp4_dequantize.restype = C.c_int
        L.svg_fp4_dequantize.argtypes = [tp, vp, vp, vp, vp]
        L.svg_fp4_linear_workspace_bytes.restype = C.c_size_t
        L.svg_fp4_linear_workspace_bytes.argtypes = [i64, i64, i64]
        L.svg_fp4_linear.restype = C.c_int
        L.svg_fp4_linear.argtypes = [i64, i64, i64, vp, vp, vp, vp, vp, C.c_int, tp, vp, vp, C.c_size_t, vp]
        L.svg_fp4_linear_quantize.restype = C.c_int
        L.svg_fp4_linear_quantize.argtypes = [i64, i64, i64, vp, vp, vp, vp, vp, C.c_int, vp, vp, vp, C.c_size_t, vp]
        L.svg_fp4_linear_rows.restype = C.c_int
        L.svg_fp4_linear_rows.argtypes = [tp, vp, C.c_int, i64, vp, vp, vp, C.c_int, tp, vp, vp]
        kp, ap = C.POINTER(SvgKv4), C.POINTER(SvgKv4Attn)
        L.svg_kv4_bytes.restype = C.c_size_t
        L.svg_kv4_bytes.argtypes = [kp]
        L.svg_kv4_resize.restype = C.c_int
        L.svg_kv4_resize.argtypes = [kp, vp, vp, vp, vp, vp, vp, vp, C.c_int32, vp, vp]
        L.svg_kv4_write.restype = C.c_int
        L.svg_kv4_write.argtypes = [kp, tp, vp, tp, vp, vp, vp]
        L.svg_kv4_read.restype = C.c_int
        L.svg_kv4_read.argtypes = [kp, vp, tp, vp, tp, vp, vp]
        L.svg_kv4_attn_workspace_bytes.restype = C.c_size_t
        L.svg_kv4_attn_workspace_bytes.argtypes = [kp, ap, tp]
        L.svg_kv4_attn_fwd.restype = C.c_int
        L.svg_kv4_attn_fwd.argtypes = [kp, ap, tp, vp, tp, vp, vp, vp, C.c_size_t, vp]
        _lib = L
    return _lib


def shape_from_config(cfg: dict, **overrides) -> SvgShape:
    keys = ("B", "H", "F", "P", "T", "D", "text_first", "w_s", "w_t", "sink_first_frame",
            "block_m", "block_n")
    vals = {k: int(cfg[k]) for k in keys}
    vals.update(overrides)
    return SvgShape(softmax_scale=float(cfg.get("softmax_scale", 0.0)), **vals)


def _check(status, where):
    if status != SVG_OK:
        raise SvgError(status, where)


def _ptr(x):
    """Device (or host) address of a torch tensor / numpy array / int / None."""
    if x is None:
        return None
    if isinstance(x, torch.Tensor):
        return x.data_ptr()
    if isinstance(x, int):
        return x
    if isinstance(x, np.ndarray):
        return x.ctypes.data
    return x.data_ptr()


# The current stream's handle as torch's own launchers ask for it.  torch.cuda.current_stream() builds a Stream object,
# 2.8 us of the 7.5 a call with one kernel takes on the host (now 4.9); the handle alone takes 0.2.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_current_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream):
    if stream is None:
        if _raw_stream is not None and _current_device is not None and torch.cuda.is_initialized():
            return _raw_stream(_current_device())
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def svg_strerror(status: int) -> str:
    return lib().svg_strerror(int(status)).decode()


def svg_version() -> str:
    return lib().svg_version().decode()


def svg_workspace_bytes(shape: SvgShape, t: int) -> int:
    return int(lib().svg_workspace_bytes(C.byref(shape), int(t)))


def svg_profile_plan(shape: SvgShape, t: int):
    """Returns (n_full, n_masked, full_bound[0 .. n_full])."""
    nf, nm = C.c_int32(), C.c_int32()
    bound = (C.c_int32 * 17)()
    _check(lib().svg_profile_plan(C.byref(shape), int(t), C.byref(nf), C.byref(nm), bound), "svg_profile_plan")
    return nf.value, nm.value, list(bound)[:nf.value + 1]


def svg_tile_counts(shape: SvgShape):
    nq, nk = C.c_int32(), C.c_int32()
    _check(lib().svg_tile_counts(C.byref(shape), C.byref(nq), C.byref(nk)), "svg_tile_counts")
    return nq.value, nk.value


def svg_tile_list_build(shape: SvgShape, pattern: int):
    """Host CSR (row_ptr int32[nq+1], col_idx int32[nnz]) as numpy arrays."""
    nq, _ = svg_tile_counts(shape)
    row_ptr = np.zeros(nq + 1, dtype=np.int32)
    nnz = C.c_int64()
    _check(lib().svg_tile_list_build(C.byref(shape), int(pattern), row_ptr.ctypes.data, None, 0,
                                     C.byref(nnz)), "svg_tile_list_build")
    col_idx = np.zeros(max(nnz.value, 1), dtype=np.int32)
    _check(lib().svg_tile_list_build(C.byref(shape), int(pattern), row_ptr.ctypes.data,
                                     col_idx.ctypes.data, nnz.value, C.byref(nnz)),
           "svg_tile_list_build")
    return row_ptr, col_idx[:nnz.value]


def svg_profile_heads(shape, q, k, v, rows, t, labels, mse, workspace, workspace_bytes, stream=None):
    _check(lib().svg_profile_heads(C.byref(shape), _ptr(q), _ptr(k), _ptr(v), _ptr(rows), int(t),
                                   _ptr(labels), _ptr(mse), _ptr(workspace), int(workspace_bytes),
                                   _stream(stream)), "svg_profile_heads")


SVG_STATIC_SCRATCH_BYTES = 160 << 20


def svg_profile_heads_static(shape, q, k, v, rows, t, labels, mse, stream=None):
    _check(lib().svg_profile_heads_static(C.byref(shape), _ptr(q), _ptr(k), _ptr(v), _ptr(rows), int(t),
                                          _ptr(labels), _ptr(mse), _stream(stream)), "svg_profile_heads_static")


def svg_layout_fwd(shape, x, out, labels=None, stream=None):
    _check(lib().svg_layout_fwd(C.byref(shape), _ptr(x), _ptr(out), _ptr(labels), _stream(stream)),
           "svg_layout_fwd")


def svg_layout_inv(shape, x, out, labels=None, stream=None):
    _check(lib().svg_layout_inv(C.byref(shape), _ptr(x), _ptr(out), _ptr(labels), _stream(stream)),
           "svg_layout_inv")


def svg_sparse_attn_fwd(shape, q, k, v, o, labels, row_ptr_s, col_idx_s, row_ptr_t, col_idx_t,
                        workspace=None, workspace_bytes=0, stream=None):
    _check(lib().svg_sparse_attn_fwd(C.byref(shape), _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(labels),
                                     _ptr(row_ptr_s), _ptr(col_idx_s), _ptr(row_ptr_t),
                                     _ptr(col_idx_t), _ptr(workspace), int(workspace_bytes),
                                     _stream(stream)), "svg_sparse_attn_fwd")


def svg_sparse_attn_fwd_ex(shape, q, k, v, o, labels, row_ptr_s, col_idx_s, row_ptr_t, col_idx_t,
                           flags=0, workspace=None, workspace_bytes=0, stream=None):
    _check(lib().svg_sparse_attn_fwd_ex(C.byref(shape), _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(labels),
                                        _ptr(row_ptr_s), _ptr(col_idx_s), _ptr(row_ptr_t),
                                        _ptr(col_idx_t), int(flags), _ptr(workspace),
                                        int(workspace_bytes), _stream(stream)), "svg_sparse_attn_fwd_ex")


def svg_layout_kv_temporal(shape, k, v, k_t, v_t, labels, stream=None):
    _check(lib().svg_layout_kv_temporal(C.byref(shape), _ptr(k), _ptr(v), _ptr(k_t), _ptr(v_t), _ptr(labels),
                                        _stream(stream)), "svg_layout_kv_temporal")


def svg_sparse_attn_fwd_kv2(shape, q, k, v, k_t, v_t, o, labels, row_ptr_s, col_idx_s, row_ptr_t, col_idx_t,
                            flags=0, stream=None):
    _check(lib().svg_sparse_attn_fwd_kv2(C.byref(shape), _ptr(q), _ptr(k), _ptr(v), _ptr(k_t), _ptr(v_t), _ptr(o),
                                         _ptr(labels), _ptr(row_ptr_s), _ptr(col_idx_s), _ptr(row_ptr_t),
                                         _ptr(col_idx_t), int(flags), _stream(stream)), "svg_sparse_attn_fwd_kv2")


def svg_dense_attn_fwd(shape, q, k, v, o, workspace=None, workspace_bytes=0, stream=None):
    _check(lib().svg_dense_attn_fwd(C.byref(shape), _ptr(q), _ptr(k), _ptr(v), _ptr(o),
                                    _ptr(workspace), int(workspace_bytes), _stream(stream)),
           "svg_dense_attn_fwd")


def svg_fp8_buffer_bytes(shape, which) -> int:
    return int(lib().svg_fp8_buffer_bytes(C.byref(shape), int(which)))


def svg_fp8_quantize(shape, q, k, v, labels, q8, k8, v8t, scales, stream=None):
    _check(lib().svg_fp8_quantize(C.byref(shape), _ptr(q), _ptr(k), _ptr(v), _ptr(labels), _ptr(q8),
                                  _ptr(k8), _ptr(v8t), _ptr(scales), _stream(stream)), "svg_fp8_quantize")


def svg_sparse_attn_fp8_fwd(shape, q8, k8, v8t, scales, o, labels, row_ptr_s, col_idx_s, row_ptr_t,
                            col_idx_t, stream=None):
    _check(lib().svg_sparse_attn_fp8_fwd(C.byref(shape), _ptr(q8), _ptr(k8), _ptr(v8t), _ptr(scales),
                                         _ptr(o), _ptr(labels), _ptr(row_ptr_s), _ptr(col_idx_s),
                                         _ptr(row_ptr_t), _ptr(col_idx_t), _stream(stream)),
           "svg_sparse_attn_fp8_fwd")


def svg_qk_norm_rope(shape, x, y, norm=SVG_NORM_NONE, weight=None, bias=None, eps=1e-6, cos=None, sin=None,
                     pairing=SVG_ROPE_INTERLEAVED, stream=None):
    _check(lib().svg_qk_norm_rope(C.byref(shape), _ptr(x), _ptr(y), int(norm), _ptr(weight), _ptr(bias),
                                  float(eps), _ptr(cos), _ptr(sin), int(pairing), _stream(stream)),
           "svg_qk_norm_rope")


def svg_probe_mfma_bf16(form, workgroups, iterations, operands, sink, stream=None) -> float:
    """Enqueues the matrix-core rate probe; returns the floating point operations of the launch."""
    flop = C.c_double()
    _check(lib().svg_probe_mfma_bf16(int(form), int(workgroups), int(iterations), _ptr(operands), _ptr(sink),
                                     C.byref(flop), _stream(stream)), "svg_probe_mfma_bf16")
    return flop.value


def svg_probe_lds(form, waves, iterations, scratch, stream=None) -> int:
    """Enqueues the LDS rate probe; returns the bytes one wave instruction of this form moves.  Entry w of
    scratch (viewed as int64) receives the shader clocks wavefront w took."""
    _check(lib().svg_probe_lds(int(form), int(waves), int(iterations), _ptr(scratch),
                               scratch.numel() * scratch.element_size(), _stream(stream)), "svg_probe_lds")
    return 1024 if form in (0, 3) else 512


# ---- around the attention ----------------------------------------------------------------------

_TYPE_OF = {torch.bfloat16: SVG_BF16, torch.float16: SVG_F16, torch.float32: SVG_F32}


def gate_norm_desc(rows, channels, groups=1, group_ptr=None, stream_type=SVG_BF16, branch_type=SVG_BF16, post_norm=SVG_NORM_NONE,
                   pre_norm=SVG_NORM_NONE, residual_scale=1.0, post_eps=1e-6, eps=1e-6, ld_x=0, ld_y=0, ld_r=0, ld_h=0, ld_mod=0,
                   gate=None, scale=None, shift=None, post_weight=None, post_bias=None, weight=None, bias=None) -> SvgGateNorm:
    """The descriptor of svg_gate_norm_fwd / _bwd; tables and weights as fp32 tensors, which the caller keeps alive."""
    return SvgGateNorm(rows, channels, groups, stream_type, branch_type, post_norm, pre_norm, residual_scale, post_eps, eps, 0,
                       ld_x, ld_y, ld_r, ld_h, ld_mod, _ptr(gate), _ptr(scale), _ptr(shift), _ptr(group_ptr),
                       _ptr(post_weight), _ptr(post_bias), _ptr(weight), _ptr(bias))


def gate_norm_grads(gate=None, scale=None, shift=None, post_weight=None, post_bias=None, weight=None, bias=None,
                    ld_mod=0) -> SvgGateNormGrads:
    return SvgGateNormGrads(ld_mod, _ptr(gate), _ptr(scale), _ptr(shift), _ptr(post_weight), _ptr(post_bias), _ptr(weight),
                            _ptr(bias))


def tokens_of(x) -> SvgTokens:
    """The token matrix of a tensor [rows, columns] or [B, H, N, D] with neighbouring last elements."""
    shape, stride, kind = x.shape, x.stride(), _TYPE_OF.get(x.dtype)
    if len(shape) not in (2, 4):
        raise ValueError("a token matrix is [rows, columns] or [B, H, N, D]")
    if stride[-1] != 1 and shape[-1] > 1:
        raise ValueError("the elements of a row (of a head) have to be neighbours")
    if kind is None:
        raise ValueError(f"a token matrix has no element type {x.dtype}: bfloat16, float16 or float32")
    if len(shape) == 2:
        return SvgTokens(1, shape[0], 1, shape[1], 0, stride[0], 0, kind)
    return SvgTokens(shape[0], shape[2], shape[1], shape[3], stride[0], stride[2], stride[1], kind)


def svg_gate_norm_fwd(desc, x, y, r, h, codes=None, scales=None, stream=None):
    _check(lib().svg_gate_norm_fwd(C.byref(desc), _ptr(x), _ptr(y), _ptr(r), _ptr(h), _ptr(codes), _ptr(scales), _stream(stream)),
           "svg_gate_norm_fwd")


def svg_gate_norm_workspace_bytes(desc) -> int:
    return int(lib().svg_gate_norm_workspace_bytes(C.byref(desc)))


def svg_gate_norm_bwd(desc, r, y, dr, dh, dx, dy, grads=None, workspace=None, workspace_bytes=0, stream=None):
    _check(lib().svg_gate_norm_bwd(C.byref(desc), _ptr(r), _ptr(y), _ptr(dr), _ptr(dh), _ptr(dx), _ptr(dy),
                                   C.byref(grads) if grads is not None else None, _ptr(workspace), int(workspace_bytes),
                                   _stream(stream)), "svg_gate_norm_bwd")


def svg_fp4_buffer_bytes(rows, cols, which) -> int:
    return int(lib().svg_fp4_buffer_bytes(int(rows), int(cols), int(which)))


def svg_fp4_quantize(tokens, x, activation, codes, scales, stream=None):
    _check(lib().svg_fp4_quantize(C.byref(tokens), _ptr(x), int(activation), _ptr(codes), _ptr(scales), _stream(stream)),
           "svg_fp4_quantize")


def svg_fp4_dequantize(tokens, codes, scales, x, stream=None):
    _check(lib().svg_fp4_dequantize(C.byref(tokens), _ptr(codes), _ptr(scales), _ptr(x), _stream(stream)), "svg_fp4_dequantize")


def svg_fp4_linear_workspace_bytes(M, N, K) -> int:
    return int(lib().svg_fp4_linear_workspace_bytes(int(M), int(N), int(K)))


def svg_fp4_linear(M, N, K, a, a_scales, w, w_scales, bias, activation, out_tokens, out, workspace=None, workspace_bytes=0,
                   stream=None):
    _check(lib().svg_fp4_linear(M, N, K, _ptr(a), _ptr(a_scales), _ptr(w), _ptr(w_scales), _ptr(bias), int(activation),
                                C.byref(out_tokens), _ptr(out), _ptr(workspace), int(workspace_bytes), _stream(stream)),
           "svg_fp4_linear")


def svg_fp4_linear_quantize(M, N, K, a, a_scales, w, w_scales, bias, activation, codes, scales, workspace=None, workspace_bytes=0,
                            stream=None):
    _check(lib().svg_fp4_linear_quantize(M, N, K, _ptr(a), _ptr(a_scales), _ptr(w), _ptr(w_scales), _ptr(bias), int(activation),
                                         _ptr(codes), _ptr(scales), _ptr(workspace), int(workspace_bytes), _stream(stream)),
           "svg_fp4_linear_quantize")


def svg_fp4_linear_rows(x_tokens, x, in_activation, N, w, w_scales, bias, activation, out_tokens, out, stream=None):
    _check(lib().svg_fp4_linear_rows(C.byref(x_tokens), _ptr(x), int(in_activation), int(N), _ptr(w), _ptr(w_scales), _ptr(bias),
                                     int(activation), C.byref(out_tokens), _ptr(out), _stream(stream)), "svg_fp4_linear_rows")


# ---- a cache of keys and values in 4 bits ---------------------------------------------------------

def _whole(x, kind, name, count=None):
    """Address of a tensor that the device reads or writes as it lies; count: how many elements there have to be."""
    if not isinstance(x, torch.Tensor):
        return _ptr(x)
    if x.dtype is not kind or not x.is_contiguous():
        raise ValueError(f"{name} has to be a contiguous tensor of {kind}")
    if count is not None and x.numel() != count:
        raise ValueError(f"{name} has to have {count} elements, not {x.numel()}")
    return x.data_ptr()


def kv4_cache(sequences, pages, max_pages, heads, head_dim, page_size, data=None, page_table=None) -> SvgKv4:
    """The descriptor of a cache: `pages` pages of `page_size` tokens, `max_pages` entries in a row of the page table.  The caller keeps
    data (uint8, svg_kv4_bytes) and page_table (int32 [sequences, max_pages]) alive."""
    if isinstance(data, torch.Tensor):
        need = pages * heads * page_size * (head_dim + head_dim // 16)
        if not data.is_contiguous() or data.numel() * data.element_size() < need:
            raise ValueError(f"a cache of this size has {need} bytes in one run")
    return SvgKv4(sequences, heads, head_dim, page_size, pages, max_pages, 0, _ptr(data),
                  _whole(page_table, torch.int32, "page_table", sequences * max_pages))


def kv4_attn(kv_len, q_len=None, max_kv=0, causal=False, block=1, window=-1, sink=0, softmax_scale=0.0) -> SvgKv4Attn:
    """The descriptor of svg_kv4_attn_fwd; lengths as int32 tensors [sequences], which the caller keeps alive."""
    attn = SvgKv4Attn(softmax_scale, int(causal), block, window, sink, max_kv, _whole(kv_len, torch.int32, "kv_len"), None)
    if isinstance(kv_len, torch.Tensor):
        attn.sequences = kv_len.numel()
    attn.q_len = _whole(q_len, torch.int32, "q_len", attn.sequences)
    return attn


def svg_kv4_bytes(cache) -> int:
    return int(lib().svg_kv4_bytes(C.byref(cache)))


def svg_kv4_resize(cache, lengths, wanted, free_pages, free_count, new_lengths, new_count, slots, tokens, status, stream=None):
    i32, n = torch.int32, cache.B
    _check(lib().svg_kv4_resize(C.byref(cache), _whole(lengths, i32, "lengths", n), _whole(wanted, i32, "wanted", n),
                                _whole(free_pages, i32, "free_pages", cache.pages), _whole(free_count, i32, "free_count", 1),
                                _whole(new_lengths, i32, "new_lengths", n), _whole(new_count, i32, "new_count", 1),
                                _whole(slots, torch.int64, "slots", n * tokens), int(tokens), _whole(status, i32, "status", 1),
                                _stream(stream)), "svg_kv4_resize")


def svg_kv4_write(cache, k_tokens, k, v_tokens, v, slots, stream=None):
    _check(lib().svg_kv4_write(C.byref(cache), C.byref(k_tokens), _ptr(k), C.byref(v_tokens), _ptr(v),
                               _whole(slots, torch.int64, "slots", k_tokens.B * k_tokens.N), _stream(stream)), "svg_kv4_write")


def svg_kv4_read(cache, slots, k_tokens, k, v_tokens, v, stream=None):
    _check(lib().svg_kv4_read(C.byref(cache), _whole(slots, torch.int64, "slots", k_tokens.B * k_tokens.N), C.byref(k_tokens), _ptr(k),
                              C.byref(v_tokens), _ptr(v), _stream(stream)), "svg_kv4_read")


def svg_kv4_attn_workspace_bytes(cache, attn, q_tokens) -> int:
    return int(lib().svg_kv4_attn_workspace_bytes(C.byref(cache), C.byref(attn), C.byref(q_tokens)))


def svg_kv4_attn_fwd(cache, attn, q_tokens, q, o_tokens, o, lse=None, workspace=None, workspace_bytes=0, stream=None):
    if attn.sequences not in (None, cache.B):
        raise ValueError(f"kv_len has {attn.sequences} lengths for {cache.B} sequences")
    if lse is not None:
        lse = _whole(lse, torch.float32, "lse", q_tokens.B * q_tokens.N * (q_tokens.H * q_tokens.D // max(cache.D, 1)))
    _check(lib().svg_kv4_attn_fwd(C.byref(cache), C.byref(attn), C.byref(q_tokens), _ptr(q), C.byref(o_tokens), _ptr(o), lse,
                                  _ptr(workspace), int(workspace_bytes), _stream(stream)), "svg_kv4_attn_fwd")
