"""Thin ctypes binding over the C ABI in include/lba.h, lba_layer.h and lba_attention.h (argument marshalling only).

Every step of the computation runs in the HIP library; there is no CPU fallback: if the library
has not been built, loading raises.  torch is used for device memory and for the current stream.
"""
import ctypes
import functools
import math
import os
import typing

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIBPATH = os.path.join(_HERE, "liblba_hip.so")

ROUND_FLOOR, ROUND_RNE = 0, 1
STE_IDENTITY, STE_IMMEDIATE_OF, STE_RECURSIVE_OF, STE_COEF_PLANE = 0, 1, 2, 3
ORDER_SEQ, ORDER_CHUNK16 = 0, 1
ACT_NONE, ACT_RELU, ACT_GELU, ACT_SILU = 0, 1, 2, 3
F32, BF16, CODE8 = 0, 1, 2
FINE = 0x100                                             # may be added to the type of attention's inputs
OK, ERR_NULL, ERR_SHAPE, ERR_FORMAT, ERR_UNSUPPORTED, ERR_ALIGN, ERR_LAUNCH = range(7)


class lba_qfmt(ctypes.Structure):
    _fields_ = [("exp_bits", ctypes.c_int32), ("man_bits", ctypes.c_int32),
                ("bias", ctypes.c_int32), ("round", ctypes.c_int32)]


class lba_infmt(ctypes.Structure):
    _fields_ = [("exp_bits", ctypes.c_int32), ("man_bits", ctypes.c_int32), ("bias", ctypes.c_int32)]


def infmt(f):
    return f if isinstance(f, lba_infmt) else lba_infmt(*[int(v) for v in f])


class lba_drop(ctypes.Structure):
    _fields_ = [("p", ctypes.c_double), ("seed", ctypes.c_uint64), ("stream", ctypes.c_uint64), ("step", ctypes.c_void_p)]


class lba_strides(ctypes.Structure):
    _fields_ = [("row", ctypes.c_int64), ("head", ctypes.c_int64)]


class lba_attn(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int64) for n in ("T", "Tk", "count")] + [(n, ctypes.c_void_p) for n in ("starts", "starts_k")]
                + [(n, ctypes.c_int32) for n in ("H", "KV", "D", "type", "causal", "clear")] + [("scale", ctypes.c_float)]
                + [(n, lba_strides) for n in ("q", "k", "v")])


class lba_cache4(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_void_p) for n in ("k", "k_scale", "v", "v_scale")] + [(n, ctypes.c_int64) for n in ("pages", "table_row", "count")]
                + [(n, ctypes.c_void_p) for n in ("table", "lens")] + [(n, ctypes.c_int32) for n in ("page", "KV", "D")])


class lba_conv2d_desc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n", "h", "w", "c", "kh", "kw", "stride", "pad")]


class lba_plan_info(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "kernel", "prod_mode", "round", "tile_m", "tile_n", "tile_k", "thread_m", "thread_n",
        "grid_x", "grid_y", "valu_per_mac_x100", "tail_blocks", "mid_blocks")]


class LbaError(RuntimeError):
    def __init__(self, code, text):
        super().__init__("lba error %d: %s" % (code, text))
        self.code = code


_lib = None


def lib(path=None):
    """Load paper_2401_14110_amd/liblba_hip.so (built by __graft_entry__.build()).  `path`: another build of
    the same library, honoured only on the first call of a process (A/B measurements)."""
    global _lib
    if _lib is None:
        libpath = path or _LIBPATH
        if not os.path.exists(libpath):
            raise RuntimeError("HIP library %s is missing: run `python __graft_entry__.py` "
                               "(there is no fallback path)" % libpath)
        L = ctypes.CDLL(libpath)
        vp, i64, i32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32
        L.lba_gemm.restype = ctypes.c_int
        L.lba_gemm.argtypes = [vp, vp, vp, i64, i64, i64, lba_qfmt, lba_qfmt, i32, vp]
        L.lba_gemm_bwd.restype = ctypes.c_int
        L.lba_gemm_bwd.argtypes = [vp, vp, vp, vp, vp, i64, i64, i64, lba_qfmt, lba_qfmt, i32, vp]
        L.lba_gemm_batched.restype = ctypes.c_int
        L.lba_gemm_batched.argtypes = [vp, vp, vp, i64, i64, i64, i64, i64, i64, i64, lba_qfmt, lba_qfmt, i32, vp]
        L.lba_gemm_bwd_diff.restype = ctypes.c_int
        L.lba_gemm_bwd_diff.argtypes = [vp, vp, vp, vp, i64, i64, i64, lba_qfmt, lba_qfmt, i32, ctypes.c_float, vp]
        L.lba_gemm_bwd_diff_in.restype = ctypes.c_int
        L.lba_gemm_bwd_diff_in.argtypes = [vp, vp, vp, vp, i64, i64, i64, lba_infmt, lba_infmt, lba_qfmt, lba_qfmt, i32,
                                           ctypes.c_float, vp]
        L.lba_gemm_bwd_chunked.restype = ctypes.c_int
        L.lba_gemm_bwd_chunked.argtypes = [vp, vp, vp, vp, vp, vp, vp, i64, i64, i64, lba_qfmt, lba_qfmt, vp]
        L.lba_mask_words_level2.restype = ctypes.c_size_t
        L.lba_mask_words_level2.argtypes = [i64, i64, i64]
        L.lba_gemm_in.restype = ctypes.c_int
        L.lba_gemm_in.argtypes = [vp, vp, vp, i64, i64, i64, lba_infmt, lba_infmt, lba_qfmt, lba_qfmt, i32, vp]
        L.lba_gemm_bwd_in.restype = ctypes.c_int
        L.lba_gemm_bwd_in.argtypes = [vp, vp, vp, vp, vp, i64, i64, i64, lba_infmt, lba_infmt, lba_qfmt, lba_qfmt, i32, vp]
        L.lba_conv2d.restype = ctypes.c_int
        L.lba_conv2d.argtypes = [vp, vp, vp, lba_conv2d_desc, i64, lba_qfmt, lba_qfmt, i32, vp]
        L.lba_conv2d_bwd.restype = ctypes.c_int
        L.lba_conv2d_bwd.argtypes = [vp, vp, vp, vp, vp, lba_conv2d_desc, i64, lba_qfmt, lba_qfmt, i32, vp]
        L.lba_conv2d_out_shape.restype = ctypes.c_int
        L.lba_conv2d_out_shape.argtypes = [lba_conv2d_desc, ctypes.POINTER(ctypes.c_int32), ctypes.POINTER(ctypes.c_int32)]
        L.lba_plan_query_in.restype = ctypes.c_int
        L.lba_plan_query_in.argtypes = [i64, i64, i64, lba_infmt, lba_infmt, lba_qfmt, lba_qfmt, i32, i32,
                                        ctypes.POINTER(lba_plan_info)]
        L.lba_last_overflow.restype = ctypes.c_int
        L.lba_last_overflow.argtypes = [vp, vp, i64, i64, i64, vp]
        L.lba_ste_plane.restype = ctypes.c_int
        L.lba_ste_plane.argtypes = [vp, vp, vp, i64, i64, i64, i32, i32, vp]
        L.lba_grad.restype = ctypes.c_int
        L.lba_grad.argtypes = [vp, vp, vp, vp, vp, vp, vp, i64, i64, i64, i32, vp]
        L.lba_grad_ws.restype = ctypes.c_int
        L.lba_grad_ws.argtypes = [vp, vp, vp, vp, vp, vp, vp, i64, i64, i64, i32, vp, ctypes.c_size_t, vp]
        L.lba_gemm_bwd_ws.restype = ctypes.c_int
        L.lba_gemm_bwd_ws.argtypes = [vp, vp, vp, vp, vp, i64, i64, i64, lba_qfmt, lba_qfmt, vp, ctypes.c_size_t, vp]
        L.lba_grad_premapped.restype = ctypes.c_int
        L.lba_grad_premapped.argtypes = [vp, vp, vp, vp, vp, vp, i64, i64, i64, vp, ctypes.c_size_t, vp]
        L.lba_grad_static.restype = ctypes.c_int
        L.lba_grad_static.argtypes = [vp, vp, vp, vp, vp, vp, vp, i64, i64, i64, i32, vp]
        L.lba_grad_workspace_bytes.restype = ctypes.c_size_t
        L.lba_grad_workspace_bytes.argtypes = [i64, i64, i64]
        L.lba_grad_workspace_bytes_fast.restype = ctypes.c_size_t
        L.lba_grad_workspace_bytes_fast.argtypes = [i64, i64, i64]
        L.lba_mask_words.restype = ctypes.c_size_t
        L.lba_mask_words.argtypes = [i64, i64, i64]
        L.lba_strerror.restype = ctypes.c_char_p
        L.lba_strerror.argtypes = [ctypes.c_int]
        L.lba_plan_kernel_name_in.restype = ctypes.c_int
        L.lba_plan_kernel_name_in.argtypes = [i64, i64, i64, lba_infmt, lba_infmt, lba_qfmt, lba_qfmt, i32, i32, ctypes.c_char_p,
                                              ctypes.c_size_t]
        L.lba_plan_kernel_name.restype = ctypes.c_int
        L.lba_plan_kernel_name.argtypes = [i64, i64, i64, lba_qfmt, lba_qfmt, i32, i32, ctypes.c_char_p, ctypes.c_size_t]
        L.lba_plan_query.restype = ctypes.c_int
        L.lba_plan_query.argtypes = [i64, i64, i64, lba_qfmt, lba_qfmt, i32, i32,
                                     ctypes.POINTER(lba_plan_info)]
        f32, size = ctypes.c_float, ctypes.c_size_t
        L.lba_layernorm.restype = ctypes.c_int
        L.lba_layernorm.argtypes = [vp, i32, vp, vp, f32, vp, i32, lba_infmt, vp, vp, i64, i64, vp]
        L.lba_layernorm_bwd.restype = ctypes.c_int
        L.lba_layernorm_bwd.argtypes = [vp, i32, vp, i32, vp, vp, vp, vp, vp, vp, i64, i64, vp, size, vp]
        L.lba_layernorm_bwd_workspace_bytes.restype = size
        L.lba_layernorm_bwd_workspace_bytes.argtypes = [i64, i64]
        L.lba_dropout.restype = ctypes.c_int
        L.lba_dropout.argtypes = [vp, i32, f32, vp, i32, lba_drop, vp, i32, vp, i32, lba_infmt, i64, i64, vp]
        L.lba_dropout_bwd.restype = ctypes.c_int
        L.lba_dropout_bwd.argtypes = [vp, i32, vp, i32, f32, vp, i32, lba_drop, vp, vp, i64, i64, vp, size, vp]
        L.lba_dropout_bwd_workspace_bytes.restype = size
        L.lba_dropout_bwd_workspace_bytes.argtypes = [i64, i64]
        L.lba_dense.restype = ctypes.c_int
        L.lba_dense.argtypes = [vp, vp, i64, i64, i64, lba_infmt, lba_infmt, i32, vp, i32, lba_drop, vp, i32, vp, i32, lba_infmt, vp, size, vp]
        L.lba_dense_workspace_bytes.restype = size
        L.lba_dense_workspace_bytes.argtypes = [i64, i64, i64, lba_infmt, lba_infmt, i32, i32]
        L.lba_dense_bwd.restype = ctypes.c_int
        L.lba_dense_bwd.argtypes = [vp, i32, vp, vp, i64, i64, i64, lba_infmt, lba_infmt, i32, vp, i32, lba_drop, vp, vp, vp, vp, size, vp]
        L.lba_dense_bwd_workspace_bytes.restype = size
        L.lba_dense_bwd_workspace_bytes.argtypes = [i64, i64, i64, lba_infmt, lba_infmt, i32, i32, i32, i32]
        st = lba_strides
        for name in ("lba_rope", "lba_rope_bwd"):
            f = getattr(L, name)
            f.restype = ctypes.c_int
            f.argtypes = [vp, st, i32, vp, i32, vp, i64, i32, f32, vp, st, i64, i64, i64, vp]
        L.lba_attention.restype = ctypes.c_int
        L.lba_attention.argtypes = [lba_attn, vp, vp, vp, vp, i32, lba_infmt, vp, vp, size, vp]
        L.lba_attention_workspace_bytes.restype = size
        L.lba_attention_workspace_bytes.argtypes = [lba_attn]
        L.lba_attention_bwd.restype = ctypes.c_int
        L.lba_attention_bwd.argtypes = [lba_attn, vp, vp, vp, vp, vp, vp, vp, st, vp, st, vp, st, vp, size, vp]
        L.lba_attention_bwd_workspace_bytes.restype = size
        L.lba_attention_bwd_workspace_bytes.argtypes = [lba_attn]
        L.lba_cache_write.restype = ctypes.c_int
        L.lba_cache_write.argtypes = [lba_cache4, vp, i64, vp, st, vp, st, i32, vp]
        L.lba_cache_read.restype = ctypes.c_int
        L.lba_cache_read.argtypes = [lba_cache4, vp, i64, vp, st, vp, st, i32, i32, vp]
        L.lba_cache_attention.restype = ctypes.c_int
        L.lba_cache_attention.argtypes = [lba_cache4, vp, st, i32, i64, i64, f32, vp, i32, lba_infmt, vp, size, vp]
        L.lba_cache_attention_workspace_bytes.restype = size
        L.lba_cache_attention_workspace_bytes.argtypes = [i64, i64, i32, i64, i64, i32, i32]
        _lib = L
    return _lib


def qfmt(f):
    """(E, M, b, round) tuple or lba_qfmt -> lba_qfmt."""
    if isinstance(f, lba_qfmt):
        return f
    f = tuple(f)
    try:
        return lba_qfmt(*f)
    except TypeError:                              # fields that are numbers without being integers
        return lba_qfmt(*[int(v) for v in f])


def lba_strerror(code):
    return lib().lba_strerror(int(code)).decode()


strerror = lba_strerror


def _check(rc):
    if rc != OK:
        raise LbaError(rc, strerror(rc))


def _stream(stream):
    if stream is None:
        # the current device's current stream, without the Stream object torch.cuda.current_stream() builds around it (2.9 us of the
        # 8.3 us that a call took on the host; 0.3 us)
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    return ctypes.c_void_p(stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream))


# ---- raw calls: same names and argument order as include/lba.h ------------------------------

def lba_gemm(A, B, C, M, N, K, qprod, qacc, order=ORDER_SEQ, hip_stream=None):
    """Raw call: A, B, C are device addresses (ints) or None; returns the status code."""
    return lib().lba_gemm(A, B, C, M, N, K, qfmt(qprod), qfmt(qacc), order,
                          ctypes.c_void_p(hip_stream) if isinstance(hip_stream, int) else hip_stream)


def lba_gemm_bwd(A, B, C, of_mask, uf_mask, M, N, K, qprod, qacc, order=ORDER_SEQ, hip_stream=None):
    return lib().lba_gemm_bwd(A, B, C, of_mask, uf_mask, M, N, K, qfmt(qprod), qfmt(qacc), order,
                              ctypes.c_void_p(hip_stream) if isinstance(hip_stream, int) else hip_stream)


def lba_gemm_batched(A, B, C, batch, stride_a, stride_b, stride_c, M, N, K, qprod, qacc,
                     order=ORDER_SEQ, hip_stream=None):
    return lib().lba_gemm_batched(A, B, C, batch, stride_a, stride_b, stride_c, M, N, K, qfmt(qprod),
                                  qfmt(qacc), order,
                                  ctypes.c_void_p(hip_stream) if isinstance(hip_stream, int) else hip_stream)


def lba_gemm_bwd_diff(A, B, C, diff_mask, M, N, K, qprod, qacc, order, eps2, hip_stream=None):
    return lib().lba_gemm_bwd_diff(A, B, C, diff_mask, M, N, K, qfmt(qprod), qfmt(qacc), order, float(eps2), hip_stream)


def lba_gemm_bwd_diff_in(A, B, C, diff_mask, M, N, K, fmt_a, fmt_b, qprod, qacc, order, eps2, hip_stream=None):
    return lib().lba_gemm_bwd_diff_in(A, B, C, diff_mask, M, N, K, infmt(fmt_a), infmt(fmt_b), qfmt(qprod), qfmt(qacc),
                                      order, float(eps2), hip_stream)


def lba_gemm_bwd_chunked(A, B, C, of_mask, uf_mask, of_mask2, uf_mask2, M, N, K, qprod, qacc, hip_stream=None):
    return lib().lba_gemm_bwd_chunked(A, B, C, of_mask, uf_mask, of_mask2, uf_mask2, M, N, K, qfmt(qprod),
                                      qfmt(qacc),
                                      ctypes.c_void_p(hip_stream) if isinstance(hip_stream, int) else hip_stream)


def lba_gemm_in(A, B, C, M, N, K, fmt_a, fmt_b, qprod, qacc, order=ORDER_SEQ, hip_stream=None):
    return lib().lba_gemm_in(A, B, C, M, N, K, infmt(fmt_a), infmt(fmt_b), qfmt(qprod), qfmt(qacc), order,
                             ctypes.c_void_p(hip_stream) if isinstance(hip_stream, int) else hip_stream)


def lba_gemm_bwd_in(A, B, C, of_mask, uf_mask, M, N, K, fmt_a, fmt_b, qprod, qacc, order=ORDER_SEQ, hip_stream=None):
    return lib().lba_gemm_bwd_in(A, B, C, of_mask, uf_mask, M, N, K, infmt(fmt_a), infmt(fmt_b), qfmt(qprod),
                                 qfmt(qacc), order,
                                 ctypes.c_void_p(hip_stream) if isinstance(hip_stream, int) else hip_stream)


def _desc(d):
    return d if isinstance(d, lba_conv2d_desc) else lba_conv2d_desc(*[int(v) for v in d])


def lba_conv2d(X, W, Y, desc, cout, qprod, qacc, order=ORDER_SEQ, hip_stream=None):
    return lib().lba_conv2d(X, W, Y, _desc(desc), cout, qfmt(qprod), qfmt(qacc), order,
                            ctypes.c_void_p(hip_stream) if isinstance(hip_stream, int) else hip_stream)


def lba_conv2d_bwd(X, W, Y, of_mask, uf_mask, desc, cout, qprod, qacc, order=ORDER_SEQ, hip_stream=None):
    return lib().lba_conv2d_bwd(X, W, Y, of_mask, uf_mask, _desc(desc), cout, qfmt(qprod), qfmt(qacc), order,
                                ctypes.c_void_p(hip_stream) if isinstance(hip_stream, int) else hip_stream)


def lba_conv2d_out_shape(desc):
    """(status, oh, ow)"""
    oh, ow = ctypes.c_int32(0), ctypes.c_int32(0)
    rc = lib().lba_conv2d_out_shape(_desc(desc), ctypes.byref(oh), ctypes.byref(ow))
    return rc, oh.value, ow.value


def lba_last_overflow(of_mask, last_of, M, N, K, hip_stream=None):
    return lib().lba_last_overflow(of_mask, last_of, M, N, K,
                                   ctypes.c_void_p(hip_stream) if isinstance(hip_stream, int) else hip_stream)


def lba_ste_plane(of_mask, of_mask2, coef, M, N, K, ste, order, hip_stream=None):
    return lib().lba_ste_plane(of_mask, of_mask2, coef, M, N, K, ste, order,
                               ctypes.c_void_p(hip_stream) if isinstance(hip_stream, int) else hip_stream)


def lba_grad(G, A, B, of_mask, last_of, dX, dW, M, N, K, ste, hip_stream=None):
    return lib().lba_grad(G, A, B, of_mask, last_of, dX, dW, M, N, K, ste,
                          ctypes.c_void_p(hip_stream) if isinstance(hip_stream, int) else hip_stream)


def lba_grad_ws(G, A, B, of_mask, last_of, dX, dW, M, N, K, ste, workspace, workspace_bytes, hip_stream=None):
    return lib().lba_grad_ws(G, A, B, of_mask, last_of, dX, dW, M, N, K, ste, workspace, workspace_bytes,
                             ctypes.c_void_p(hip_stream) if isinstance(hip_stream, int) else hip_stream)


def lba_grad_static(G, A, B, of_mask, last_of, dX, dW, M, N, K, ste, hip_stream=None):
    return lib().lba_grad_static(G, A, B, of_mask, last_of, dX, dW, M, N, K, ste,
                                 ctypes.c_void_p(hip_stream) if isinstance(hip_stream, int) else hip_stream)


def lba_gemm_bwd_ws(A, B, C, of_mask, uf_mask, M, N, K, qprod, qacc, workspace, workspace_bytes, hip_stream=None):
    return lib().lba_gemm_bwd_ws(A, B, C, of_mask, uf_mask, M, N, K, qfmt(qprod), qfmt(qacc), workspace, workspace_bytes,
                                 ctypes.c_void_p(hip_stream) if isinstance(hip_stream, int) else hip_stream)


def lba_grad_premapped(G, A, B, of_mask, dX, dW, M, N, K, workspace, workspace_bytes, hip_stream=None):
    return lib().lba_grad_premapped(G, A, B, of_mask, dX, dW, M, N, K, workspace, workspace_bytes,
                                    ctypes.c_void_p(hip_stream) if isinstance(hip_stream, int) else hip_stream)


def lba_grad_workspace_bytes(M, N, K):
    return int(lib().lba_grad_workspace_bytes(M, N, K))


def lba_grad_workspace_bytes_fast(M, N, K):
    return int(lib().lba_grad_workspace_bytes_fast(M, N, K))


def lba_mask_words(M, N, K):
    return int(lib().lba_mask_words(M, N, K))


def lba_mask_words_level2(M, N, K):
    return int(lib().lba_mask_words_level2(M, N, K))


def lba_plan_query_in(M, N, K, fmt_a, fmt_b, qprod, qacc, order=ORDER_SEQ, with_masks=0):
    info = lba_plan_info()
    _check(lib().lba_plan_query_in(M, N, K, infmt(fmt_a), infmt(fmt_b), qfmt(qprod), qfmt(qacc), order, with_masks,
                                   ctypes.byref(info)))
    return {n: getattr(info, n) for n, _ in lba_plan_info._fields_}


def lba_plan_query(M, N, K, qprod, qacc, order=ORDER_SEQ, with_masks=0):
    info = lba_plan_info()
    _check(lib().lba_plan_query(M, N, K, qfmt(qprod), qfmt(qacc), order, with_masks, ctypes.byref(info)))
    return {n: getattr(info, n) for n, _ in lba_plan_info._fields_}


def lba_plan_kernel_name(M, N, K, qprod, qacc, order=ORDER_SEQ, with_masks=0):
    buf = ctypes.create_string_buffer(128)
    _check(lib().lba_plan_kernel_name(M, N, K, qfmt(qprod), qfmt(qacc), order, with_masks, buf, len(buf)))
    return buf.value.decode()


def lba_plan_kernel_name_in(M, N, K, fmt_a, fmt_b, qprod, qacc, order=ORDER_SEQ, with_masks=0):
    buf = ctypes.create_string_buffer(128)
    _check(lib().lba_plan_kernel_name_in(M, N, K, infmt(fmt_a), infmt(fmt_b), qfmt(qprod), qfmt(qacc), order, with_masks, buf,
                                         len(buf)))
    return buf.value.decode()


def lba_layernorm(X, x_type, gamma, beta, eps, Y, y_type, y_fmt, mean, rstd, M, N, hip_stream=None):
    return lib().lba_layernorm(X, x_type, gamma, beta, float(eps), Y, y_type, infmt(y_fmt), mean, rstd, M, N, hip_stream)


def lba_layernorm_bwd(G, g_type, X, x_type, gamma, mean, rstd, dX, dgamma, dbeta, M, N, workspace, workspace_bytes, hip_stream=None):
    return lib().lba_layernorm_bwd(G, g_type, X, x_type, gamma, mean, rstd, dX, dgamma, dbeta, M, N, workspace, workspace_bytes,
                                   hip_stream)


def lba_layernorm_bwd_workspace_bytes(M, N):
    return int(lib().lba_layernorm_bwd_workspace_bytes(M, N))


def lba_dropout(X, x_type, scale, bias, act, drop, residual, r_type, Y, y_type, y_fmt, M, N, hip_stream=None):
    return lib().lba_dropout(X, x_type, float(scale), bias, act, drop, residual, r_type, Y, y_type, infmt(y_fmt), M, N, hip_stream)


def lba_dropout_bwd(G, g_type, X, x_type, scale, bias, act, drop, dX, dbias, M, N, workspace, workspace_bytes, hip_stream=None):
    return lib().lba_dropout_bwd(G, g_type, X, x_type, float(scale), bias, act, drop, dX, dbias, M, N, workspace, workspace_bytes,
                                 hip_stream)


def lba_dropout_bwd_workspace_bytes(M, N):
    return int(lib().lba_dropout_bwd_workspace_bytes(M, N))


def lba_dense(A, B, M, N, K, fmt_a, fmt_b, gated, bias, act, drop, residual, r_type, Y, y_type, y_fmt, workspace, workspace_bytes,
              hip_stream=None):
    return lib().lba_dense(A, B, M, N, K, infmt(fmt_a), infmt(fmt_b), gated, bias, act, drop, residual, r_type, Y, y_type, infmt(y_fmt),
                           workspace, workspace_bytes, hip_stream)


def lba_dense_workspace_bytes(M, N, K, fmt_a, fmt_b, gated, aligned=1):
    return int(lib().lba_dense_workspace_bytes(M, N, K, infmt(fmt_a), infmt(fmt_b), gated, aligned))


def lba_dense_bwd(G, g_type, A, B, M, N, K, fmt_a, fmt_b, gated, bias, act, drop, dA, dB, dbias, workspace, workspace_bytes,
                  hip_stream=None):
    return lib().lba_dense_bwd(G, g_type, A, B, M, N, K, infmt(fmt_a), infmt(fmt_b), gated, bias, act, drop, dA, dB, dbias, workspace,
                               workspace_bytes, hip_stream)


def lba_dense_bwd_workspace_bytes(M, N, K, fmt_a, fmt_b, gated, act, g_type, aligned=1):
    return int(lib().lba_dense_bwd_workspace_bytes(M, N, K, infmt(fmt_a), infmt(fmt_b), gated, act, g_type, aligned))


def lba_rope(X, x_at, type, positions, pos_bits, freq, pairs, interleaved, gain, Y, y_at, T, H, D, hip_stream=None):
    return lib().lba_rope(X, x_at, type, positions, pos_bits, freq, pairs, interleaved, gain, Y, y_at, T, H, D, hip_stream)


def lba_rope_bwd(G, g_at, type, positions, pos_bits, freq, pairs, interleaved, gain, dX, dx_at, T, H, D, hip_stream=None):
    return lib().lba_rope_bwd(G, g_at, type, positions, pos_bits, freq, pairs, interleaved, gain, dX, dx_at, T, H, D, hip_stream)


def lba_attention(a, Q, K, V, O, o_type, o_fmt, lse, workspace, workspace_bytes, hip_stream=None):
    return lib().lba_attention(a, Q, K, V, O, o_type, infmt(o_fmt), lse, workspace, workspace_bytes, hip_stream)


def lba_attention_workspace_bytes(a):
    return int(lib().lba_attention_workspace_bytes(a))


def lba_attention_bwd(a, G, Q, K, V, O, lse, dQ, dq_at, dK, dk_at, dV, dv_at, workspace, workspace_bytes, hip_stream=None):
    return lib().lba_attention_bwd(a, G, Q, K, V, O, lse, dQ, dq_at, dK, dk_at, dV, dv_at, workspace, workspace_bytes, hip_stream)


def lba_attention_bwd_workspace_bytes(a):
    return int(lib().lba_attention_bwd_workspace_bytes(a))


def lba_cache_write(c, starts, T, K, k_at, V, v_at, type, hip_stream=None):
    return lib().lba_cache_write(c, starts, T, K, k_at, V, v_at, type, hip_stream)


def lba_cache_read(c, starts, T, K, k_at, V, v_at, type, clear, hip_stream=None):
    return lib().lba_cache_read(c, starts, T, K, k_at, V, v_at, type, clear, hip_stream)


def lba_cache_attention(c, Q, q_at, type, fresh, H, scale, O, o_type, o_fmt, workspace, workspace_bytes, hip_stream=None):
    return lib().lba_cache_attention(c, Q, q_at, type, fresh, H, scale, O, o_type, infmt(o_fmt), workspace, workspace_bytes, hip_stream)


def lba_cache_attention_workspace_bytes(count, table_row, page, fresh, H, KV, D):
    return int(lib().lba_cache_attention_workspace_bytes(count, table_row, page, fresh, H, KV, D))


# ---- tensor conveniences --------------------------------------------------------------------

def _ops(A, B):
    if A.dtype != torch.uint8 or B.dtype != torch.uint8:
        raise TypeError("A and B must be uint8 E4M3 codes")
    if not (A.is_cuda and B.is_cuda):
        raise ValueError("A and B must be device tensors")
    if A.dim() != 2 or B.dim() != 2 or A.shape[1] != B.shape[1]:
        raise ValueError("A must be [M, K] and B [N, K]")
    return A.contiguous(), B.contiguous()


def gemm(A, B, qprod, qacc, order=ORDER_SEQ, out=None, stream=None):
    """C[M,N] (float32, device) = LBA product of A [M,K] and B [N,K] uint8 E4M3 device tensors."""
    A, B = _ops(A, B)
    M, K = A.shape
    N = B.shape[0]
    C = out if out is not None else torch.empty((M, N), dtype=torch.float32, device=A.device)
    _check(lib().lba_gemm(A.data_ptr() or None, B.data_ptr() or None, C.data_ptr() or None,
                          M, N, K, qfmt(qprod), qfmt(qacc), order, _stream(stream)))
    return C


def gemm_batched(A, B, qprod, qacc, order=ORDER_SEQ, stream=None):
    """A [batch, M, K], B [batch, N, K] or [N, K] (shared) uint8 device tensors -> C [batch, M, N]."""
    if A.dtype != torch.uint8 or B.dtype != torch.uint8 or not (A.is_cuda and B.is_cuda):
        raise TypeError("A and B must be uint8 device tensors")
    A = A.contiguous()
    B = B.contiguous()
    batch, M, K = A.shape
    shared = B.dim() == 2
    N = B.shape[-2]
    if B.shape[-1] != K or (not shared and B.shape[0] != batch):
        raise ValueError("shape mismatch")
    C = torch.empty((batch, M, N), dtype=torch.float32, device=A.device)
    _check(lib().lba_gemm_batched(A.data_ptr() or None, B.data_ptr() or None, C.data_ptr() or None, batch,
                                  M * K, 0 if shared else N * K, M * N, M, N, K,
                                  qfmt(qprod), qfmt(qacc), order, _stream(stream)))
    return C


def gemm_bwd(A, B, qprod, qacc, order=ORDER_SEQ, want_c=True, stream=None, want_uf=True):
    """Returns (C or None, OF plane, UF plane or None); planes are int32 tensors [ceil(K/32), M, N]."""
    A, B = _ops(A, B)
    M, K = A.shape
    N = B.shape[0]
    W = (K + 31) // 32
    C = torch.empty((M, N), dtype=torch.float32, device=A.device) if want_c else None
    of = torch.empty((W, M, N), dtype=torch.int32, device=A.device)
    uf = torch.empty((W, M, N), dtype=torch.int32, device=A.device) if want_uf else None
    _check(lib().lba_gemm_bwd(A.data_ptr() or None, B.data_ptr() or None,
                              (C.data_ptr() or None) if want_c else None,
                              of.data_ptr() or None, (uf.data_ptr() or None) if want_uf else None,
                              M, N, K, qfmt(qprod), qfmt(qacc), order, _stream(stream)))
    return C, of, uf


def _workspace(workspace):
    if workspace.dtype != torch.uint8 or not workspace.is_cuda or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous uint8 device tensor")
    return workspace


def gemm_bwd_ws(A, B, qprod, qacc, workspace=None, want_c=True, stream=None, want_uf=True):
    """lba_gemm_bwd_ws: as gemm_bwd (sequential order), and `workspace` (allocated here if None: a uint8 device tensor
    of lba_grad_workspace_bytes_fast(M, N, K) bytes: the maps, and behind them the scratch memory in which
    grad_premapped combines its split sums) receives the brick maps of the OF plane for grad_premapped.
    Returns (C or None, OF plane, UF plane or None, workspace)."""
    A, B = _ops(A, B)
    M, K = A.shape
    N = B.shape[0]
    W = (K + 31) // 32
    if workspace is None:
        workspace = torch.empty(max(256, lba_grad_workspace_bytes_fast(M, N, K)), dtype=torch.uint8, device=A.device)
    workspace = _workspace(workspace)
    C = torch.empty((M, N), dtype=torch.float32, device=A.device) if want_c else None
    of = torch.empty((W, M, N), dtype=torch.int32, device=A.device)
    uf = torch.empty((W, M, N), dtype=torch.int32, device=A.device) if want_uf else None
    _check(lib().lba_gemm_bwd_ws(A.data_ptr() or None, B.data_ptr() or None,
                                 (C.data_ptr() or None) if want_c else None,
                                 of.data_ptr() or None, (uf.data_ptr() or None) if want_uf else None,
                                 M, N, K, qfmt(qprod), qfmt(qacc), workspace.data_ptr() or None, workspace.numel(),
                                 _stream(stream)))
    return C, of, uf, workspace


def grad_premapped(G, A, B, of_plane, workspace, want_dx=True, want_dw=True, stream=None):
    """lba_grad_premapped: the immediate estimator's dX, dW from the OF plane and the workspace of gemm_bwd_ws."""
    A, B = _ops(A, B)
    M, K = A.shape
    N = B.shape[0]
    if G.dtype != torch.float32 or tuple(G.shape) != (M, N) or not G.is_cuda:
        raise ValueError("G must be a float32 device tensor [M, N]")
    G = G.contiguous()
    of_plane = _plane(of_plane, K, M, N, "of_plane")
    workspace = _workspace(workspace)
    dX = torch.empty((M, K), dtype=torch.float32, device=A.device) if want_dx else None
    dW = torch.empty((N, K), dtype=torch.float32, device=A.device) if want_dw else None
    ptr = lambda t: (t.data_ptr() or None) if t is not None else None
    _check(lib().lba_grad_premapped(ptr(G), ptr(A), ptr(B), ptr(of_plane), ptr(dX), ptr(dW), M, N, K,
                                    ptr(workspace), workspace.numel(), _stream(stream)))
    return dX, dW


def gemm_bwd_diff(A, B, qprod, qacc, eps2, order=ORDER_SEQ, want_c=True, stream=None, fmt_a=None, fmt_b=None):
    """Returns (C or None, DIFF plane [ceil(K/32), M, N] int32): bit k is 1 - STE^DIFF of step k.
    With fmt_a / fmt_b: lba_gemm_bwd_diff_in."""
    A, B = _ops(A, B)
    M, K = A.shape
    N = B.shape[0]
    C = torch.empty((M, N), dtype=torch.float32, device=A.device) if want_c else None
    diff = torch.empty(((K + 31) // 32, M, N), dtype=torch.int32, device=A.device)
    if fmt_a is not None or fmt_b is not None:
        _check(lib().lba_gemm_bwd_diff_in(A.data_ptr() or None, B.data_ptr() or None,
                                          (C.data_ptr() or None) if want_c else None, diff.data_ptr() or None, M, N, K,
                                          infmt(fmt_a or (4, 3, 7)), infmt(fmt_b or (4, 3, 7)), qfmt(qprod), qfmt(qacc),
                                          order, float(eps2), _stream(stream)))
        return C, diff
    _check(lib().lba_gemm_bwd_diff(A.data_ptr() or None, B.data_ptr() or None, (C.data_ptr() or None) if want_c else None,
                                   diff.data_ptr() or None, M, N, K, qfmt(qprod), qfmt(qacc), order, float(eps2),
                                   _stream(stream)))
    return C, diff


def gemm_bwd_chunked(A, B, qprod, qacc, want_c=True, stream=None, want_uf=True):
    """Chunked order.  Returns (C or None, OF, UF, OF2, UF2): first-level planes [ceil(K/32), M, N] and
    second-level planes [ceil(ceil(K/16)/32), M, N], int32 tensors (UF, UF2 are None without want_uf)."""
    A, B = _ops(A, B)
    M, K = A.shape
    N = B.shape[0]
    W = (K + 31) // 32
    W2 = ((K + 15) // 16 + 31) // 32
    C = torch.empty((M, N), dtype=torch.float32, device=A.device) if want_c else None
    planes = [torch.empty((w, M, N), dtype=torch.int32, device=A.device) if (want_uf or i % 2 == 0) else None
              for i, w in enumerate((W, W, W2, W2))]
    _check(lib().lba_gemm_bwd_chunked(A.data_ptr() or None, B.data_ptr() or None,
                                      (C.data_ptr() or None) if want_c else None,
                                      *[(t.data_ptr() or None) if t is not None else None for t in planes],
                                      M, N, K, qfmt(qprod), qfmt(qacc), _stream(stream)))
    return (C, *planes)


def _plane(t, K, M=None, N=None, what="plane"):
    """An event / coefficient plane as the library reads it: int32 [ceil(K/32), M, N], contiguous, on the device."""
    if t.dtype not in (torch.int32, torch.uint32) or not t.is_cuda or t.dim() != 3:
        raise ValueError("%s must be a 3-d int32 device tensor [ceil(K/32), M, N]" % what)
    if t.shape[0] != (K + 31) // 32 or (M is not None and tuple(t.shape[1:]) != (M, N)):
        raise ValueError("%s has shape %s, expected [%d, M, N]" % (what, tuple(t.shape), (K + 31) // 32))
    return t.contiguous()


def last_overflow(of_plane, K, stream=None):
    """int32 [M, N] index of the last overflowing step of every chain (-1: none) from an OF plane."""
    of_plane = _plane(of_plane, K, what="of_plane")
    W, M, N = of_plane.shape
    out = torch.empty((M, N), dtype=torch.int32, device=of_plane.device)
    _check(lib().lba_last_overflow(of_plane.data_ptr() or None, out.data_ptr() or None, M, N, K, _stream(stream)))
    return out


def grad(G, A, B, ste, of_plane=None, last_of=None, want_dx=True, want_dw=True, stream=None, workspace=None):
    """Masked gradient products: returns (dX [M, K] or None, dW [N, K] or None), float32 device tensors.
    workspace: a uint8 device tensor of at least lba_grad_workspace_bytes(M, N, K) bytes: lba_grad_ws."""
    A, B = _ops(A, B)
    M, K = A.shape
    N = B.shape[0]
    if G.dtype != torch.float32 or tuple(G.shape) != (M, N) or not G.is_cuda:
        raise ValueError("G must be a float32 device tensor [M, N]")
    G = G.contiguous()
    if of_plane is not None:
        of_plane = _plane(of_plane, K, M, N, "of_plane")
    if last_of is not None:
        if last_of.dtype != torch.int32 or tuple(last_of.shape) != (M, N) or not last_of.is_cuda:
            raise ValueError("last_of must be an int32 device tensor [M, N]")
        last_of = last_of.contiguous()
    dX = torch.empty((M, K), dtype=torch.float32, device=A.device) if want_dx else None
    dW = torch.empty((N, K), dtype=torch.float32, device=A.device) if want_dw else None
    ptr = lambda t: (t.data_ptr() or None) if t is not None else None
    if workspace is not None:
        if workspace.dtype != torch.uint8 or not workspace.is_cuda or not workspace.is_contiguous():
            raise ValueError("workspace must be a contiguous uint8 device tensor")
        _check(lib().lba_grad_ws(ptr(G), ptr(A), ptr(B), ptr(of_plane), ptr(last_of), ptr(dX), ptr(dW), M, N, K, ste,
                                 ptr(workspace), workspace.numel(), _stream(stream)))
        return dX, dW
    _check(lib().lba_grad(ptr(G), ptr(A), ptr(B), ptr(of_plane), ptr(last_of), ptr(dX), ptr(dW), M, N, K, ste,
                          _stream(stream)))
    return dX, dW


def ste_plane(of_plane, K, ste, order=ORDER_SEQ, of_plane2=None, stream=None):
    """Coefficient plane (int32 [ceil(K/32), M, N], bit = 1: passes) of an estimator from the OF plane(s)."""
    of_plane = _plane(of_plane, K, what="of_plane")
    W, M, N = of_plane.shape
    if of_plane2 is not None:
        if of_plane2.dtype not in (torch.int32, torch.uint32) or not of_plane2.is_cuda or \
                tuple(of_plane2.shape) != (((K + 15) // 16 + 31) // 32, M, N):
            raise ValueError("of_plane2 must be an int32 device tensor [ceil(ceil(K/16)/32), M, N]")
        of_plane2 = of_plane2.contiguous()
    out = torch.empty_like(of_plane)
    _check(lib().lba_ste_plane(of_plane.data_ptr() or None,
                               (of_plane2.data_ptr() or None) if of_plane2 is not None else None,
                               out.data_ptr() or None, M, N, K, ste, order, _stream(stream)))
    return out


def gemm_in(A, B, fmt_a, fmt_b, qprod, qacc, order=ORDER_SEQ, planes=False, stream=None, uf_plane=True):
    """lba_gemm_in (or, with planes, lba_gemm_bwd_in: returns (C, OF, UF); UF is None without uf_plane) on uint8
    device tensors."""
    A, B = _ops(A, B)
    M, K = A.shape
    N = B.shape[0]
    C = torch.empty((M, N), dtype=torch.float32, device=A.device)
    if not planes:
        _check(lib().lba_gemm_in(A.data_ptr() or None, B.data_ptr() or None, C.data_ptr() or None, M, N, K,
                                 infmt(fmt_a), infmt(fmt_b), qfmt(qprod), qfmt(qacc), order, _stream(stream)))
        return C
    W = (K + 31) // 32
    of = torch.empty((W, M, N), dtype=torch.int32, device=A.device)
    uf = torch.empty((W, M, N), dtype=torch.int32, device=A.device) if uf_plane else None
    _check(lib().lba_gemm_bwd_in(A.data_ptr() or None, B.data_ptr() or None, C.data_ptr() or None,
                                 of.data_ptr() or None, (uf.data_ptr() or None) if uf_plane else None, M, N, K,
                                 infmt(fmt_a), infmt(fmt_b), qfmt(qprod), qfmt(qacc), order, _stream(stream)))
    return C, of, uf


def conv2d(X, W, qprod, qacc, stride=1, pad=0, order=ORDER_SEQ, planes=False, stream=None):
    """X [n, h, w, c] and W [cout, kh, kw, c] uint8 device tensors -> Y [n, oh, ow, cout] float32
    (with planes: also the OF and UF planes [ceil(K/32), n*oh*ow, cout] of the recompute call)."""
    if X.dtype != torch.uint8 or W.dtype != torch.uint8 or not (X.is_cuda and W.is_cuda):
        raise TypeError("X and W must be uint8 device tensors")
    X = X.contiguous()
    W = W.contiguous()
    n, h, w, c = X.shape
    cout, kh, kw, c2 = W.shape
    if c != c2:
        raise ValueError("channel mismatch")
    desc = lba_conv2d_desc(n, h, w, c, kh, kw, stride, pad)
    rc, oh, ow = lba_conv2d_out_shape(desc)
    _check(rc)
    Y = torch.empty((n, oh, ow, cout), dtype=torch.float32, device=X.device)
    if not planes:
        _check(lib().lba_conv2d(X.data_ptr() or None, W.data_ptr() or None, Y.data_ptr() or None, desc, cout,
                                qfmt(qprod), qfmt(qacc), order, _stream(stream)))
        return Y
    M, K = n * oh * ow, kh * kw * c
    of = torch.empty(((K + 31) // 32, M, cout), dtype=torch.int32, device=X.device)
    uf = torch.empty_like(of)
    _check(lib().lba_conv2d_bwd(X.data_ptr() or None, W.data_ptr() or None, Y.data_ptr() or None,
                                of.data_ptr() or None, uf.data_ptr() or None, desc, cout,
                                qfmt(qprod), qfmt(qacc), order, _stream(stream)))
    return Y, of, uf


# ---- the operators of include/lba_layer.h -----------------------------------------------------
#
# Codes in and out are uint8 tensors with a format (exp_bits, man_bits, bias), whose bias carries the tensor's power-of-two scale: the
# E4M3 codes of x * 2^t are those of (4, 3, 7 + t).  Outputs and temporaries come from the pool of the stream that the call runs on.

_E4M3 = (4, 3, 7)
_NO_FORMAT = lba_infmt(4, 3, 7)
_NO_DROP = lba_drop(0.0, 0, 0, None)
_TYPE = {torch.float32: F32, torch.bfloat16: BF16, torch.uint8: CODE8}
_WORD = (1 << 64) - 1


@functools.lru_cache(maxsize=1024)
def _layer_bytes(name, *shape):
    """A workspace's size, which the library derives from the shape alone."""
    return getattr(lib(), name)(*shape)


class _Format(lba_infmt):
    __hash__ = object.__hash__


_format = functools.lru_cache(maxsize=256)(_Format)   # one object a format, by its value, handed to nobody who might change it


def _infmt(f):
    if isinstance(f, lba_infmt):
        return _format(f.exp_bits, f.man_bits, f.bias)
    e, m, b = f
    return _format(int(e), int(m), int(b))


def _on(stream, device):
    """(handle, stream) of a call on tensors of the device: stream is None where it is the current one, else the object whose pool
    tensors made here come from."""
    if device != torch._C._cuda_getDevice():
        raise ValueError("the tensors' device is not the current one")
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(device), None
    handle = _stream(stream)
    if not hasattr(stream, "cuda_stream"):
        stream = torch.cuda.ExternalStream(int(stream)) if int(stream) else torch.cuda.default_stream()
    return handle, stream


def _whole(t, on):
    """t as the library reads it: contiguous (a copy is made on the call's stream)."""
    if t is None or t.is_contiguous():
        return t
    if on is None:
        return t.contiguous()
    with torch.cuda.stream(on):
        return t.contiguous()


# Memory for a call on another stream than the current one comes from that stream's pool: a block of the current stream's pool may have been
# freed a moment ago with kernels at work on it, for which the call's stream does not wait.
def _of_pool(make, on):
    with torch.cuda.stream(on):
        return make()


def _empty(shape, dtype, device, on):
    """An output.  It is recorded on the current stream, where the caller uses it and may free it."""
    if on is None:
        return torch.empty(shape, dtype=dtype, device=device)
    t = _of_pool(lambda: torch.empty(shape, dtype=dtype, device=device), on)
    t.record_stream(torch.cuda.current_stream(device))
    return t


def _empty_as(t, dtype, on):
    """A tensor of the contiguous t's shape (0.5 us less than from the shape)."""
    return torch.empty_like(t, dtype=dtype) if on is None else _empty(t.shape, dtype, t.device, on)


def _scratch(size, device, on):
    if not size:
        return None
    make = lambda: torch.empty((size,), dtype=torch.uint8, device=device)  # noqa: E731
    return make() if on is None else _of_pool(make, on)


_REAL = (torch.float32, torch.bfloat16)


def _rows(t, what, dtypes=_REAL):
    """(M, N, device) of a device tensor whose rows run along its last axis."""
    device = t.get_device()
    if t.dtype not in dtypes or device < 0:
        raise TypeError("%s must be a device tensor of %s" % (what, " or ".join(str(d) for d in dtypes)))
    if t.dim() < 1:
        raise ValueError("%s must have at least one axis" % what)
    n = t.size(-1)
    return t.numel() // n if n else math.prod(t.shape[:-1]), n, device


def _like(t, shape, device, what, dtypes=_REAL):
    if t.dtype not in dtypes or t.get_device() != device:
        raise TypeError("%s must be a tensor of %s on the call's device" % (what, " or ".join(str(d) for d in dtypes)))
    if t.shape != shape:
        raise ValueError("%s has shape %s, expected %s" % (what, tuple(t.shape), tuple(shape)))
    return t


def _vector(t, n, device, what, on):
    if t is None:
        return None
    if t.dtype != torch.float32 or t.get_device() != device or t.dim() != 1 or t.numel() != n:
        raise ValueError("%s must be a float32 tensor [%d] on the call's device" % (what, n))
    return _whole(t, on)


def _out_type(dtype, fmt):
    """(type code, lba_infmt) of an output."""
    if dtype not in _TYPE:
        raise TypeError("an output is torch.float32, torch.bfloat16, or torch.uint8 codes")
    if dtype is torch.uint8:
        if fmt is None:
            raise ValueError("codes need out_fmt = (exp_bits, man_bits, bias)")
        return CODE8, _infmt(fmt)
    if fmt is not None:
        raise ValueError("out_fmt is for torch.uint8 codes")
    return _TYPE[dtype], _NO_FORMAT


def _output(out, like, shape, dtype, on):
    if out is None:
        return _empty_as(like, dtype, on) if shape == like.shape else _empty(shape, dtype, like.device, on)
    if out.dtype != dtype or out.shape != shape or out.get_device() != like.get_device() or not out.is_contiguous():
        raise ValueError("out must be a contiguous tensor %s of %s on the call's device" % (tuple(shape), dtype))
    return out


def _drop(drop, device):
    """None, (p, seed, stream) or (p, seed, stream, step) with step a one-element int64 device tensor (read when the kernel runs)."""
    if drop is None:
        return _NO_DROP
    if isinstance(drop, lba_drop):
        return drop
    p, seed, stream = drop[:3]
    step = drop[3] if len(drop) > 3 else None
    if step is not None and (step.dtype != torch.int64 or step.get_device() != device or step.numel() != 1):
        raise ValueError("step must be an int64 tensor of one element on the call's device")
    return lba_drop(float(p), int(seed) & _WORD, int(stream) & _WORD, step.data_ptr() if step is not None else None)


def _at(t):
    return (t.data_ptr() or None) if t is not None else None


def layernorm(x, gamma=None, beta=None, eps=1e-5, out_dtype=None, out_fmt=None, want_stats=False, out=None, stream=None):
    """Layer norm over the last axis of x (float32 or bfloat16): y of out_dtype (x's by default; torch.uint8 codes need out_fmt), and
    with want_stats (y, mean, rstd), float32 tensors of x's leading shape, which layernorm_bwd reads."""
    M, N, device = _rows(x, "x")
    dtype = out_dtype or x.dtype
    y_type, fmt = _out_type(dtype, out_fmt)
    handle, on = _on(stream, device)
    x, gamma, beta = _whole(x, on), _vector(gamma, N, device, "gamma", on), _vector(beta, N, device, "beta", on)
    y = _output(out, x, x.shape, dtype, on)
    mean = _empty(x.shape[:-1], torch.float32, x.device, on) if want_stats else None
    rstd = _empty_as(mean, torch.float32, on) if want_stats else None
    _check(lib().lba_layernorm(_at(x), _TYPE[x.dtype], _at(gamma), _at(beta), eps, _at(y), y_type, fmt, _at(mean), _at(rstd), M, N, handle))
    return (y, mean, rstd) if want_stats else y


def layernorm_bwd(G, x, gamma, mean, rstd, want_dx=True, want_params=True, stream=None):
    """Gradients of layernorm: (dx of x's type or None, dgamma, dbeta: float32 or None)."""
    M, N, device = _rows(x, "x")
    rows = x.shape[:-1]
    _like(G, x.shape, device, "G")
    _like(mean, rows, device, "mean", (torch.float32,))
    _like(rstd, rows, device, "rstd", (torch.float32,))
    handle, on = _on(stream, device)
    G, x, mean, rstd, gamma = _whole(G, on), _whole(x, on), _whole(mean, on), _whole(rstd, on), _vector(gamma, N, device, "gamma", on)
    dx = _empty_as(x, x.dtype, on) if want_dx else None
    dgamma = _empty((N,), torch.float32, x.device, on) if want_params else None
    dbeta = _empty_as(dgamma, torch.float32, on) if want_params else None
    size = _layer_bytes("lba_layernorm_bwd_workspace_bytes", M, N) if want_params else 0
    ws = _scratch(size, x.device, on)
    _check(lib().lba_layernorm_bwd(_at(G), _TYPE[G.dtype], _at(x), _TYPE[x.dtype], _at(gamma), _at(mean), _at(rstd), _at(dx),
                                   _at(dgamma), _at(dbeta), M, N, _at(ws), size, handle))
    return dx, dgamma, dbeta


def dropout(x, drop, bias=None, act=ACT_NONE, residual=None, scale=1.0, out_dtype=None, out_fmt=None, out=None, stream=None):
    """residual + keep * act(scale * x + bias) / (1 - p) with drop = (p, seed, stream[, step]) or None; x and residual are float32
    or bfloat16, bias runs along the last axis, y is of out_dtype (x's by default; torch.uint8 codes need out_fmt).  After a simulated
    product scale = 2^-T undoes its operands' scales."""
    M, N, device = _rows(x, "x")
    dtype = out_dtype or x.dtype
    y_type, fmt = _out_type(dtype, out_fmt)
    d = _drop(drop, device)
    handle, on = _on(stream, device)
    x, bias = _whole(x, on), _vector(bias, N, device, "bias", on)
    if residual is not None:
        residual = _whole(_like(residual, x.shape, device, "residual"), on)
    y = _output(out, x, x.shape, dtype, on)
    _check(lib().lba_dropout(_at(x), _TYPE[x.dtype], scale, _at(bias), act, d, _at(residual),
                             _TYPE[residual.dtype] if residual is not None else F32, _at(y), y_type, fmt, M, N, handle))
    return y


def dropout_bwd(G, drop, x=None, bias=None, act=ACT_NONE, scale=1.0, want_dx=True, want_dbias=False, out_dtype=None, stream=None):
    """Gradients of dropout: (dx or None, dbias or None).  x and bias are needed where act is not ACT_NONE; dx is of x's type, of
    out_dtype without x, of G's without both.  The residual's gradient is G."""
    M, N, device = _rows(G, "G")
    dtype = x.dtype if x is not None else out_dtype or G.dtype
    if out_dtype is not None and out_dtype != dtype:
        raise ValueError("dx has x's type")
    if x is not None:
        _like(x, G.shape, device, "x")
    elif act != ACT_NONE:
        raise ValueError("the gradient of an activation needs x")
    if dtype not in _REAL:
        raise TypeError("dx is torch.float32 or torch.bfloat16")
    d = _drop(drop, device)
    handle, on = _on(stream, device)
    G, x, bias = _whole(G, on), _whole(x, on), _vector(bias, N, device, "bias", on)
    dx = _empty_as(G, dtype, on) if want_dx else None
    dbias = _empty((N,), torch.float32, G.device, on) if want_dbias else None
    size = _layer_bytes("lba_dropout_bwd_workspace_bytes", M, N) if want_dbias else 0
    ws = _scratch(size, G.device, on)
    _check(lib().lba_dropout_bwd(_at(G), _TYPE[G.dtype], _at(x), _TYPE[dtype], scale, _at(bias), act, d, _at(dx), _at(dbias), M, N,
                                 _at(ws), size, handle))
    return dx, dbias


def _codes2(A, B, gated):
    """(M, N, K, device) of the operands of a dense product: A [..., K], B [N, K], gated [2 N, K]."""
    M, K, device = _rows(A, "A", (torch.uint8,))
    if B.dtype != torch.uint8 or B.get_device() != device:
        raise TypeError("B must be a tensor of torch.uint8 codes on A's device")
    if B.dim() != 2 or B.shape[1] != K or (gated and B.shape[0] % 2):
        raise ValueError("B must be [%s, %d]" % ("2 N" if gated else "N", K))
    return M, B.shape[0] // 2 if gated else B.shape[0], K, device


def dense(A, B, fmt_a=_E4M3, fmt_b=_E4M3, bias=None, act=ACT_NONE, residual=None, drop=None, gated=False, out_dtype=torch.float32,
          out_fmt=None, out=None, stream=None):
    """residual + keep * act(A . B^T + bias) / (1 - p) on codes A [..., K], B [N, K] with float32 accumulation; gated:
    act(A . Bg^T + bg) * (A . Bu^T + bu) with B [2 N, K] and bias [2 N], the gate's rows first.  drop = (p, seed, stream[, step]) or None."""
    M, N, K, device = _codes2(A, B, gated)
    y_type, y_fmt = _out_type(out_dtype, out_fmt)
    d = _drop(drop, device)
    handle, on = _on(stream, device)
    A, B, bias = _whole(A, on), _whole(B, on), _vector(bias, 2 * N if gated else N, device, "bias", on)
    shape = A.shape[:-1] + (N,)
    if residual is not None:
        residual = _whole(_like(residual, shape, device, "residual"), on)
    y = _output(out, A, shape, out_dtype, on)
    fa, fb, a, b = _infmt(fmt_a), _infmt(fmt_b), _at(A), _at(B)
    size = _layer_bytes("lba_dense_workspace_bytes", M, N, K, fa, fb, gated, ((a or 0) | (b or 0)) % 16 == 0)
    ws = _scratch(size, A.device, on)
    _check(lib().lba_dense(a, b, M, N, K, fa, fb, gated, _at(bias), act, d, _at(residual),
                           _TYPE[residual.dtype] if residual is not None else F32, _at(y), y_type, y_fmt, _at(ws), size, handle))
    return y


def dense_bwd(G, A, B, fmt_a=_E4M3, fmt_b=_E4M3, bias=None, act=ACT_NONE, drop=None, gated=False, want_da=True, want_db=True,
              want_dbias=False, stream=None):
    """Gradients of dense: (dA, dB of G's type, dbias float32; None where not asked for), of the operands' real values.  The sums that an
    activation or a gate needs are computed again from A, B and bias.  The residual's gradient is G."""
    M, N, K, device = _codes2(A, B, gated)
    _like(G, A.shape[:-1] + (N,), device, "G")
    d = _drop(drop, device)
    handle, on = _on(stream, device)
    cols = 2 * N if gated else N
    G, A, B, bias = _whole(G, on), _whole(A, on), _whole(B, on), _vector(bias, cols, device, "bias", on)
    dA = _empty_as(A, G.dtype, on) if want_da else None
    dB = _empty_as(B, G.dtype, on) if want_db else None
    dbias = _empty((cols,), torch.float32, A.device, on) if want_dbias else None
    fa, fb, a, b, t = _infmt(fmt_a), _infmt(fmt_b), _at(A), _at(B), _TYPE[G.dtype]
    size = _layer_bytes("lba_dense_bwd_workspace_bytes", M, N, K, fa, fb, gated, act, t, ((a or 0) | (b or 0)) % 16 == 0)
    ws = _scratch(size, A.device, on)
    _check(lib().lba_dense_bwd(_at(G), t, a, b, M, N, K, fa, fb, gated, _at(bias), act, d, _at(dA), _at(dB), _at(dbias), _at(ws), size,
                               handle))
    return dA, dB, dbias


# ---- the operators of include/lba_attention.h -------------------------------------------------
#
# Tensors of heads are [rows, heads, D], or [batch, length, heads, D], float32 or bfloat16, and may be views whose rows and heads are any distance
# apart (the queries inside the output of one product): what is read or written is where it is, and copied only where D is not the last
# axis in memory.  `starts`: an int32 device tensor [sequences + 1] of packed sequences' first rows and the end of the last, read when the
# kernels run; without it [rows, heads, D] is one sequence and [batch, length, heads, D] are `batch` of them.

def _heads(t, what, on, device=None, dtype=None):
    """(t as [rows, heads, D] with D along memory, its strides) of an input."""
    if (t.dtype is not dtype or t.get_device() != device) if dtype is not None else (t.dtype not in _REAL or t.get_device() < 0):
        raise TypeError("%s must be a tensor of %s on %s device" % (what, dtype or "torch.float32 or torch.bfloat16", "a" if dtype is None else "the call's"))
    if t.dim() == 3:
        row, head, step = t.stride()
        if step == 1 or t.size(2) == 1:
            return t, (row, head)
        t = _whole(t, on)
        return t, t.stride()[:2]
    if t.dim() < 3:
        raise ValueError("%s must be [rows, heads, D] or have more leading axes" % what)
    shape = (math.prod(t.shape[:-2]),) + tuple(t.shape[-2:])
    try:
        v = t.view(shape)
    except RuntimeError:
        v = None
    if v is None or (v.stride(2) != 1 and shape[2] != 1):
        v = _whole(t, on).view(shape)
    return v, v.stride()[:2]


def _heads_made(t):
    """The same of a contiguous output that the call has made."""
    n = t.dim()
    return t, (t.stride(n - 3), t.stride(n - 2))


def _heads_out(t, like, what):
    """The same of an output given by the caller: a view that can be written where it is, no element of which shares another's place."""
    if t.dtype != like.dtype or t.get_device() != like.get_device() or t.shape != like.shape:
        raise ValueError("%s must be a tensor %s of %s on the call's device" % (what, tuple(like.shape), like.dtype))
    try:
        v = t.view((math.prod(t.shape[:-2]),) + tuple(t.shape[-2:])) if t.dim() != 3 else t
    except RuntimeError:
        raise ValueError("%s must be a view whose leading axes are one in memory" % what) from None
    (T, H, D), (r, h, d) = v.shape, v.stride()
    if d != 1 and D > 1:
        raise ValueError("%s must have its last axis along memory" % what)
    inner, outer = ((H, h), (T, r)) if h <= r or T <= 1 else ((T, r), (H, h))
    end = D
    for n, step in (inner, outer):
        if n > 1:
            if step < end:
                raise ValueError("%s has elements that share a place" % what)
            end = (n - 1) * step + end
    return v, (r, h)


def _made(t, dtype, on):
    """A contiguous tensor of t's shape."""
    return torch.empty_like(t, dtype=dtype, memory_format=torch.contiguous_format) if on is None else _empty(t.shape, dtype, t.device, on)


def _starts(t, device, what, on):
    if t is None:
        return None
    if t.dtype != torch.int32 or t.get_device() != device or t.dim() != 1 or t.numel() < 1:
        raise ValueError("%s must be an int32 tensor [sequences + 1] on the call's device" % what)
    return _whole(t, on)


def _rope(fn, x, positions, freq, interleaved, gain, out, stream):
    device = x.get_device()
    if device < 0:
        raise TypeError("x must be a device tensor")
    handle, on = _on(stream, device)
    v, at = _heads(x, "x", on)
    T, H, D = v.shape
    at = lba_strides(*at)
    if positions.dtype not in (torch.int32, torch.int64) or positions.get_device() != device or positions.shape != x.shape[:-2]:
        raise ValueError("positions must be an int32 or int64 tensor %s on the call's device" % (tuple(x.shape[:-2]),))
    if freq.dtype != torch.float64 or freq.get_device() != device or freq.dim() != 1 or 2 * freq.numel() > D:
        raise ValueError("freq must be a float64 tensor of at most %d elements on the call's device" % (D // 2))
    positions, freq = _whole(positions, on), _whole(freq, on)
    y = _made(x, x.dtype, on) if out is None else out
    w, y_at = _heads_made(y) if out is None else _heads_out(y, x, "out")
    _check(fn(_at(v), at, _TYPE[x.dtype], _at(positions), 64 if positions.dtype is torch.int64 else 32, _at(freq), freq.numel(), interleaved, gain, _at(w),
              lba_strides(*y_at), T, H, D, handle))
    return y


def rope(x, positions, freq, interleaved=False, gain=1.0, out=None, stream=None):
    """Rotary positions on x [..., heads, D]: the pairs (i, i + R / 2), interleaved (2 i, 2 i + 1), of the first R = 2 * len(freq) elements of a head
    are turned by positions * freq and scaled by gain; the rest is copied.  positions: int32 or int64 of x's leading shape; freq: float64,
    radians a position.  out may be x."""
    return _rope(lib().lba_rope, x, positions, freq, interleaved, gain, out, stream)


def rope_bwd(G, positions, freq, interleaved=False, gain=1.0, out=None, stream=None):
    """The gradient of rope: G turned back.  out may be G."""
    return _rope(lib().lba_rope_bwd, G, positions, freq, interleaved, gain, out, stream)


def _attn(q, k, v, starts, starts_k, causal, scale, clear, fine, on, device):
    """(lba_attn, (q, k, v, starts, starts_k) as they are read) of a call, which keeps them all until the kernels are launched: copies among them are
    nobody else's."""
    n, qs, ks = q.dim(), q.shape, k.shape
    if n not in (3, 4) or len(ks) != n or ks != v.shape or ks[-1] != qs[-1]:
        raise ValueError("q must be [rows, heads, D] or [batch, length, heads, D], k and v alike")
    H, KV, D = qs[-2], ks[-2], qs[-1]
    if H and (not KV or H % KV):
        raise ValueError("%d query heads do not share %d heads of keys" % (H, KV))
    if not 1 <= D <= 128:
        raise ValueError("heads have 1 to 128 elements")
    if starts is None:
        if starts_k is not None:
            raise ValueError("starts_k needs starts")
        count = qs[0] if n == 4 else 1
        if n == 4 and ks[0] != count:
            raise ValueError("q and k have different batches")
    else:
        if n != 3:
            raise ValueError("packed sequences are [rows, heads, D]")
        starts = _starts(starts, device, "starts", on)
        count = starts.numel() - 1
        if starts_k is None:
            if ks[0] != qs[0]:
                raise ValueError("q and k have different rows: starts_k is needed")
        else:
            starts_k = _starts(starts_k, device, "starts_k", on)
            if starts_k.numel() != count + 1:
                raise ValueError("starts and starts_k are of different sequences")
    dtype = q.dtype
    (q, q_at), (k, k_at), (v, v_at) = _heads(q, "q", on), _heads(k, "k", on, device, dtype), _heads(v, "v", on, device, dtype)
    a = lba_attn(q.size(0), k.size(0), count, _at(starts), _at(starts_k), H, KV, D, _TYPE[dtype] | (FINE if fine else 0), causal, clear, D ** -0.5 if scale is None else scale,
                 q_at, k_at, v_at)
    return a, (q, k, v, starts, starts_k)


@functools.lru_cache(maxsize=1024)
def _attn_bytes_of(name, T, Tk, count, starts, starts_k, H, KV, D, type):
    a = lba_attn(T, Tk, count, 256 if starts else None, 256 if starts_k else None, H, KV, D, type)
    return getattr(lib(), name)(a)


def _attn_bytes(name, a):
    """A workspace's size, which the library derives from the shape, and from which lists there are."""
    return _attn_bytes_of(name, a.T, a.Tk, a.count, bool(a.starts), bool(a.starts_k), a.H, a.KV, a.D, a.type)


def attention(q, k, v, starts=None, starts_k=None, causal=True, scale=None, out_dtype=None, out_fmt=None, want_stats=False, out=None, stream=None, fine=False):
    """softmax(scale * q . k^T) . v of packed sequences: query head h reads head h * KV // H of k and v, and, causal, query i of n sees key j of m
    iff j <= i + m - n.  starts_k: the keys' sequences where they are not the queries'.  scale: D^-1/2 by default.  Returns o of q's
    shape and out_dtype (q's by default; torch.uint8 codes need out_fmt), and with want_stats (o, lse), float32 of q.shape[:-1], which
    attention_bwd reads.  Rows of no sequence are zeros, in `out` left as they were, and in lse -infinity.  Weights of bfloat16 inputs are rounded to bfloat16 for
    the product with v, but for outputs of float32, and with `fine` not for any: it takes up to twice as long."""
    device = q.get_device()
    dtype = out_dtype or q.dtype
    o_type, fmt = _out_type(dtype, out_fmt)
    if device < 0:
        raise TypeError("q must be a device tensor")
    handle, on = _on(stream, device)
    a, held = _attn(q, k, v, starts, starts_k, causal, scale, out is None, fine, on, device)
    q3, k3, v3 = held[:3]
    o = _made(q, dtype, on) if out is None else _output(out, q, q.shape, dtype, on)
    lse = _empty(q.shape[:-1], torch.float32, q.device, on) if want_stats else None
    if want_stats and out is not None and starts is not None:        # the library leaves rows of no sequence as they are in both or in neither
        lse.fill_(-math.inf) if on is None else _of_pool(lambda: lse.fill_(-math.inf), on)
    size = _attn_bytes("lba_attention_workspace_bytes", a)
    ws = _scratch(size, q.device, on)
    _check(lib().lba_attention(a, _at(q3), _at(k3), _at(v3), _at(o), o_type, fmt, _at(lse), _at(ws), size, handle))
    return (o, lse) if want_stats else o


def attention_bwd(G, q, k, v, o, lse, starts=None, starts_k=None, causal=True, scale=None, out=None, stream=None, fine=False):
    """Gradients of attention: (dq, dk, dv) of the inputs' shapes and type, from G = dL/do and o and lse as the forward call gave them (o of
    q's type).  out: three tensors, or views of one, to write them to; rows of no sequence are left as they were there, and zeros elsewhere.
    fine, for bfloat16: rowsum(G * o) has no rounding of o for any query, not only for those that see up to 512 keys;
    the call takes up to 1.3 times as long.  It tells where values have a mean."""
    device = q.get_device()
    if device < 0:
        raise TypeError("q must be a device tensor")
    _like(G, q.shape, device, "G", (q.dtype,))
    _like(o, q.shape, device, "o", (q.dtype,))
    _like(lse, q.shape[:-1], device, "lse", (torch.float32,))
    handle, on = _on(stream, device)
    a, held = _attn(q, k, v, starts, starts_k, causal, scale, out is None, fine, on, device)
    q3, k3, v3 = held[:3]
    G, o, lse = _whole(G, on), _whole(o, on), _whole(lse, on)
    if out is None:
        got = (_made(q, q.dtype, on), _made(k, k.dtype, on), _made(v, v.dtype, on))
        (dq, dq_at), (dk, dk_at), (dv, dv_at) = (_heads_made(t) for t in got)
    else:
        got = tuple(out)
        (dq, dq_at), (dk, dk_at), (dv, dv_at) = (_heads_out(t, w, n) for t, w, n in zip(got, (q, k, v), ("dq", "dk", "dv")))
    size = _attn_bytes("lba_attention_bwd_workspace_bytes", a)
    ws = _scratch(size, q.device, on)
    _check(lib().lba_attention_bwd(a, _at(G), _at(q3), _at(k3), _at(v3), _at(o), _at(lse), _at(dq), lba_strides(*dq_at), _at(dk),
                                   lba_strides(*dk_at), _at(dv), lba_strides(*dv_at), _at(ws), size, handle))
    return got


class KVCache(typing.NamedTuple):
    """Keys and values in 4 bits: codes uint8 [pages, KV, page, D / 2] and powers of two uint8 [pages, KV, page, D / 32] (include/lba_attention.h)."""
    k: torch.Tensor
    k_scale: torch.Tensor
    v: torch.Tensor
    v_scale: torch.Tensor


def kv_cache(pages, page, heads, D, device="cuda"):
    """An empty KVCache of `pages` pages of `page` tokens each."""
    if D % 32 or not 32 <= D <= 128:
        raise ValueError("heads of a cache have 32, 64, 96 or 128 elements")
    make = lambda n: torch.zeros((pages, heads, page, n), dtype=torch.uint8, device=device)  # noqa: E731
    return KVCache(make(D // 2), make(D // 32), make(D // 2), make(D // 32))


def _cache4(cache, table, lens, device, on):
    """(lba_cache4, what it points to, to be kept as with _attn)."""
    k, k_scale, v, v_scale = cache
    shape, powers = k.shape, k_scale.shape
    if len(shape) != 4 or shape[3] % 16 or not 16 <= shape[3] <= 64 or powers != shape[:3] + (shape[3] // 16,):
        raise ValueError("a cache's codes are [pages, heads, page, D / 2] with D 32, 64, 96 or 128, its powers [pages, heads, page, D / 32]")
    if v.shape != shape or v_scale.shape != powers:
        raise ValueError("a cache's keys and values are of one shape")
    for t in cache:
        if t.dtype is not torch.uint8 or t.get_device() != device or not t.is_contiguous():
            raise ValueError("a cache's tensors are contiguous torch.uint8 on the call's device")
    if table.dtype is not torch.int32 or table.get_device() != device or table.dim() != 2:
        raise ValueError("table must be an int32 tensor [sequences, pages of each] on the call's device")
    count, row = table.shape
    if lens.dtype is not torch.int32 or lens.get_device() != device or lens.dim() != 1 or lens.size(0) != count:
        raise ValueError("lens must be an int32 tensor [sequences] on the call's device")
    table, lens = _whole(table, on), _whole(lens, on)
    c = lba_cache4(_at(k), _at(k_scale), _at(v), _at(v_scale), shape[0], row, count, _at(table), _at(lens), shape[2], shape[1], 2 * shape[3])
    return c, (table, lens)


def _cache_starts(starts, count, shape, device, on):
    if starts is not None:
        starts = _starts(starts, device, "starts", on)
        if starts.numel() != count + 1:
            raise ValueError("starts and table are of different sequences")
        if len(shape) != 3:
            raise ValueError("packed sequences are [rows, heads, D]")
    elif (len(shape) == 4 and shape[0] != count) or (len(shape) == 3 and count != 1 and shape[0] != count):
        raise ValueError("without starts rows are [sequences, length, heads, D], or [sequences, heads, D] for one token each")
    return starts


def cache_write(k, v, cache, table, starts, lens, stream=None):
    """Writes the newest tokens' keys and values to their pages: rows starts[b] .. of k and v [rows, KV, D] are the last ones of sequence b, which has
    lens[b] tokens with them; position p of it is in page table[b, p // page].  starts None: [sequences, length, KV, D], or
    [sequences, KV, D] for a token each."""
    device = k.get_device()
    if device < 0 or k.shape != v.shape:
        raise TypeError("k and v must be device tensors of one shape")
    handle, on = _on(stream, device)
    c, held = _cache4(cache, table, lens, device, on)
    starts = _cache_starts(starts, c.count, k.shape, device, on)
    if tuple(k.shape[-2:]) != (c.KV, c.D):
        raise ValueError("k and v must be [rows, %d, %d]" % (c.KV, c.D))
    (k3, k_at), (v3, v_at) = _heads(k, "k", on), _heads(v, "v", on, device, k.dtype)
    _check(lib().lba_cache_write(c, _at(starts), k3.size(0), _at(k3), lba_strides(*k_at), _at(v3), lba_strides(*v_at), _TYPE[k.dtype], handle))


def cache_read(cache, table, starts, lens, rows, out_dtype=torch.bfloat16, out=None, stream=None):
    """The newest tokens' keys and values [rows, KV, D] back from their pages, in the arrangement of cache_write, of out_dtype: exact in float32 and
    bfloat16.  starts None: rows / sequences tokens each.  out: two tensors to write them to; rows of no sequence are left as they were there,
    and zeros elsewhere."""
    device = cache.k.get_device()
    if device < 0:
        raise TypeError("a cache is on a device")
    if out_dtype not in _REAL:
        raise TypeError("keys and values are torch.float32 or torch.bfloat16")
    handle, on = _on(stream, device)
    c, held = _cache4(cache, table, lens, device, on)
    if starts is None:
        if rows % max(c.count, 1) or (rows and not c.count):
            raise ValueError("%d rows of %d sequences need starts" % (rows, c.count))
    else:
        starts = _cache_starts(starts, c.count, (rows, c.KV, c.D), device, on)
    shape = (rows, c.KV, c.D)
    if out is None:
        got = (_empty(shape, out_dtype, cache.k.device, on), _empty(shape, out_dtype, cache.k.device, on))
        (k3, k_at), (v3, v_at) = (_heads_made(t) for t in got)
    else:
        got = tuple(out)
        for t in got:
            if tuple(t.shape) != shape or t.dtype != out_dtype or t.get_device() != device:
                raise ValueError("out must be two tensors %s of %s on the call's device" % (shape, out_dtype))
        (k3, k_at), (v3, v_at) = (_heads_out(t, got[0], "out") for t in got)
    _check(lib().lba_cache_read(c, _at(starts), rows, _at(k3), lba_strides(*k_at), _at(v3), lba_strides(*v_at), _TYPE[out_dtype], out is None, handle))
    return got


def cache_attention(q, cache, table, lens, scale=None, out_dtype=None, out_fmt=None, out=None, stream=None, fine=False):
    """Attention of new tokens over a cache: q [sequences, heads, D] for one token each, or [sequences, tokens, heads, D], which have been written
    (lens counts them): each sees the positions up to its own.  Returns o of q's shape and out_dtype (q's by default; torch.uint8 codes need
    out_fmt); a query that sees nothing has zeros.  fine: as in attention."""
    device = q.get_device()
    dtype = out_dtype or q.dtype
    o_type, fmt = _out_type(dtype, out_fmt)
    if device < 0:
        raise TypeError("q must be a device tensor")
    handle, on = _on(stream, device)
    c, held = _cache4(cache, table, lens, device, on)
    if q.dim() not in (3, 4) or q.shape[0] != c.count or q.shape[-1] != c.D:
        raise ValueError("q must be [%d, heads, %d] or [%d, tokens, heads, %d]" % (c.count, c.D, c.count, c.D))
    H = q.shape[-2]
    if H and (not c.KV or H % c.KV):
        raise ValueError("%d query heads do not share %d heads of keys" % (H, c.KV))
    fresh = q.shape[1] if q.dim() == 4 else 1
    q3, q_at = _heads(q, "q", on)
    o = _made(q, dtype, on) if out is None else _output(out, q, q.shape, dtype, on)
    size = _layer_bytes("lba_cache_attention_workspace_bytes", c.count, c.table_row, c.page, fresh, H, c.KV, c.D)
    ws = _scratch(size, q.device, on)
    _check(lib().lba_cache_attention(c, _at(q3), lba_strides(*q_at), _TYPE[q.dtype] | (FINE if fine else 0), fresh, H, c.D ** -0.5 if scale is None else scale, _at(o), o_type,
                                     fmt, _at(ws), size, handle))
    return o
