"""Thin Python binding of libnm_mvue (the C ABI declared in include/nm_mvue.h).

Argument marshalling only: torch supplies device memory and the current HIP stream, every
step of the path runs in the library's kernels.  There is no fallback: if the shared library
is missing, or a call returns an error status, an exception is raised.
"""
from __future__ import annotations

import ctypes as C
import math
import os
import warnings
from typing import Optional, Tuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libnm_mvue.so")

NM_F32, NM_BF16, NM_F32_BF16X3 = 0, 1, 2
_lib = None
_native = None            # the common forms of the hot calls in C++ (csrc/nm_torch.cpp)


class NmError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"nm_status {status}: {message}")
        self.status = status


def load():
    """Load libnm_mvue.so (built in-tree by ``python -m paper_2203_10991_amd.build``)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is not built: run `python -m paper_2203_10991_amd.build` (needs hipcc)")
    lib = C.CDLL(LIB_PATH)
    vp, i64, u64, u32, i32, f32, sz = C.c_void_p, C.c_int64, C.c_uint64, C.c_uint32, C.c_int, C.c_float, C.c_size_t
    lib.mvue_prune_1of2.argtypes = [vp, i64, i64, i64, i32, u64, u32, vp, vp, vp, i64, vp]
    lib.mvue_prune_2of4.argtypes = [vp, i64, i64, i64, i32, u64, u32, i32, vp, vp, vp, i64, vp]
    lib.mvue_prune_1of4.argtypes = [vp, i64, i64, i64, i32, u64, u32, vp, vp, vp, i64, vp]
    lib.mvue_prune_1of4.restype = i32
    lib.mvue_prune_2of4_producer.argtypes = [vp, i64, vp, i64, i64, i64, i32, u64, u32, i32, vp, i64, vp, vp, vp]
    lib.mvue_prune_2of4_producer.restype = i32
    lib.mvue_prune_1of2_producer.argtypes = [vp, i64, vp, i64, i64, i64, i32, u64, u32, vp, i64, vp, vp, vp]
    lib.mvue_prune_1of2_producer.restype = i32
    lib.mvue_prune_4of8_approx.argtypes = [vp, i64, i64, i64, i32, u64, u32, vp, vp, vp, i64, vp]
    lib.mvue_prune_4of8_approx.restype = i32
    lib.nm_prune_greedy.argtypes = [vp, i64, i64, i64, i32, i32, i32, vp, vp, vp, i64, vp]
    lib.nm_prune_greedy.restype = i32
    lib.nm_rw_mix_probe.argtypes = [vp, vp, i64, vp]
    lib.nm_rw_mix_probe.restype = i32
    lib.mvue_prune_2of4_t.argtypes = [vp, i64, i64, i64, i32, u64, u32, i32, vp, vp, vp]
    lib.mvue_prune_2of4_t.restype = i32
    lib.mvue_prune_1of2_t.argtypes = [vp, i64, i64, i64, i32, u64, u32, vp, vp, vp]
    lib.mvue_prune_1of2_t.restype = i32
    lib.nm_compress.argtypes = [vp, i64, i64, i64, i32, i32, i32, vp, vp, vp, vp]
    lib.nm_update_gemm.argtypes = [vp, vp, vp, i64, vp, i64, i64, i64, i64, i32, f32, vp, sz, vp]
    lib.nm_update_gemm_workspace.argtypes = [i64, i64, i64, i32]
    lib.nm_update_gemm_static.argtypes = [vp, vp, vp, i64, vp, i64, i64, i64, i64, i32, f32, vp]
    lib.nm_update_gemm_static.restype = i32
    lib.nm_update_gemm_static_max.argtypes = []
    lib.nm_update_gemm_static_max.restype = sz
    lib.nm_update_gemm_shifted.argtypes = [vp, vp, vp, i64, i64, vp, i32, vp, i64, i64, i64, i32, f32, vp, sz, vp]
    lib.nm_update_gemm_shifted.restype = i32
    lib.nm_update_gemm_shifted_workspace.argtypes = [i64, i64, i64, i32]
    lib.nm_update_gemm_shifted_workspace.restype = sz
    lib.nm_update_gemm_q8_shifted.argtypes = [vp, vp, vp, i64, i64, vp, i32, vp, i64, i64, i64, f32, f32, vp, sz, vp]
    lib.nm_update_gemm_q8_shifted.restype = i32
    lib.nm_update_gemm_q8_shifted_workspace.argtypes = [i64, i64, i64, i32]
    lib.nm_update_gemm_q8_shifted_workspace.restype = sz
    lib.mvue_prune_2of4_q8.argtypes = [vp, i64, i64, i64, i32, u64, u32, i32, f32, vp, vp, vp]
    lib.mvue_prune_1of2_q8.argtypes = [vp, i64, i64, i64, i32, u64, u32, f32, vp, vp, vp]
    lib.mvue_prune_1of2_q8.restype = i32
    lib.nm_update_gemm_q8.argtypes = [vp, vp, vp, i64, vp, i64, i64, i64, i64, f32, f32, vp, sz, vp]
    lib.nm_update_gemm_q8_workspace.argtypes = [i64, i64, i64]
    lib.nm_q8_scale.argtypes = [vp, i64, i64, i64, i32, f32, vp, vp]
    lib.nm_q8_scale.restype = i32
    lib.nm_cast_e4m3.argtypes = [vp, i64, i64, i64, i32, vp, vp, i64, vp]
    lib.nm_cast_e4m3.restype = i32
    lib.mvue_prune_2of4_q8_ds.argtypes = [vp, i64, i64, i64, i32, u64, u32, i32, vp, vp, vp, vp]
    lib.mvue_prune_2of4_q8_ds.restype = i32
    lib.mvue_prune_1of2_q8_ds.argtypes = [vp, i64, i64, i64, i32, u64, u32, vp, vp, vp, vp]
    lib.mvue_prune_1of2_q8_ds.restype = i32
    lib.mvue_prune_2of4_q8_t.argtypes = [vp, i64, i64, i64, i32, u64, u32, i32, f32, vp, vp, vp, vp]
    lib.mvue_prune_2of4_q8_t.restype = i32
    lib.mvue_prune_1of2_q8_t.argtypes = [vp, i64, i64, i64, i32, u64, u32, f32, vp, vp, vp, vp]
    lib.mvue_prune_1of2_q8_t.restype = i32
    lib.nm_update_gemm_q8_ds.argtypes = [vp, vp, vp, i64, vp, i64, i64, i64, i64, vp, vp, f32, vp, sz, vp]
    lib.nm_update_gemm_q8_ds.restype = i32
    lib.nm_update_gemm_q8_shifted_ds.argtypes = [vp, vp, vp, i64, i64, vp, i32, vp, i64, i64, i64, vp, vp, f32, vp, sz, vp]
    lib.nm_update_gemm_q8_shifted_ds.restype = i32
    lib.nm_conv_update.argtypes = [vp, i32, vp, i32, i64, i64, i64, i64, i64, i32, i32, i32, u64, u32, vp, vp, sz, vp]
    lib.nm_conv_update.restype = i32
    lib.nm_conv_update_workspace.argtypes = [i64, i64, i64, i64, i64, i32, i32]
    lib.nm_conv_update_workspace.restype = sz
    lib.nm_linear_update.argtypes = [vp, i64, vp, i64, vp, i64, i64, i64, i64, i32, i32, i32, u64, u32, vp, i64, vp, vp, vp, sz, vp]
    lib.nm_linear_update.restype = i32
    lib.nm_linear_update_workspace.argtypes = [i64, i64, i64, i32, i32]
    lib.nm_linear_update_workspace.restype = sz
    lib.nm_linear_forward.argtypes = [vp, i64, vp, vp, i64, i64, i64, i32, vp, vp]
    lib.nm_linear_forward.restype = i32
    lib.nm_linear_input_grad.argtypes = [vp, i64, vp, i64, i64, i64, vp, vp]
    lib.nm_linear_input_grad.restype = i32
    lib.nm_quant_i8.argtypes = [vp, i64, i64, i64, i32, vp, i64, vp, vp]
    lib.nm_quant_i8.restype = i32
    lib.nm_quant_i8_t.argtypes = [vp, i64, i64, i64, i32, vp, i64, vp, vp, sz, vp]
    lib.nm_quant_i8_t.restype = i32
    lib.nm_quant_i8_t_workspace.argtypes = [i64, i64]
    lib.nm_quant_i8_t_workspace.restype = sz
    lib.nm_gemm_i8.argtypes = [vp, i64, vp, vp, i64, vp, vp, i32, i64, i64, i64, i32, vp, i64, i32, vp]
    lib.nm_gemm_i8.restype = i32
    lib.nm_linear_i8.argtypes = [vp, i64, i32, vp, i64, vp, vp, i32, i64, i64, i64, i32, vp, i64, i32, vp, sz, vp]
    lib.nm_linear_i8.restype = i32
    lib.nm_linear_i8_workspace.argtypes = [i64, i64]
    lib.nm_linear_i8_workspace.restype = sz
    lib.nm_embed.argtypes = [vp, i64, i64, i64, i32, vp, i32, i64, f32, vp, i64, i32, vp]
    lib.nm_embed.restype = i32
    lib.nm_embed_grad.argtypes = [vp, i64, i32, vp, i32, i64, i64, i64, f32, i64, i32, vp, i64, i32, vp, sz, vp]
    lib.nm_embed_grad.restype = i32
    lib.nm_embed_grad_workspace.argtypes = [i64, i64, i64]
    lib.nm_embed_grad_workspace.restype = sz
    lib.nm_layer_norm.argtypes = [vp, i64, i32, vp, vp, i32, i64, i64, f32, vp, i64, vp, vp, vp]
    lib.nm_layer_norm.restype = i32
    lib.nm_layer_norm_grad.argtypes = [vp, i64, vp, i64, i32, vp, i32, vp, vp, i64, i64, vp, i64, vp, vp, vp, sz, vp]
    lib.nm_layer_norm_grad.restype = i32
    lib.nm_layer_norm_grad_workspace.argtypes = [i64, i64]
    lib.nm_layer_norm_grad_workspace.restype = sz
    heads = C.POINTER(_Heads)
    lib.nm_rotary.argtypes = [heads, heads, i32, i64, i64, i64, i64, i64, vp, vp, i32, i64, i32, f32, i32, vp]
    lib.nm_rotary.restype = i32
    sizes = [i64] * 6 + [i32]                                                # B, Tq, Tk, Hq, Hk, D, dtype
    lib.nm_attention.argtypes = [heads] * 4 + [vp, vp, *sizes, i32, f32, vp, vp, vp, sz, vp]
    lib.nm_attention.restype = i32
    lib.nm_attention_grad.argtypes = [heads] * 5 + [vp, vp, *sizes, i32, f32, vp, vp, heads, heads, heads, vp, sz, vp]
    lib.nm_attention_grad.restype = i32
    for f in (lib.nm_attention_workspace, lib.nm_attention_grad_workspace):
        f.argtypes, f.restype = sizes, sz
    lib.nm_adamw.argtypes = [vp, i32, i32, i32, i32, C.c_double, C.c_double, C.c_double, C.c_double, C.c_double, i64, f32, vp, u64, vp]
    lib.nm_adamw.restype = i32
    for f in (lib.mvue_prune_1of2, lib.mvue_prune_2of4, lib.nm_compress, lib.nm_update_gemm, lib.mvue_prune_2of4_q8,
              lib.nm_update_gemm_q8):
        f.restype = i32
    lib.nm_update_gemm_workspace.restype = sz
    lib.nm_update_gemm_q8_workspace.restype = sz
    lib.nm_last_error.restype = C.c_char_p
    lib.nm_version.restype = C.c_char_p
    try:
        from . import _nm_torch as native
        native.bind({f: C.cast(getattr(lib, f), vp).value for f in (
            "mvue_prune_1of2", "mvue_prune_2of4", "nm_update_gemm", "nm_update_gemm_workspace", "nm_linear_update", "nm_linear_update_workspace",
            "nm_linear_forward", "nm_linear_input_grad", "nm_adamw", "nm_embed", "nm_embed_grad", "nm_embed_grad_workspace",
            "nm_quant_i8", "nm_quant_i8_t", "nm_quant_i8_t_workspace", "nm_linear_i8", "nm_linear_i8_workspace",
            "nm_layer_norm", "nm_layer_norm_grad", "nm_layer_norm_grad_workspace", "nm_rotary", "nm_attention", "nm_attention_workspace",
            "nm_attention_grad", "nm_attention_grad_workspace")}, _raw_stream or (lambda d: torch.cuda.current_stream(d).cuda_stream))
    except ImportError as e:
        warnings.warn(f"_nm_torch.so is not built for this torch ({e}): every call takes the slower way through ctypes and linear layers take the "
                      "framework's products until `python -m paper_2203_10991_amd.build` has run")
        native = _NoNative
    global _native
    _native, _lib = native, lib
    return lib


class _Heads(C.Structure):
    _fields_ = [("data", C.c_void_p), ("batch", C.c_int64), ("token", C.c_int64), ("head", C.c_int64)]


class _NoNative:
    """In the place of _nm_torch: no call is its own."""
    prune = update_gemm = linear_update = linear_forward = linear_input_grad = adamw = embed = embed_grad = quant_i8 = linear_i8 = staticmethod(lambda *a: None)
    layer_norm = layer_norm_grad = rotary = attention = attention_grad = staticmethod(lambda *a: None)


def _native_result(r):
    """What a call of _native gave: its outputs, None where api.py's own way is to be taken, or an error status that is raised here."""
    if type(r) is int:
        _check(r)
    return r


def _check(rc: int):
    if rc != 0:
        raise NmError(rc, load().nm_last_error().decode())


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return NM_F32
    if t.dtype == torch.bfloat16:
        return NM_BF16
    raise TypeError(f"nm_mvue tensors are float32 or bfloat16, got {t.dtype}")


# (a Stream object made for every call costs 1.7 us; the function is not public: a torch without it takes the public way)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(t: torch.Tensor) -> int:
    if t.is_cuda and _raw_stream is not None:
        return _raw_stream(t.get_device())
    return torch.cuda.current_stream(t.device).cuda_stream             # raises where t is not a GPU tensor


def _rowmajor(t: torch.Tensor, what: str) -> int:
    if t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1):
        raise ValueError(f"{what} must be a 2-D tensor with unit column stride")
    return t.stride(0) if t.shape[0] > 1 else max(t.shape[1], t.stride(0))


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def alloc_compressed(T: int, O: int, dtype: torch.dtype, device) -> Tuple[torch.Tensor, torch.Tensor]:
    """Buffers of the group format: vals[T/16, O, 8] and meta[T/16, O] (int16 holds the uint16 words)."""
    return (torch.empty((T // 16, O, 8), dtype=dtype, device=device),
            torch.empty((T // 16, O), dtype=torch.int16, device=device))


def _prune(which: str, g, seed, stream_id, mode, vals, meta, dense_out, want_dense):
    lib = load()
    if vals is None and meta is None and dense_out is None and not want_dense and which != "1of4":
        r = _native_result(_native.prune(2 if which == "1of2" else 4, g, seed, stream_id, mode))
        if r is not None:
            return r[0], r[1], None
    if not g.is_cuda:
        raise ValueError("g must live on the GPU")
    T, O = g.shape
    ldg = _rowmajor(g, "g")
    if vals is None or meta is None:
        vals, meta = alloc_compressed(T - T % 16, O, g.dtype, g.device)
    if dense_out is None and want_dense:
        dense_out = torch.empty((T, O), dtype=g.dtype, device=g.device)
    ldd = _rowmajor(dense_out, "dense_out") if dense_out is not None else 0
    if which == "1of4":
        rc = lib.mvue_prune_1of4(_ptr(g), T, O, ldg, _dtype_code(g), seed, stream_id, _ptr(vals), _ptr(meta),
                                 _ptr(dense_out), ldd, _stream(g))
    elif which == "1of2":
        rc = lib.mvue_prune_1of2(_ptr(g), T, O, ldg, _dtype_code(g), seed, stream_id, _ptr(vals), _ptr(meta),
                                 _ptr(dense_out), ldd, _stream(g))
    else:
        rc = lib.mvue_prune_2of4(_ptr(g), T, O, ldg, _dtype_code(g), seed, stream_id, mode, _ptr(vals), _ptr(meta),
                                 _ptr(dense_out), ldd, _stream(g))
    _check(rc)
    return vals, meta, dense_out


def mvue_prune_1of2(g: torch.Tensor, seed: int = 0, stream_id: int = 0, vals=None, meta=None, dense_out=None,
                    want_dense: bool = False):
    """MVUE 1:2 prune + compress of g[T x O] along T.  Returns (vals, meta, dense_out or None)."""
    return _prune("1of2", g, seed, stream_id, 0, vals, meta, dense_out, want_dense)


def mvue_prune_1of4(g: torch.Tensor, seed: int = 0, stream_id: int = 0, vals=None, meta=None, dense_out=None,
                    want_dense: bool = False):
    """MVUE 1:4 prune of g[T x O] along T, stored in the 2:4 group format.  Returns (vals, meta, dense_out or None)."""
    return _prune("1of4", g, seed, stream_id, 0, vals, meta, dense_out, want_dense)


def mvue_prune_2of4(g: torch.Tensor, seed: int = 0, stream_id: int = 0, mode: int = 0, vals=None, meta=None,
                    dense_out=None, want_dense: bool = False):
    """Optimal MVUE 2:4 prune + compress of g[T x O] along T.  Returns (vals, meta, dense_out or None)."""
    return _prune("2of4", g, seed, stream_id, mode, vals, meta, dense_out, want_dense)


def mvue_prune_producer(u: torch.Tensor, d: torch.Tensor, nm: str = "2:4", seed: int = 0, stream_id: int = 0, mode: int = 0,
                        g_out=None, vals=None, meta=None):
    """g = u * d (eq. (2): d = f'(z), u = W^T g_next) written dense, and its MVUE prune + compress, in one pass.
    Returns (g_out, vals, meta)."""
    lib = load()
    if not (u.is_cuda and d.is_cuda) or u.shape != d.shape or u.dtype != d.dtype:
        raise ValueError("u and d must be GPU tensors of one shape and dtype")
    T, O = u.shape
    if g_out is None:
        g_out = torch.empty((T, O), dtype=u.dtype, device=u.device)
    if vals is None or meta is None:
        vals, meta = alloc_compressed(T - T % 16, O, u.dtype, u.device)
    if nm == "1:2":
        rc = lib.mvue_prune_1of2_producer(_ptr(u), _rowmajor(u, "u"), _ptr(d), _rowmajor(d, "d"), T, O, _dtype_code(u), seed, stream_id,
                                          _ptr(g_out), _rowmajor(g_out, "g_out"), _ptr(vals), _ptr(meta), _stream(u))
    else:
        rc = lib.mvue_prune_2of4_producer(_ptr(u), _rowmajor(u, "u"), _ptr(d), _rowmajor(d, "d"), T, O, _dtype_code(u), seed, stream_id,
                                          mode, _ptr(g_out), _rowmajor(g_out, "g_out"), _ptr(vals), _ptr(meta), _stream(u))
    _check(rc)
    return g_out, vals, meta


def mvue_prune_4of8_approx(g: torch.Tensor, seed: int = 0, stream_id: int = 0, vals=None, meta32=None, dense_out=None,
                           want_dense: bool = False):
    """approx-MVUE 4:8 prune + compress of g[T x O] along T.  Returns (vals[T/16, O, 8], meta32[T/16, O] int32, dense_out or None)."""
    lib = load()
    if not g.is_cuda:
        raise ValueError("g must live on the GPU")
    T, O = g.shape
    ldg = _rowmajor(g, "g")
    if vals is None or meta32 is None:
        vals = torch.empty(((T - T % 16) // 16, O, 8), dtype=g.dtype, device=g.device)
        meta32 = torch.empty(((T - T % 16) // 16, O), dtype=torch.int32, device=g.device)
    if dense_out is None and want_dense:
        dense_out = torch.empty((T, O), dtype=g.dtype, device=g.device)
    ldd = _rowmajor(dense_out, "dense_out") if dense_out is not None else 0
    _check(lib.mvue_prune_4of8_approx(_ptr(g), T, O, ldg, _dtype_code(g), seed, stream_id, _ptr(vals), _ptr(meta32),
                                      _ptr(dense_out), ldd, _stream(g)))
    return vals, meta32, dense_out


def nm_prune_greedy(g: torch.Tensor, n: int, m: int, vals=None, meta=None, dense_out=None, want_dense: bool = False):
    """Greedy n:m prune + compress (keep the n largest magnitudes of every block along T, unchanged): the paper's
    biased baseline.  Returns (vals, meta, dense_out or None)."""
    lib = load()
    if not g.is_cuda:
        raise ValueError("g must live on the GPU")
    T, O = g.shape
    ldg = _rowmajor(g, "g")
    if vals is None or meta is None:
        vals, meta = alloc_compressed(T - T % 16, O, g.dtype, g.device)
    if dense_out is None and want_dense:
        dense_out = torch.empty((T, O), dtype=g.dtype, device=g.device)
    ldd = _rowmajor(dense_out, "dense_out") if dense_out is not None else 0
    _check(lib.nm_prune_greedy(_ptr(g), T, O, ldg, _dtype_code(g), n, m, _ptr(vals), _ptr(meta), _ptr(dense_out), ldd, _stream(g)))
    return vals, meta, dense_out


def _prune_transposed(gT: torch.Tensor, vals, meta):
    if not gT.is_cuda:
        raise ValueError("gT must live on the GPU")
    O, T = gT.shape
    ldt = _rowmajor(gT, "gT")
    if vals is None or meta is None:
        vals, meta = alloc_compressed(T - T % 16, O, gT.dtype, gT.device)
    return T, O, ldt, vals, meta


def mvue_prune_2of4_t(gT: torch.Tensor, seed: int = 0, stream_id: int = 0, mode: int = 0, vals=None, meta=None):
    """MVUE 2:4 prune + compress of a gradient stored transposed, gT[O x T] (tokens contiguous).  Returns (vals, meta)."""
    lib = load()
    T, O, ldt, vals, meta = _prune_transposed(gT, vals, meta)
    _check(lib.mvue_prune_2of4_t(_ptr(gT), T, O, ldt, _dtype_code(gT), seed, stream_id, mode, _ptr(vals), _ptr(meta), _stream(gT)))
    return vals, meta


def mvue_prune_1of2_t(gT: torch.Tensor, seed: int = 0, stream_id: int = 0, vals=None, meta=None):
    """MVUE 1:2 prune + compress of a gradient stored transposed, gT[O x T] (tokens contiguous).  Returns (vals, meta)."""
    lib = load()
    T, O, ldt, vals, meta = _prune_transposed(gT, vals, meta)
    _check(lib.mvue_prune_1of2_t(_ptr(gT), T, O, ldt, _dtype_code(gT), seed, stream_id, _ptr(vals), _ptr(meta), _stream(gT)))
    return vals, meta


def nm_compress(dense: torch.Tensor, n: int, m: int, vals=None, meta=None, bad_blocks: Optional[torch.Tensor] = None):
    """Compress an n:m-sparse dense tensor into the group format.  Returns (vals, meta)."""
    lib = load()
    T, O = dense.shape
    ld = _rowmajor(dense, "dense")
    if vals is None or meta is None:
        vals, meta = alloc_compressed(T - T % 16, O, dense.dtype, dense.device)
    _check(lib.nm_compress(_ptr(dense), T, O, ld, _dtype_code(dense), n, m, _ptr(vals), _ptr(meta),
                           _ptr(bad_blocks), _stream(dense)))
    return vals, meta


def _gemm_mode(dtype: torch.dtype, f32_as_bf16x3: bool) -> int:
    if dtype == torch.float32:
        return NM_F32_BF16X3 if f32_as_bf16x3 else NM_F32
    return NM_BF16


def nm_update_gemm_workspace(T: int, O: int, I: int, dtype: torch.dtype, f32_as_bf16x3: bool = False) -> int:
    return int(load().nm_update_gemm_workspace(T, O, I, _gemm_mode(dtype, f32_as_bf16x3)))


def nm_update_gemm(vals: torch.Tensor, meta: torch.Tensor, h: torch.Tensor, dW: Optional[torch.Tensor] = None,
                   beta: float = 0.0, workspace: Optional[torch.Tensor] = None, f32_as_bf16x3: bool = False) -> torch.Tensor:
    """dW[O x I] = beta*dW + decompress(vals, meta)^T h  (binary32 output).

    f32_as_bf16x3 (binary32 tensors only): multiply through three bf16 terms per value on the sparse 16-bit path."""
    lib = load()
    if dW is None and workspace is None and beta == 0.0:
        r = _native_result(_native.update_gemm(vals, meta, h, f32_as_bf16x3))
        if r is not None:
            return r
    G, O, _ = vals.shape
    T, I = h.shape
    if T != G * 16:
        raise ValueError(f"h has {T} rows, the compressed operand covers {G * 16}")
    ldh = _rowmajor(h, "h")
    if dW is None:
        dW = torch.empty((O, I), dtype=torch.float32, device=h.device)
    lddw = _rowmajor(dW, "dW")
    if vals.dtype != h.dtype:
        raise TypeError("vals and h must have the same dtype")
    need = nm_update_gemm_workspace(T, O, I, h.dtype, f32_as_bf16x3)
    if need and (workspace is None or workspace.numel() * workspace.element_size() < need):
        workspace = torch.empty(need, dtype=torch.uint8, device=h.device)
    wbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib.nm_update_gemm(_ptr(vals), _ptr(meta), _ptr(h), ldh, _ptr(dW), lddw, T, O, I, _gemm_mode(h.dtype, f32_as_bf16x3),
                              float(beta), _ptr(workspace), wbytes, _stream(h)))
    return dW


def nm_update_gemm_static(vals: torch.Tensor, meta: torch.Tensor, h: torch.Tensor, dW: torch.Tensor, beta: float = 0.0,
                          f32_as_bf16x3: bool = False) -> torch.Tensor:
    """nm_update_gemm without a workspace: split-K partial sums go to the library's static device array.  The caller
    passes dW; nothing is allocated."""
    lib = load()
    G, O, _ = vals.shape
    T, I = h.shape
    if T != G * 16:
        raise ValueError(f"h has {T} rows, the compressed operand covers {G * 16}")
    if vals.dtype != h.dtype:
        raise TypeError("vals and h must have the same dtype")
    _check(lib.nm_update_gemm_static(_ptr(vals), _ptr(meta), _ptr(h), _rowmajor(h, "h"), _ptr(dW), _rowmajor(dW, "dW"), T, O, I,
                                     _gemm_mode(h.dtype, f32_as_bf16x3), float(beta), _stream(h)))
    return dW


def nm_update_gemm_static_max() -> int:
    return int(load().nm_update_gemm_static_max())


# ---- 8-bit neural gradients (e5m2, stochastic rounding) on top of 2:4 sparsity

def alloc_compressed_q8(T: int, O: int, device) -> Tuple[torch.Tensor, torch.Tensor]:
    """Buffers of the 8-bit group format: vals8[T/32, O, 16] (uint8 e5m2 codes) and meta32[T/32, O] (int32 holds the words)."""
    return (torch.empty((T // 32, O, 16), dtype=torch.uint8, device=device),
            torch.empty((T // 32, O), dtype=torch.int32, device=device))


def mvue_prune_2of4_q8(g: torch.Tensor, seed: int = 0, stream_id: int = 0, mode: int = 0, scale=1.0,
                       vals8=None, meta32=None):
    """MVUE 2:4 prune of g[T x O] along T with kept values scaled and rounded stochastically to e5m2.  Returns (vals8, meta32)."""
    lib = load()
    if not g.is_cuda:
        raise ValueError("g must live on the GPU")
    T, O = g.shape
    ldg = _rowmajor(g, "g")
    if vals8 is None or meta32 is None:
        vals8, meta32 = alloc_compressed_q8(T - T % 32, O, g.device)
    if isinstance(scale, torch.Tensor):          # a scale record in device memory (nm_q8_scale)
        _check(lib.mvue_prune_2of4_q8_ds(_ptr(g), T, O, ldg, _dtype_code(g), seed, stream_id, mode, _ptr(scale),
                                         _ptr(vals8), _ptr(meta32), _stream(g)))
    else:
        _check(lib.mvue_prune_2of4_q8(_ptr(g), T, O, ldg, _dtype_code(g), seed, stream_id, mode, float(scale),
                                      _ptr(vals8), _ptr(meta32), _stream(g)))
    return vals8, meta32


def mvue_prune_1of2_q8(g: torch.Tensor, seed: int = 0, stream_id: int = 0, scale=1.0, vals8=None, meta32=None):
    """MVUE 1:2 prune of g[T x O] along T with kept values scaled and rounded stochastically to e5m2.  Returns (vals8, meta32)."""
    lib = load()
    if not g.is_cuda:
        raise ValueError("g must live on the GPU")
    T, O = g.shape
    ldg = _rowmajor(g, "g")
    if vals8 is None or meta32 is None:
        vals8, meta32 = alloc_compressed_q8(T - T % 32, O, g.device)
    if isinstance(scale, torch.Tensor):
        _check(lib.mvue_prune_1of2_q8_ds(_ptr(g), T, O, ldg, _dtype_code(g), seed, stream_id, _ptr(scale),
                                         _ptr(vals8), _ptr(meta32), _stream(g)))
    else:
        _check(lib.mvue_prune_1of2_q8(_ptr(g), T, O, ldg, _dtype_code(g), seed, stream_id, float(scale),
                                      _ptr(vals8), _ptr(meta32), _stream(g)))
    return vals8, meta32


def _prune_q8_transposed(gT: torch.Tensor, vals8, meta32, scale):
    if not gT.is_cuda:
        raise ValueError("gT must live on the GPU")
    O, T = gT.shape
    ldt = _rowmajor(gT, "gT")
    if vals8 is None or meta32 is None:
        vals8, meta32 = alloc_compressed_q8(T - T % 32, O, gT.device)
    rec = scale if isinstance(scale, torch.Tensor) else None          # a scale record in device memory (nm_q8_scale)
    return O, T, ldt, vals8, meta32, (1.0 if rec is not None else float(scale)), rec


def mvue_prune_2of4_q8_t(gT: torch.Tensor, seed: int = 0, stream_id: int = 0, mode: int = 0, scale=1.0, vals8=None, meta32=None):
    """mvue_prune_2of4_q8 for a gradient stored transposed: gT is [O x T], tokens contiguous.  Returns (vals8, meta32), equal to
    mvue_prune_2of4_q8(gT.t().contiguous(), ...) bit for bit."""
    lib = load()
    O, T, ldt, vals8, meta32, s, rec = _prune_q8_transposed(gT, vals8, meta32, scale)
    _check(lib.mvue_prune_2of4_q8_t(_ptr(gT), T, O, ldt, _dtype_code(gT), seed, stream_id, mode, s, _ptr(rec), _ptr(vals8),
                                    _ptr(meta32), _stream(gT)))
    return vals8, meta32


def mvue_prune_1of2_q8_t(gT: torch.Tensor, seed: int = 0, stream_id: int = 0, scale=1.0, vals8=None, meta32=None):
    """mvue_prune_1of2_q8 for a gradient stored transposed (gT [O x T])."""
    lib = load()
    O, T, ldt, vals8, meta32, s, rec = _prune_q8_transposed(gT, vals8, meta32, scale)
    _check(lib.mvue_prune_1of2_q8_t(_ptr(gT), T, O, ldt, _dtype_code(gT), seed, stream_id, s, _ptr(rec), _ptr(vals8), _ptr(meta32),
                                    _stream(gT)))
    return vals8, meta32


def nm_update_gemm_q8_workspace(T: int, O: int, I: int) -> int:
    return int(load().nm_update_gemm_q8_workspace(T, O, I))


def nm_update_gemm_q8(vals8: torch.Tensor, meta32: torch.Tensor, h8: torch.Tensor, dW: Optional[torch.Tensor] = None,
                      alpha: float = 1.0, beta: float = 0.0, workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """dW[O x I] = beta*dW + alpha * decompress(vals8, meta32)^T h8; h8 holds e4m3 codes (uint8 or float8_e4m3fn)."""
    lib = load()
    G, O, _ = vals8.shape
    T, I = h8.shape
    if T != G * 32:
        raise ValueError(f"h8 has {T} rows, the compressed operand covers {G * 32}")
    if h8.element_size() != 1:
        raise TypeError("h8 must be an 8-bit tensor of e4m3 codes")
    ldh = _rowmajor(h8, "h8")
    if dW is None:
        dW = torch.empty((O, I), dtype=torch.float32, device=h8.device)
    lddw = _rowmajor(dW, "dW")
    need = nm_update_gemm_q8_workspace(T, O, I)
    if need and (workspace is None or workspace.numel() * workspace.element_size() < need):
        workspace = torch.empty(need, dtype=torch.uint8, device=h8.device)
    wbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    if isinstance(alpha, tuple):                 # two scale records in device memory: alpha = rec_g[1] * rec_h[1]
        _check(lib.nm_update_gemm_q8_ds(_ptr(vals8), _ptr(meta32), _ptr(h8), ldh, _ptr(dW), lddw, T, O, I, _ptr(alpha[0]),
                                        _ptr(alpha[1]), float(beta), _ptr(workspace), wbytes, _stream(h8)))
    else:
        _check(lib.nm_update_gemm_q8(_ptr(vals8), _ptr(meta32), _ptr(h8), ldh, _ptr(dW), lddw, T, O, I, float(alpha),
                                     float(beta), _ptr(workspace), wbytes, _stream(h8)))
    return dW


def nm_q8_scale(t: torch.Tensor, top: float, rec: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Scale record (device float[4] = s, 1/s, bits of max|t|, 0) of a 2-D tensor: s the largest power of two with
    s * max|t| <= top.  Nothing returns to the host."""
    lib = load()
    R, Cc = t.shape
    if rec is None:
        rec = torch.empty(4, dtype=torch.float32, device=t.device)
    _check(lib.nm_q8_scale(_ptr(t), R, Cc, _rowmajor(t, "t"), _dtype_code(t), float(top), _ptr(rec), _stream(t)))
    return rec


def nm_cast_e4m3(h: torch.Tensor, rec: torch.Tensor, h8: Optional[torch.Tensor] = None) -> torch.Tensor:
    """h8 (uint8 e4m3 codes) = e4m3(h * rec[0]), round to nearest even."""
    lib = load()
    R, Cc = h.shape
    if h8 is None:
        h8 = torch.empty((R, Cc), dtype=torch.uint8, device=h.device)
    _check(lib.nm_cast_e4m3(_ptr(h), R, Cc, _rowmajor(h, "h"), _dtype_code(h), _ptr(rec), _ptr(h8), _rowmajor(h8, "h8"), _stream(h)))
    return h8


def nm_rw_mix_probe(src: torch.Tensor, dst: torch.Tensor, n_blocks: int) -> None:
    """Measurement aid: streams n_blocks * 64 KiB from src and writes n_blocks * 36 KiB to dst (the 16:9 read:write mix of
    the 16-bit prune + compress, contiguous 4 KiB instructions).  src, dst: contiguous device tensors of any dtype."""
    lib = load()
    if src.numel() * src.element_size() < n_blocks * 65536 or dst.numel() * dst.element_size() < n_blocks * 36864:
        raise ValueError("nm_rw_mix_probe: src needs 64 KiB and dst 36 KiB per block")
    _check(lib.nm_rw_mix_probe(_ptr(src), _ptr(dst), n_blocks, _stream(src)))


def nm_update_gemm_shifted(vals: torch.Tensor, meta: torch.Tensor, x_full: torch.Tensor, margin: int, shifts,
                           dW: Optional[torch.Tensor] = None, beta: float = 0.0,
                           workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """dW[O x n*C] = beta*dW + decompress(vals, meta)^T [x shifted by shifts[0] | x shifted by shifts[1] | ...].

    x_full is [margin + T + margin, C] (bf16): row 0 of the grid sits at index ``margin``; the margin rows hold zeros.
    """
    lib = load()
    G, O, _ = vals.shape
    T = G * 16
    if x_full.dim() != 2 or x_full.shape[0] != T + 2 * margin:
        raise ValueError(f"x_full must have {T + 2 * margin} rows (T = {T}, margin = {margin})")
    if max(abs(int(v)) for v in shifts) > margin:
        raise ValueError("a row shift exceeds the margin")
    ldx = _rowmajor(x_full, "x_full")
    Cb = x_full.shape[1]
    n = len(shifts)
    I = n * Cb
    if dW is None:
        dW = torch.empty((O, I), dtype=torch.float32, device=x_full.device)
    lddw = _rowmajor(dW, "dW")
    need = int(lib.nm_update_gemm_shifted_workspace(T, O, Cb, n))
    if need and (workspace is None or workspace.numel() * workspace.element_size() < need):
        workspace = torch.empty(need, dtype=torch.uint8, device=x_full.device)
    wbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    sh = (C.c_int64 * n)(*[int(v) for v in shifts])
    xp = x_full.data_ptr() + margin * ldx * x_full.element_size()
    _check(lib.nm_update_gemm_shifted(_ptr(vals), _ptr(meta), xp, ldx, Cb, sh, n, _ptr(dW), lddw, T, O,
                                      _dtype_code(x_full), float(beta), _ptr(workspace), wbytes, _stream(x_full)))
    return dW


def nm_update_gemm_q8_shifted(vals8: torch.Tensor, meta32: torch.Tensor, x8_full: torch.Tensor, margin: int, shifts,
                              dW: Optional[torch.Tensor] = None, alpha: float = 1.0, beta: float = 0.0,
                              workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """8-bit form of nm_update_gemm_shifted: x8_full is [margin + T + margin, C] e4m3 codes, margin rows zero."""
    lib = load()
    G, O, _ = vals8.shape
    T = G * 32
    if x8_full.dim() != 2 or x8_full.shape[0] != T + 2 * margin or x8_full.element_size() != 1:
        raise ValueError(f"x8_full must be an 8-bit tensor with {T + 2 * margin} rows (T = {T}, margin = {margin})")
    if max(abs(int(v)) for v in shifts) > margin:
        raise ValueError("a row shift exceeds the margin")
    ldx = _rowmajor(x8_full, "x8_full")
    Cb = x8_full.shape[1]
    n = len(shifts)
    if dW is None:
        dW = torch.empty((O, n * Cb), dtype=torch.float32, device=x8_full.device)
    lddw = _rowmajor(dW, "dW")
    need = int(lib.nm_update_gemm_q8_shifted_workspace(T, O, Cb, n))
    if need and (workspace is None or workspace.numel() * workspace.element_size() < need):
        workspace = torch.empty(need, dtype=torch.uint8, device=x8_full.device)
    wbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    sh = (C.c_int64 * n)(*[int(v) for v in shifts])
    xp = x8_full.data_ptr() + margin * ldx
    if isinstance(alpha, tuple):
        _check(lib.nm_update_gemm_q8_shifted_ds(_ptr(vals8), _ptr(meta32), xp, ldx, Cb, sh, n, _ptr(dW), lddw, T, O, _ptr(alpha[0]),
                                                _ptr(alpha[1]), float(beta), _ptr(workspace), wbytes, _stream(x8_full)))
    else:
        _check(lib.nm_update_gemm_q8_shifted(_ptr(vals8), _ptr(meta32), xp, ldx, Cb, sh, n, _ptr(dW), lddw, T, O, float(alpha),
                                             float(beta), _ptr(workspace), wbytes, _stream(x8_full)))
    return dW


# ---- layers: one call per weight gradient

def _image_layout(t: torch.Tensor):
    """(tensor, channels_last) of a 4-D tensor as nm_conv_update takes it: contiguous in one of the two layouts, on a 16-byte
    boundary (a view into a larger buffer may start anywhere); a copy where it is not."""
    cl = not t.is_contiguous() and t.is_contiguous(memory_format=torch.channels_last)
    if t.data_ptr() % 16 or not (cl or t.is_contiguous()):
        t = t.clone(memory_format=torch.channels_last if cl else torch.contiguous_format)
    return t, int(cl)


def nm_conv_update_workspace(N: int, C: int, O: int, H: int, W: int, k: int, q8: bool = False) -> int:
    """Bytes of workspace of nm_conv_update; 0 where it does not take the sizes."""
    return int(load().nm_conv_update_workspace(N, C, O, H, W, k, int(q8)))


def nm_conv_update(gy: torch.Tensor, x: torch.Tensor, k: int, q8: bool = False, mode: int = 0, seed: int = 0, stream_id: int = 0,
                   workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Weight gradient [O, C, k, k] (bf16) of a k x k, stride-1, "same" convolution from gy [N, O, H, W] and x [N, C, H, W] (bf16):
    2:4 prune of gy on the zero-padded channels-last grid and the update GEMM on shifted views, in one library call."""
    lib = load()
    if gy.dtype != torch.bfloat16 or x.dtype != torch.bfloat16 or not (gy.is_cuda and x.is_cuda):
        raise TypeError("nm_conv_update takes bfloat16 tensors on the GPU")
    N, O, H, W = gy.shape
    C = x.shape[1]
    if tuple(x.shape) != (N, C, H, W):
        raise ValueError(f"x {tuple(x.shape)} does not fit gy {tuple(gy.shape)}")
    need = nm_conv_update_workspace(N, C, O, H, W, k, q8)
    gy, g_cl = _image_layout(gy)
    x, x_cl = _image_layout(x)
    if workspace is None or workspace.numel() * workspace.element_size() < need:
        workspace = torch.empty(max(need, 1), dtype=torch.uint8, device=gy.device)
    dW = torch.empty((O, C, k, k), dtype=torch.bfloat16, device=gy.device)
    _check(lib.nm_conv_update(_ptr(gy), g_cl, _ptr(x), x_cl, N, C, O, H, W, k, int(q8), mode, seed, stream_id, _ptr(dW), _ptr(workspace),
                              workspace.numel() * workspace.element_size(), _stream(gy)))
    return dW


def _rows_of(t: torch.Tensor):
    """(tensor, row stride) of a 2-D bf16 tensor whose rows start on 16-byte boundaries; a copy where they do not."""
    if t.stride(1) != 1 or t.stride(0) < t.shape[1] or t.stride(0) % 8 or t.stride(0) > 1 << 21 or t.data_ptr() % 16:
        t = t.clone(memory_format=torch.contiguous_format)
    return t, t.stride(0) if t.shape[0] > 1 else t.shape[1]


def nm_linear_update_workspace(T: int, O: int, I: int, q8: bool = False, bias: bool = False) -> int:
    """Bytes of workspace of nm_linear_update; 0 where it does not take the sizes."""
    return int(load().nm_linear_update_workspace(T, O, I, int(q8), int(bias)))


def nm_linear_update(g: torch.Tensor, h: torch.Tensor, nm: str = "2:4", mode: int = 0, q8: bool = False, seed: int = 0, stream_id: int = 0,
                     act: Optional[torch.Tensor] = None, bias: bool = False):
    """(dW [O x I], db [O] or None, g_out or None) of a linear layer, bf16, from its gradient g [T x O] and input h [T x I], in one
    library call.  act: the output of a ReLU behind the layer; the gradient is then g * [act > 0], returned as g_out."""
    lib = load()
    r = _native_result(_native.linear_update(g, h, 2 if nm == "1:2" else 4, 0 if nm == "1:2" else mode, q8, seed, stream_id, act, bias))
    if r is not None:
        return r
    if any(t.dtype != torch.bfloat16 or not t.is_cuda or t.dim() != 2 for t in ((g, h) if act is None else (g, h, act))):
        raise TypeError("nm_linear_update takes 2-D bfloat16 tensors on the GPU")
    (T, O), I = g.shape, h.shape[1]
    if h.shape[0] != T or (act is not None and act.shape != g.shape):
        raise ValueError(f"g {tuple(g.shape)}, h {tuple(h.shape)} and act do not fit")
    need = lib.nm_linear_update_workspace(T, O, I, q8, bias)
    g, ldg = _rows_of(g)
    h, ldh = _rows_of(h)
    act, lda = _rows_of(act) if act is not None else (None, 0)
    new = lambda *shape: torch.empty(shape, dtype=torch.bfloat16, device=g.device)          # noqa: E731
    dW, db, g_out = new(O, I), new(O) if bias else None, new(T, O) if act is not None else None
    workspace = torch.empty(max(need, 1), dtype=torch.uint8, device=g.device)
    _check(lib.nm_linear_update(_ptr(g), ldg, _ptr(act), lda, _ptr(h), ldh, T, O, I, 2 if nm == "1:2" else 4, 0 if nm == "1:2" else mode, q8,
                                seed, stream_id, _ptr(g_out), O, _ptr(dW), _ptr(db), _ptr(workspace), need, _stream(g)))
    return dW, db, g_out


def nm_linear_forward(x: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor] = None, relu: bool = False) -> torch.Tensor:
    """y [T x O] = x [T x I] weight^T + bias (bf16), with the ReLU behind it where asked, in one kernel."""
    if any(t.dtype != torch.bfloat16 or not t.is_cuda for t in ((x, weight) if bias is None else (x, weight, bias))) or x.dim() != 2:
        raise TypeError("nm_linear_forward takes bfloat16 tensors on the GPU, x with two dimensions")
    (O, I), T = weight.shape, x.shape[0]
    if x.shape[1] != I or (bias is not None and tuple(bias.shape) != (O,)) or not weight.is_contiguous() or (bias is not None and not bias.is_contiguous()):
        raise ValueError(f"x {tuple(x.shape)}, weight {tuple(weight.shape)} and bias do not fit, or the weight is not contiguous")
    x, ldx = _rows_of(x)
    y = torch.empty((T, O), dtype=torch.bfloat16, device=x.device)
    _check(load().nm_linear_forward(_ptr(x), ldx, _ptr(weight), _ptr(bias), T, O, I, relu, _ptr(y), _stream(x)))
    return y


def nm_linear_input_grad(g: torch.Tensor, weight: torch.Tensor) -> torch.Tensor:
    """dx [T x I] = g [T x O] weight (bf16)."""
    if g.dtype != torch.bfloat16 or weight.dtype != torch.bfloat16 or not (g.is_cuda and weight.is_cuda) or g.dim() != 2:
        raise TypeError("nm_linear_input_grad takes bfloat16 tensors on the GPU, g with two dimensions")
    (O, I), T = weight.shape, g.shape[0]
    if g.shape[1] != O or not weight.is_contiguous():
        raise ValueError(f"g {tuple(g.shape)} and weight {tuple(weight.shape)} do not fit, or the weight is not contiguous")
    g, ldg = _rows_of(g)
    dx = torch.empty((T, I), dtype=torch.bfloat16, device=g.device)
    _check(load().nm_linear_input_grad(_ptr(g), ldg, _ptr(weight), T, O, I, _ptr(dx), _stream(g)))
    return dx


def own_linear_forward(x: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor] = None, relu: bool = False) -> Optional[torch.Tensor]:
    """nm_linear_forward over the last dimension of x where that is the faster way and can take the place of the framework's operators (csrc/nm_torch.cpp
    says when); None otherwise."""
    if not x.is_cuda:
        return None
    load()
    return _native_result(_native.linear_forward(x, weight, bias, relu))


def own_linear_input_grad(g: torch.Tensor, weight: torch.Tensor) -> Optional[torch.Tensor]:
    """The same of nm_linear_input_grad; None where gradients are recorded, too."""
    if not g.is_cuda:
        return None
    load()
    return _native_result(_native.linear_input_grad(g, weight))


# ---- products in 8-bit integers

def _quant_i8(x: torch.Tensor, columns: bool):
    lib = load()
    r = _native_result(_native.quant_i8(x, columns))
    if r is not None:
        return r
    if not x.is_cuda or x.dim() != 2:
        raise ValueError("x is a 2-D tensor on the GPU")
    dt = _dtype_code(x)
    x = _unit_columns(x)
    R, Cc = x.shape
    rows, cols = (Cc, R) if columns else (R, Cc)
    q = torch.empty((rows, max(-(-cols // 128) * 128, 128)), dtype=torch.int8, device=x.device)
    scale = torch.empty(rows, dtype=torch.float32, device=x.device)
    with torch.cuda.device(x.device):
        if columns:
            need = int(lib.nm_quant_i8_t_workspace(R, Cc))
            ws = torch.empty(need, dtype=torch.uint8, device=x.device)
            _check(lib.nm_quant_i8_t(_ptr(x), R, Cc, _rowmajor(x, "x"), dt, _ptr(q), q.shape[1], _ptr(scale), _ptr(ws), need, _stream(x)))
        else:
            _check(lib.nm_quant_i8(_ptr(x), R, Cc, _rowmajor(x, "x"), dt, _ptr(q), q.shape[1], _ptr(scale), _stream(x)))
    return q[:, :cols], scale


def nm_quant_i8(x: torch.Tensor) -> Tuple[torch.Tensor, torch.Tensor]:
    """(codes int8 [R x C], scales [R]) of the rows of x: codes = round(x * (127 * (1 / max|x|))), scale = max|x| / 127.  The codes' rows are laid out a
    multiple of 128 bytes apart with zeros behind them."""
    return _quant_i8(x, False)


def nm_quant_i8_t(x: torch.Tensor) -> Tuple[torch.Tensor, torch.Tensor]:
    """nm_quant_i8(x.t()): (codes int8 [C x R], scales [C]) of the columns of x."""
    return _quant_i8(x, True)


def _codes(q: torch.Tensor, scale: torch.Tensor, what: str, width: int, device) -> Tuple[torch.Tensor, int]:
    """(codes, row stride) as the products read them; a copy where the rows do not start on 16-byte boundaries or end with the memory."""
    if q.dtype != torch.int8 or scale.dtype != torch.float32:
        raise TypeError(f"{what} is int8 codes and float32 scales, got {q.dtype} and {scale.dtype}")
    if q.dim() != 2 or q.shape[1] != width or tuple(scale.shape) != (q.shape[0],) or q.device != device or scale.device != device:
        raise ValueError(f"{what}: codes {tuple(q.shape)} and scales {tuple(scale.shape)} do not fit a width of {width}, or live elsewhere")
    wide = -(-width // 16) * 16
    ld = q.stride(0) if q.shape[0] > 1 else wide
    end = q.storage_offset() + (q.shape[0] - 1) * ld + wide
    if q.stride(1) != 1 or ld < wide or ld % 16 or q.data_ptr() % 16 or end > q.untyped_storage().nbytes():
        p = torch.zeros((q.shape[0], wide), dtype=torch.int8, device=device)
        p[:, :width] = q
        return p, wide
    return q, ld


def _i8_result(x_rows: int, wq: torch.Tensor, bias: Optional[torch.Tensor], dtype: torch.dtype, device):
    O, I = wq.shape
    if I < 1:
        raise ValueError("the reduction axis is empty")
    if bias is not None and (tuple(bias.shape) != (O,) or bias.device != device):
        raise ValueError(f"bias {tuple(bias.shape)} on {bias.device} for {O} outputs on {device}")
    _bf16_or_not(dtype)
    return torch.empty((x_rows, O), dtype=dtype, device=device), None if bias is None else bias.contiguous()


def nm_gemm_i8(xq: torch.Tensor, xs: torch.Tensor, wq: torch.Tensor, ws: torch.Tensor, bias: Optional[torch.Tensor] = None, relu: bool = False,
               out_dtype: torch.dtype = torch.bfloat16) -> torch.Tensor:
    """y [T x O] = (xq [T x I] wq [O x I]^T) * xs[:, None] * ws + bias, with the ReLU behind it where asked: 8-bit integer codes with a scale for each
    row, 32-bit integer sums."""
    lib = load()
    if not xq.is_cuda:
        raise ValueError("nm_gemm_i8 takes tensors on the GPU")
    if wq.dim() != 2:
        raise ValueError(f"wq is a matrix, got {tuple(wq.shape)}")
    (O, I), device = wq.shape, xq.device
    y, bias = _i8_result(xq.shape[0], wq, bias, out_dtype, device)
    xq, ldx = _codes(xq, xs, "x", I, device)
    wq, ldw = _codes(wq, ws, "w", I, device)
    xs, ws = xs.contiguous(), ws.contiguous()
    with torch.cuda.device(device):
        _check(lib.nm_gemm_i8(_ptr(xq), ldx, _ptr(xs), _ptr(wq), ldw, _ptr(ws), _ptr(bias), 0 if bias is None else _dtype_code(bias), xq.shape[0], O, I, int(relu), _ptr(y), max(O, 1),
                              _dtype_code(y), _stream(y)))
    return y


def nm_linear_i8(x: torch.Tensor, wq: torch.Tensor, ws: torch.Tensor, bias: Optional[torch.Tensor] = None, relu: bool = False,
                 out_dtype: Optional[torch.dtype] = None) -> torch.Tensor:
    """A linear layer over the last dimension of x (float32 or bfloat16) whose weights are 8-bit integers wq [O x I] with a scale ws [O] for each output: x is
    rounded to 8-bit integers with a scale for each token, nm_gemm_i8 follows.  out_dtype: x's by default."""
    lib = load()
    r = _native_result(_native.linear_i8(x, wq, ws, bias, relu, _bf16_or_not(out_dtype)))
    if r is not None:
        return r
    if not x.is_cuda or x.dim() < 1:
        raise ValueError("nm_linear_i8 takes tensors on the GPU")
    if wq.dim() != 2 or x.shape[-1] != wq.shape[1]:
        raise ValueError(f"x {tuple(x.shape)} and wq {tuple(wq.shape)} do not fit")
    (O, I), device, dt = wq.shape, x.device, _dtype_code(x)
    shape, x = x.shape, _unit_columns(x.reshape(-1, I)) if I else x
    y, bias = _i8_result(x.shape[0], wq, bias, out_dtype or x.dtype, device)
    wq, ldw = _codes(wq, ws, "w", I, device)
    ws = ws.contiguous()
    need = int(lib.nm_linear_i8_workspace(x.shape[0], I))
    work = torch.empty(need, dtype=torch.uint8, device=device)
    with torch.cuda.device(device):
        _check(lib.nm_linear_i8(_ptr(x), _rowmajor(x, "x"), dt, _ptr(wq), ldw, _ptr(ws), _ptr(bias), 0 if bias is None else _dtype_code(bias), x.shape[0], O, I, int(relu), _ptr(y),
                                max(O, 1), _dtype_code(y), _ptr(work), need, _stream(x)))
    return y.reshape(*shape[:-1], O)


# ---- embedding

def _ids(ids: torch.Tensor, device) -> Tuple[torch.Tensor, int]:
    if ids.dtype not in (torch.int32, torch.int64):
        raise TypeError(f"ids are int32 or int64, got {ids.dtype}")
    if ids.device != device:
        raise ValueError("ids live on the GPU of the table or gradient")
    return ids.contiguous(), 64 if ids.dtype == torch.int64 else 32


def _unit_columns(t: torch.Tensor) -> torch.Tensor:
    """A matrix as the kernels read it; a copy where columns are apart or rows share memory (autograd's gradient of a sum over rows has row stride 0)."""
    return t if (t.stride(1) == 1 or t.shape[1] == 1) and (t.stride(0) >= t.shape[1] or t.shape[0] <= 1) else t.contiguous()


def _bf16_or_not(dtype: Optional[torch.dtype]):
    if dtype not in (None, torch.float32, torch.bfloat16):
        raise TypeError(f"results are float32 or bfloat16, got {dtype}")
    return None if dtype is None else dtype == torch.bfloat16


def nm_embed(table: torch.Tensor, ids: torch.Tensor, scale: float = 1.0, out_dtype: Optional[torch.dtype] = None) -> torch.Tensor:
    """scale * table[ids], rounded once to out_dtype (the table's by default).  table [V x D] float32 or bfloat16, ids int32 or int64 of any shape;
    a token outside the table gives a row of NaN."""
    lib = load()
    r = _native_result(_native.embed(table, ids, float(scale), _bf16_or_not(out_dtype)))
    if r is not None:
        return r
    if not table.is_cuda or table.dim() != 2:
        raise ValueError("the table is a 2-D tensor on the GPU")
    dt = _dtype_code(table)
    ids, bits = _ids(ids, table.device)
    table = _unit_columns(table)
    (V, D), N = table.shape, ids.numel()
    out = torch.empty((*ids.shape, D), dtype=out_dtype or table.dtype, device=table.device)
    with torch.cuda.device(table.device):
        _check(lib.nm_embed(_ptr(table), V, D, _rowmajor(table, "table"), dt, _ptr(ids), bits, N, float(scale), _ptr(out), D, _dtype_code(out), _stream(table)))
    return out


def nm_embed_grad(g: torch.Tensor, ids: torch.Tensor, vocab: int, scale: float = 1.0, padding_idx: Optional[int] = None, out_dtype: Optional[torch.dtype] = None,
                  out: Optional[torch.Tensor] = None, accumulate: bool = False) -> torch.Tensor:
    """Gradient [vocab x D] of an embedding table: row v is scale times the sum of the rows of g (ids.shape + (D,), float32 or bfloat16) whose token is v,
    in binary32 and in a fixed order.  Tokens outside the table and padding_idx count for nothing.  out, accumulate: write, or add, to a given tensor."""
    lib = load()
    padding = -1 if padding_idx is None else int(padding_idx)
    if accumulate and out is None:
        raise ValueError("accumulate adds to a given tensor: pass out")
    if out is None:
        r = _native_result(_native.embed_grad(g, ids, vocab, float(scale), padding, _bf16_or_not(out_dtype)))
        if r is not None:
            return r
    if not g.is_cuda or tuple(g.shape[:-1]) != tuple(ids.shape) or g.dim() < 1:
        raise ValueError(f"a gradient {tuple(g.shape)} on {g.device} of ids {tuple(ids.shape)}")
    dt = _dtype_code(g)
    ids, bits = _ids(ids, g.device)
    D, N = g.shape[-1], ids.numel()
    g = _unit_columns(g.reshape(N, D))
    given = out
    if out is None:
        out = torch.empty((vocab, D), dtype=out_dtype or g.dtype, device=g.device)
    elif tuple(out.shape) != (vocab, D) or out.device != g.device or (out_dtype is not None and out.dtype != out_dtype):
        raise ValueError(f"out has to be a {vocab} x {D} tensor of the wanted type on the gradient's device")
    need = int(lib.nm_embed_grad_workspace(N, vocab, D))
    ws = torch.empty(need, dtype=torch.uint8, device=g.device)
    with torch.cuda.device(g.device):
        _check(lib.nm_embed_grad(_ptr(g), _rowmajor(g, "g"), dt, _ptr(ids), bits, N, vocab, D, float(scale), padding, int(accumulate), _ptr(out), _rowmajor(out, "out"),
                                 _dtype_code(out), _ptr(ws), need, _stream(g)))
    if given is not None and not given.is_inference():
        torch.autograd.graph.increment_version([given])                      # (a graph that has saved it then says so)
    return out


# ---- between a block's linear layers: layer norm, rotary positions, attention

def _norm_weights(weight: Optional[torch.Tensor], bias: Optional[torch.Tensor], x: torch.Tensor):
    width = x.shape[-1]
    for t in (weight, bias):
        if t is not None and (tuple(t.shape) != (width,) or t.device != x.device):
            raise ValueError(f"weight and bias of rows of {width} have one element for each, on the tensor's device")
    if weight is not None and bias is not None and weight.dtype != bias.dtype:
        raise TypeError("weight and bias are of one type")
    known = weight if weight is not None else bias
    return None if weight is None else weight.contiguous(), None if bias is None else bias.contiguous(), NM_F32 if known is None else _dtype_code(known)


def nm_layer_norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None, eps: float = 1e-5, want_stats: bool = False):
    """(x - mean) / sqrt(variance + eps) * weight + bias over the last dimension (1 to 32768), of x's type; x, weight and bias float32 or bfloat16.
    want_stats: (y, mean, rstd), the last two float32 of x's shape without its last dimension, as nm_layer_norm_grad reads them."""
    lib = load()
    r = _native_result(_native.layer_norm(x, weight, bias, float(eps), want_stats))
    if r is not None:
        return r
    if not x.is_cuda or x.dim() < 1:
        raise ValueError("x is a tensor on the GPU with at least one dimension")
    dt = _dtype_code(x)
    w, b, wt = _norm_weights(weight, bias, x)
    shape, C = x.shape, x.shape[-1]
    x = _unit_columns(x.reshape(-1, C) if C else x.reshape(0, C))
    R = x.shape[0]
    y = torch.empty(shape, dtype=x.dtype, device=x.device)
    mean, rstd = (torch.empty(shape[:-1], dtype=torch.float32, device=x.device) for _ in range(2)) if want_stats else (None, None)
    with torch.cuda.device(x.device):
        _check(lib.nm_layer_norm(_ptr(x), _rowmajor(x, "x"), dt, _ptr(w), _ptr(b), wt, R, C, float(eps), _ptr(y), C, _ptr(mean), _ptr(rstd), _stream(x)))
    return (y, mean, rstd) if want_stats else y


def nm_layer_norm_grad(g: torch.Tensor, x: torch.Tensor, weight: Optional[torch.Tensor], mean: torch.Tensor, rstd: torch.Tensor, want_weight: bool = True,
                       want_bias: bool = True):
    """(dx, dweight, dbias) of nm_layer_norm from the gradient g of its result, its x and weight (None: ones), and the mean and rstd that it left.  dx is of
    x's type, dweight and dbias of weight's (float32 without one); None where not wanted."""
    lib = load()
    if want_weight and want_bias:
        r = _native_result(_native.layer_norm_grad(g, x, weight, mean, rstd))
        if r is not None:
            return r
    if not x.is_cuda or x.dim() < 1 or g.shape != x.shape or g.dtype != x.dtype or g.device != x.device:
        raise ValueError("x and g are tensors of one shape and type on one GPU")
    dt = _dtype_code(x)
    w, _, wt = _norm_weights(weight, None, x)
    for t in (mean, rstd):
        if t.dtype != torch.float32 or t.shape != x.shape[:-1] or t.device != x.device:
            raise ValueError("mean and rstd are float32, one for each row, on the tensor's device")
    mean, rstd = mean.contiguous(), rstd.contiguous()
    shape, C = x.shape, x.shape[-1]
    x, g = (_unit_columns(t.reshape(-1, C) if C else t.reshape(0, C)) for t in (x, g))
    R = x.shape[0]
    dx = torch.empty(shape, dtype=x.dtype, device=x.device)
    kind = torch.float32 if weight is None else weight.dtype
    dw = torch.empty(C, dtype=kind, device=x.device) if want_weight else None
    db = torch.empty(C, dtype=kind, device=x.device) if want_bias else None
    need = int(lib.nm_layer_norm_grad_workspace(R, C)) if want_weight or want_bias else 0
    ws = torch.empty(need, dtype=torch.uint8, device=x.device)
    with torch.cuda.device(x.device):
        _check(lib.nm_layer_norm_grad(_ptr(g), _rowmajor(g, "g"), _ptr(x), _rowmajor(x, "x"), dt, _ptr(w), wt, _ptr(mean), _ptr(rstd), R, C, _ptr(dx), C, _ptr(dw), _ptr(db),
                                      _ptr(ws), need, _stream(x)))
    return dx, dw, db


def rotary_freqs(width: int, base: float = 10000.0, scaling: Optional[str] = None, factor: float = 1.0, original_length: int = 0, slow: float = 1.0, fast: float = 32.0,
                 device=None) -> torch.Tensor:
    """Radians to a position of `width` turned elements, for nm_rotary: float64 [width / 2], base ** (-2 j / width).  For contexts `factor` times as long as the
    ones trained on, scaling is "linear": all divided by factor; "base": the base raised so that the slowest pair is divided by factor and the fastest kept;
    "parts": pairs that turn more than `fast` times over original_length positions kept, those that turn less than `slow` times divided, a line between."""
    if width < 2 or width % 2 or not base > 0 or not factor > 0:
        raise ValueError("width is an even number from 2 on, base and factor are positive")
    if scaling == "base" and width > 2:
        base = base * factor ** (width / (width - 2))
    with torch.inference_mode(False):                                       # (constants that a later training step may save as well)
        f = _rotary_freqs_on_host(width, base, scaling, factor, original_length, slow, fast)
        return f.to(torch.get_default_device() if device is None else device)


def _rotary_freqs_on_host(width, base, scaling, factor, original_length, slow, fast) -> torch.Tensor:
    f = base ** (-torch.arange(0, width, 2, dtype=torch.float64, device="cpu") / width)
    if scaling == "linear":
        f = f / factor
    elif scaling == "parts":
        if not (original_length > 0 and fast > slow):
            raise ValueError('"parts" needs original_length, and fast > slow')
        turns = f * original_length / (2 * math.pi)
        keep = ((turns - slow) / (fast - slow)).clamp(0, 1)
        f = f * keep + f / factor * (1 - keep)
    elif scaling not in (None, "base"):
        raise ValueError(f'scaling is None, "linear", "base" or "parts", got {scaling!r}')
    return f


def _heads(t: torch.Tensor) -> _Heads:
    return _Heads(t.data_ptr(), *t.stride()[:3])


def nm_rotary(x: torch.Tensor, freqs: torch.Tensor, positions: Optional[torch.Tensor] = None, interleaved: bool = False, scale: float = 1.0, inverse: bool = False,
              out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """x [batch x length x heads x D] (float32 or bfloat16, D up to 1024) with the pairs of each head's first 2 * len(freqs) elements turned by position times
    frequency and multiplied by scale; what lies behind them stays.  freqs: float64 on the GPU (rotary_freqs); positions: int32 or int64, [length] or
    [batch x length], 0 .. length - 1 without.  Pairs: neighbours where interleaved, otherwise half the turned elements apart.  inverse: turned back, which is the
    gradient with respect to x of the call without it.  out: a tensor for the result, x itself among them."""
    lib = load()
    if out is None:
        r = _native_result(_native.rotary(x, freqs, positions, interleaved, float(scale), inverse))
        if r is not None:
            return r
    if not x.is_cuda or x.dim() != 4:
        raise ValueError("x is a 4-D tensor on the GPU: batch, length, heads, elements")
    dt = _dtype_code(x)
    B, T, H, D = x.shape
    if freqs.dtype != torch.float64 or freqs.dim() != 1 or freqs.device != x.device:
        raise TypeError("freqs is a float64 vector on the tensor's device")
    if x.stride(3) != 1 and D > 1:
        if out is x:
            raise ValueError("elements of a head lie side by side in a tensor that is turned in place")
        x = x.contiguous()
    bits, pos_stride = 32, 0
    if positions is not None:
        if positions.dtype not in (torch.int32, torch.int64):
            raise TypeError(f"positions are int32 or int64, got {positions.dtype}")
        if positions.device != x.device or tuple(positions.shape) not in ((T,), (B, T)):
            raise ValueError(f"positions of {B} x {T} tokens have shape [{T}] or [{B}, {T}], on the tensor's device")
        bits = 64 if positions.dtype == torch.int64 else 32
        positions = positions.contiguous()
        pos_stride = T if positions.dim() == 2 else 0
    y = torch.empty((B, T, H, D), dtype=x.dtype, device=x.device) if out is None else out
    if y.shape != x.shape or y.dtype != x.dtype or y.device != x.device or (D > 1 and y.stride(3) != 1):
        raise ValueError("out has x's shape, type and device, and elements of a head side by side")
    freqs = freqs.contiguous()
    with torch.cuda.device(x.device):
        _check(lib.nm_rotary(_heads(x), _heads(y), dt, B, T, H, D, 2 * freqs.numel(), _ptr(freqs), _ptr(positions), bits, pos_stride, int(interleaved), float(scale), int(inverse),
                             _stream(x)))
    if out is not None and not out.is_inference():
        torch.autograd.graph.increment_version([out])
    return y


def _attention_input(t: torch.Tensor, what: str, like: Optional[torch.Tensor] = None) -> torch.Tensor:
    """A tensor of heads as the kernels read it: a copy where elements are apart or rows off a 16-byte boundary."""
    if not t.is_cuda or t.dim() != 4:
        raise ValueError(f"{what} is a 4-D tensor on the GPU: batch, length, heads, elements")
    if like is not None and (t.dtype != like.dtype or t.device != like.device):
        raise TypeError(f"{what} is of another type or on another device than q")
    size = t.element_size()
    fits = t.stride(3) == 1 and t.data_ptr() % 16 == 0 and all(n < 2 or s * size % 16 == 0 for n, s in zip(t.shape, t.stride()[:3]))
    return t if fits else t.clone(memory_format=torch.contiguous_format)


def _attention_sizes(q, k, v):
    B, Tq, Hq, D = q.shape
    if k.shape != v.shape or k.shape[0] != B or k.shape[3] != D:
        raise ValueError(f"q {tuple(q.shape)}, k {tuple(k.shape)} and v {tuple(v.shape)}: k and v are alike, with q's batch and elements")
    return B, Tq, k.shape[1], Hq, k.shape[2], D


def _lse_planes(q: torch.Tensor) -> int:
    return 1 + q.shape[-1] // 2 if q.dtype == torch.bfloat16 else 1


def _rest(lse: Optional[torch.Tensor]):
    """the address of what rounding took from o, behind lse's first plane"""
    return lse.data_ptr() + 4 * lse[0].numel() if lse is not None and lse.shape[0] > 1 else None


def _scale_of(scale: Optional[float], q: torch.Tensor) -> float:
    return float(scale) if scale is not None else q.shape[-1] ** -0.5 if q.dim() and q.shape[-1] else 1.0


def _lengths_of(lens: Optional[torch.Tensor], B: int, device) -> Optional[torch.Tensor]:
    if lens is None:
        return None
    if lens.dtype not in (torch.int32, torch.int64) or tuple(lens.shape) != (B,) or lens.device != device:
        raise ValueError(f"lengths of {B} sequences are int32 or int64 [{B}] on the tensors' device")
    return lens.clamp(-1, 0x7fffffff).to(torch.int32) if lens.dtype == torch.int64 else lens.contiguous()


def nm_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, causal: bool = False, scale: Optional[float] = None, q_lens: Optional[torch.Tensor] = None,
                 k_lens: Optional[torch.Tensor] = None, want_lse: bool = False):
    """softmax(scale q k^T) v for each head.  q [batch x queries x heads x D], k and v [batch x keys x kv_heads x D], float32 or bfloat16 of one type, D a multiple of
    8 up to 128; heads / kv_heads heads of q in a row share one of k and v.  scale: D ** -0.5 by default.  causal: query i of n sees the keys up to i + m - n of m, the last
    query the last key, so that one query over a cache of keys sees all of them.  q_lens, k_lens (int32 or int64 [batch], on the GPU): the tokens of each sequence, from
    the front; what lies behind counts for nothing, and the result is zero there, as for a query that sees no key.  What a causal query does not see of its own sequence has to be finite.
    want_lse: (o, lse).  lse[0] is float32 [batch x heads x queries], the logarithm of the sum of exponentials; for bfloat16 lse has D / 2 planes more, whose bits are
    what rounding took from o: element [1 + w, b, h, i] as two bfloat16, those of o[b, i, h, 2 w] and o[b, i, h, 2 w + 1].  nm_attention_grad reads all of it; cut along sequences,
    heads or queries, as the other tensors are, it stays what it is."""
    lib = load()
    scale = _scale_of(scale, q)
    r = _native_result(_native.attention(q, k, v, causal, scale, q_lens, k_lens, want_lse))
    if r is not None:
        return r
    q = _attention_input(q, "q")
    k, v = _attention_input(k, "k", q), _attention_input(v, "v", q)
    dt = _dtype_code(q)
    sizes = B, Tq, Tk, Hq, Hk, D = _attention_sizes(q, k, v)
    ql, kl = _lengths_of(q_lens, B, q.device), _lengths_of(k_lens, B, q.device)
    o = torch.empty((B, Tq, Hq, D), dtype=q.dtype, device=q.device)
    lse = torch.empty((_lse_planes(q), B, Hq, Tq), dtype=torch.float32, device=q.device) if want_lse else None
    need = int(lib.nm_attention_workspace(*sizes, dt))
    ws = torch.empty(need, dtype=torch.uint8, device=q.device) if need else None
    with torch.cuda.device(q.device):
        _check(lib.nm_attention(_heads(q), _heads(k), _heads(v), _heads(o), _ptr(lse), _rest(lse), *sizes, dt, int(causal), scale, _ptr(ql), _ptr(kl),
                                _ptr(ws), need, _stream(q)))
    return (o, lse) if want_lse else o


def nm_attention_grad(g: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, o: torch.Tensor, lse: torch.Tensor, causal: bool = False,
                      scale: Optional[float] = None, q_lens: Optional[torch.Tensor] = None, k_lens: Optional[torch.Tensor] = None, out=None):
    """(dq, dk, dv) of nm_attention from the gradient g of its result o; the other arguments as they were given to it, and the lse that it left.  The probabilities
    are computed again.  lse[:1] alone will do; gradients of queries that look at few keys are then less exact in bfloat16.  The same call gives the same bits.  out: three tensors for the results, of q's, k's and v's shapes, parts of one tensor among them."""
    lib = load()
    scale = _scale_of(scale, q)
    if out is None:
        r = _native_result(_native.attention_grad(g, q, k, v, o, lse, causal, scale, q_lens, k_lens))
        if r is not None:
            return r
    q = _attention_input(q, "q")
    k, v, g, o = (_attention_input(t, what, q) for t, what in ((k, "k"), (v, "v"), (g, "g"), (o, "o")))
    dt = _dtype_code(q)
    sizes = B, Tq, Tk, Hq, Hk, D = _attention_sizes(q, k, v)
    if g.shape != q.shape or o.shape != q.shape:
        raise ValueError("g and o have q's shape")
    if lse.dtype != torch.float32 or lse.dim() != 4 or lse.shape[0] not in (1, _lse_planes(q)) or tuple(lse.shape[1:]) != (B, Hq, Tq) or lse.device != q.device:
        raise ValueError(f"lse is float32 [{_lse_planes(q)}, {B}, {Hq}, {Tq}] on the tensors' device, as nm_attention left it")
    lse = lse.contiguous()
    ql, kl = _lengths_of(q_lens, B, q.device), _lengths_of(k_lens, B, q.device)
    if out is None:
        dq, dk, dv = (torch.empty(t.shape, dtype=q.dtype, device=q.device) for t in (q, k, v))
    else:
        dq, dk, dv = out
        for d, t in ((dq, q), (dk, k), (dv, v)):
            if d.shape != t.shape or d.dtype != t.dtype or d.device != t.device or d.stride(3) != 1:
                raise ValueError("out: tensors of q's, k's and v's shapes, type and device, elements of a head side by side")
    need = int(lib.nm_attention_grad_workspace(*sizes, dt))
    ws = torch.empty(need, dtype=torch.uint8, device=q.device)
    with torch.cuda.device(q.device):
        _check(lib.nm_attention_grad(_heads(g), _heads(q), _heads(k), _heads(v), _heads(o), _ptr(lse), _rest(lse), *sizes, dt, int(causal), scale,
                                     _ptr(ql), _ptr(kl), _heads(dq), _heads(dk), _heads(dv), _ptr(ws), need, _stream(q)))
    if out is not None:
        torch.autograd.graph.increment_version([t for t in out if not t.is_inference()])
    return dq, dk, dv


# ---- the optimizer's step

class _AdamwTensor(C.Structure):
    _fields_ = [("param", C.c_void_p), ("grad", C.c_void_p), ("m", C.c_void_p), ("v", C.c_void_p), ("m_scale", C.c_void_p),
                ("v_scale", C.c_void_p), ("master", C.c_void_p), ("n", C.c_int64), ("number", C.c_uint32)]


STATE_BLOCK = 256         # elements of an 8-bit state that share a scale


def alloc_adamw_state(param: torch.Tensor, q8: bool = False):
    """Zero state of nm_adamw for one of m and v: a binary32 tensor, or (q8) a pair of e4m3 codes and scales."""
    if not q8:
        return torch.zeros_like(param, dtype=torch.float32, memory_format=torch.preserve_format)
    codes = torch.empty_like(param, dtype=torch.float8_e4m3fn, memory_format=torch.preserve_format)
    codes.view(torch.uint8).zero_()
    return codes, torch.ones(-(-param.numel() // STATE_BLOCK), dtype=torch.float32, device=param.device)


def _adamw_state(what: str, state, p: torch.Tensor):
    """(values, scale or None) of a state that fits its parameter."""
    if isinstance(state, torch.Tensor):
        values, scale, want = state, None, torch.float32
    else:
        (values, scale), want = state, torch.float8_e4m3fn
        if scale.dtype != torch.float32 or not scale.is_contiguous() or scale.numel() != -(-p.numel() // STATE_BLOCK) or scale.device != p.device:
            raise ValueError(f"{what}: scales are contiguous float32, one for every {STATE_BLOCK} elements")
    if values.dtype != want:
        raise TypeError(f"{what} is float32, or a pair of float8_e4m3fn codes and float32 scales; got {values.dtype}")
    if values.shape != p.shape or values.stride() != p.stride() or values.device != p.device:
        raise ValueError(f"{what} has another shape, layout or device than its parameter")
    return values, scale


def nm_adamw(params, grads, exp_avgs, exp_avg_sqs, step: int, lr: float = 1e-3, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay: float = 1e-2,
             masters=None, grad_scale=1.0, seed: int = 0, numbers=None) -> None:
    """One AdamW step (number `step`, from 1) over lists of tensors, in place; tensors of one set of types share a launch.

    params and grads: float32 or bfloat16.  exp_avgs, exp_avg_sqs: of each tensor a float32 tensor, or for 8-bit states a pair
    (float8_e4m3fn codes, float32 scales) as alloc_adamw_state makes them; that of exp_avg_sqs then stands for its square
    root.  masters: float32 copies of bfloat16 parameters that take the step, None in the place of one without.  grad_scale: a
    factor on the gradients, a number or a float32 tensor of one element on the GPU.  numbers: each tensor's number in the counter of its random words
    (8-bit states), its place in the list by default.  All numbers, `step` and `seed` among them, are arguments of the launch: a graph that captures it
    repeats that step."""
    lib = load()
    params, grads, exp_avgs, exp_avg_sqs = list(params), list(grads), list(exp_avgs), list(exp_avg_sqs)
    masters = None if masters is None else list(masters)
    numbers = None if numbers is None else list(numbers)
    dev_scale = grad_scale if isinstance(grad_scale, torch.Tensor) else None
    args = (step, float(lr), float(betas[0]), float(betas[1]), float(eps), float(weight_decay), 1.0 if dev_scale is not None else float(grad_scale))
    if _native_result(_native.adamw(params, grads, exp_avgs, exp_avg_sqs, masters, numbers, *args, dev_scale, seed)):
        return
    n = len(params)
    if any(len(x) != n for x in (grads, exp_avgs, exp_avg_sqs, masters or params, numbers or params)):
        raise ValueError("nm_adamw takes lists of one length")
    if dev_scale is not None and (not dev_scale.is_cuda or dev_scale.dtype != torch.float32 or dev_scale.numel() != 1):
        raise TypeError("grad_scale is a number or a float32 tensor of one element on the GPU")
    groups, keep = {}, []
    for k, (p, g) in enumerate(zip(params, grads)):
        w = None if masters is None else masters[k]
        if not p.is_cuda or g.device != p.device or (dev_scale is not None and dev_scale.device != p.device):
            raise ValueError("nm_adamw takes tensors on the GPU, a parameter's arrays on one device")
        if g.shape != p.shape:
            raise ValueError(f"gradient {tuple(g.shape)} of a parameter {tuple(p.shape)}")
        if p.numel() and _dense_strides(p) is None:
            raise ValueError("a parameter's memory has gaps or overlaps")
        if g.stride() != p.stride():
            g = torch.empty_strided(p.shape, p.stride(), dtype=g.dtype, device=g.device).copy_(g)
            keep.append(g)
        (m, ms), (v, vs) = _adamw_state("exp_avg", exp_avgs[k], p), _adamw_state("exp_avg_sq", exp_avg_sqs[k], p)
        if (ms is None) != (vs is None):
            raise TypeError("exp_avg and exp_avg_sq are both float32 or both 8 bits")
        if w is not None and (w.dtype != torch.float32 or w.shape != p.shape or w.stride() != p.stride() or w.device != p.device):
            raise ValueError("a master copy is float32 and laid out as its parameter")
        key = (p.device, _dtype_code(p), _dtype_code(g), ms is not None, w is not None)
        groups.setdefault(key, []).append(_AdamwTensor(_ptr(p), _ptr(g), _ptr(m), _ptr(v), _ptr(ms), _ptr(vs), _ptr(w), p.numel(), k if numbers is None else numbers[k]))
    for (device, pt, gt, q8, _), tensors in groups.items():
        with torch.cuda.device(device):
            _check(lib.nm_adamw((_AdamwTensor * len(tensors))(*tensors), len(tensors), pt, gt, int(q8), *args[1:6], step, args[6], _ptr(dev_scale), seed,
                                torch.cuda.current_stream(device).cuda_stream))
    torch.autograd.graph.increment_version([t for t in params + (masters or []) if t is not None and not t.is_inference()])


def _dense_strides(t: torch.Tensor) -> Optional[Tuple[int, ...]]:
    """The strides of a tensor whose elements fill its memory without gaps or overlaps, in any order of dimensions; None of another."""
    need = 1
    for size, stride in sorted((x for x in zip(t.shape, t.stride()) if x[0] != 1), key=lambda x: x[1]):
        if stride != need:
            return None
        need *= size
    return t.stride()
