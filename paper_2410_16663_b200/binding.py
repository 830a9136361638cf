"""ctypes binding of ``libfa.so``: the same entry points as ``include/fa.h``, same names.

This layer only marshals arguments (pointers, sizes, the current CUDA stream); every step of
the attention path runs inside the library's kernels.  There is no fallback: if the library is
missing or fails to load, importing this module raises.
"""
from __future__ import annotations

import ctypes
import math
import os
import struct

import torch

FA_OK = 0
FA_ERR_NULL, FA_ERR_SHAPE, FA_ERR_UNSUPPORTED, FA_ERR_ALIGN = -1, -2, -3, -4
FA_ERR_WORKSPACE, FA_ERR_DEVICE, FA_ERR_CUDA, FA_ERR_TIMEOUT = -5, -6, -7, -8
FA_DTYPE_FP16, FA_DTYPE_BF16, FA_DTYPE_FP32, FA_DTYPE_E4M3 = 0, 1, 2, 3

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libfa.so")
if not os.path.exists(_LIB_PATH):
    raise ImportError(f"{_LIB_PATH} is missing: run `python -m paper_2410_16663_b200.build` "
                      "(the CUDA library is required; there is no fallback path)")
lib = ctypes.CDLL(_LIB_PATH)

_i, _f, _p, _sz = ctypes.c_int, ctypes.c_float, ctypes.c_void_p, ctypes.c_size_t


class fa_params(ctypes.Structure):
    _fields_ = [("q", _p), ("k", _p), ("v", _p), ("o", _p), ("lse", _p),
                ("B", _i), ("Hq", _i), ("Hkv", _i), ("Sq", _i), ("Skv", _i), ("d", _i),
                ("causal", _i), ("scale", _f), ("dtype", _i), ("o_dtype", _i),
                ("q_stride", ctypes.c_int64 * 3), ("k_stride", ctypes.c_int64 * 3),
                ("v_stride", ctypes.c_int64 * 3), ("o_stride", ctypes.c_int64 * 3),
                ("variant", _i)]


_FWD_ARGS = [_p, _p, _p, _p, _p, _i, _i, _i, _i, _i, _i, _i, _f, _p]
lib.fa_forward.restype = _i
lib.fa_forward.argtypes = _FWD_ARGS
lib.fa_forward_bf16.restype = _i
lib.fa_forward_bf16.argtypes = _FWD_ARGS
lib.fa_forward_ex.restype = _i
lib.fa_forward_ex.argtypes = [ctypes.POINTER(fa_params), _p]
lib.fa_forward_fp8.restype = _i
lib.fa_forward_fp8.argtypes = [_p, _p, _p, _p, _p, _i, _i, _i, _i, _i, _i, _i, _f, _f, _f, _f, _i, _p]
lib.fa_forward_proj.restype = _i
lib.fa_forward_proj.argtypes = [_p, _p, _p, _p, _p, _p, _p, _i, _i, _i, _i, _i, _i, _i, _i, _f, _i, _i, _p, _sz, _p]
lib.fa_forward_proj_workspace_bytes.restype = _sz
lib.fa_forward_proj_workspace_bytes.argtypes = [_i, _i]
lib.fa_decode.restype = _i
lib.fa_decode.argtypes = [_p, _p, _p, _p, _p, _p, _i, _i, _i, _i, _i, _f, _p, _sz, _p]
lib.fa_decode_workspace_bytes.restype = _sz
lib.fa_decode_workspace_bytes.argtypes = [_i, _i, _i, _i, _i]
lib.fa_forward_varlen.restype = _i
lib.fa_forward_varlen.argtypes = [_p, _p, _p, _p, _p, _p, _p, _i, _i, _i, _i, _i, _i, _i, _i, _i, _f, _i, _p]
class fa_decode_params(ctypes.Structure):
    _fields_ = [("q", _p), ("k", _p), ("v", _p), ("o", _p), ("lse", _p), ("seqlens_k", _p), ("block_table", _p),
                ("B", _i), ("Sq", _i), ("Hq", _i), ("Hkv", _i), ("Skv_max", _i), ("d", _i), ("dtype", _i),
                ("num_pages", _i), ("page_size", _i), ("max_pages", _i), ("table_stride", _i), ("scale", _f),
                ("workspace", _p), ("workspace_bytes", _sz)]


lib.fa_decode_ex.restype = _i
lib.fa_decode_ex.argtypes = [ctypes.POINTER(fa_decode_params), _p]
class fa_tree_params(ctypes.Structure):
    _fields_ = [("q", _p), ("k", _p), ("v", _p), ("o", _p), ("lse", _p), ("seqlens_k", _p), ("tree_lens", _p), ("mask", _p),
                ("block_table", _p), ("B", _i), ("T", _i), ("Hq", _i), ("Hkv", _i), ("Skv_max", _i), ("d", _i), ("dtype", _i),
                ("num_pages", _i), ("page_size", _i), ("max_pages", _i), ("table_stride", _i), ("variant", _i), ("mask_stride", ctypes.c_int64),
                ("scale", _f), ("workspace", _p), ("workspace_bytes", _sz)]


lib.fa_decode_tree.restype = _i
lib.fa_decode_tree.argtypes = [_p, _p]   # (an fa_tree_params by reference, or its bytes)
_TREE = struct.Struct("@9P12iqfPN")      # fa_tree_params
assert _TREE.size == ctypes.sizeof(fa_tree_params)
class fa_append_params(ctypes.Structure):
    _fields_ = [(name, _p) for name in ("q", "q_out", "k", "v", "k_cache", "v_cache", "turns", "positions", "first_rows", "counts",
                                        "cu_seqlens", "block_table")]
    _fields_ += [(name + "_stride", ctypes.c_int64 * 2) for name in ("q", "q_out", "k", "v", "k_cache", "v_cache")]
    _fields_ += [(name, _i) for name in ("n", "B", "T", "Hq", "Hkv", "d", "dv", "rot_dim", "rot_offset", "interleaved", "dtype",
                                         "cache_dtype", "Skv_max", "num_pages", "page_size", "max_pages", "table_stride")]
    _fields_ += [("factor", _f), ("k_scale", _f), ("v_scale", _f)]


lib.fa_rope.restype = _i
lib.fa_rope.argtypes = [_p] * 4 + [_p] * 6 + [_f] + [_p] * 6   # (sizes as words, see fa_spec_verify)
lib.fa_cache_append.restype = _i
lib.fa_cache_append.argtypes = [_p, _p]     # (an fa_append_params by reference, or its bytes)
_APPEND = struct.Struct("@12P12q17i3f")     # fa_append_params
assert _APPEND.size == ctypes.sizeof(fa_append_params)
class fa_latent_params(ctypes.Structure):
    _fields_ = [(name, _p) for name in ("q", "q_rope", "k", "k_rope", "v", "o", "lse", "cu_seqlens_q", "cu_seqlens_k")]
    _fields_ += [(name + "_stride", ctypes.c_int64 * 2) for name in ("q", "q_rope", "k", "v")] + [("k_rope_stride", ctypes.c_int64)]
    _fields_ += [(name, _i) for name in ("B", "H", "total_q", "total_k", "max_seqlen_q", "max_seqlen_k", "d", "d_rope", "causal", "dtype")]
    _fields_ += [("scale", _f)]


lib.fa_forward_latent.restype = _i
lib.fa_forward_latent.argtypes = [_p, _p]   # (an fa_latent_params by reference, or its bytes)
_LATENT = struct.Struct("@9P9q10if0q")      # fa_latent_params
assert _LATENT.size == ctypes.sizeof(fa_latent_params)
class fa_latent_decode_params(ctypes.Structure):
    _fields_ = [(name, _p) for name in ("q", "q_rope", "cache", "o", "lse", "seqlens_k", "block_table")]
    _fields_ += [("q_stride", ctypes.c_int64 * 3), ("q_rope_stride", ctypes.c_int64 * 3)]
    _fields_ += [(name, _i) for name in ("B", "T", "H", "Skv_max", "d", "d_rope", "dtype", "num_pages", "page_size", "max_pages", "table_stride")]
    _fields_ += [("scale", _f), ("workspace", _p), ("workspace_bytes", _sz)]


lib.fa_decode_latent.restype = _i
lib.fa_decode_latent.argtypes = [_p, _p]    # (an fa_latent_decode_params by reference, or its bytes)
_LATENT_DECODE = struct.Struct("@7P6q11ifPN")
assert _LATENT_DECODE.size == ctypes.sizeof(fa_latent_decode_params)
lib.fa_decode_latent_workspace_bytes.restype = _sz
lib.fa_decode_latent_workspace_bytes.argtypes = [_i, _i, _i, _i, _i]
_FA16 = {torch.float16: FA_DTYPE_FP16, torch.bfloat16: FA_DTYPE_BF16}
_FA_PROBS = {**_FA16, torch.float32: FA_DTYPE_FP32}
lib.fa_decode_tree_workspace_bytes.restype = _sz
lib.fa_decode_tree_workspace_bytes.argtypes = [_i, _i, _i, _i, _i, _i, _i]
lib.fa_spec_verify.restype = _i
# Sizes that come from shapes go as words, which an argument of int takes up anyway in the calling conventions of 64-bit Linux: ctypes
# needs half as long for one as for an int (four sizes of a call: 0.35 us).
_w = _p
lib.fa_spec_verify.argtypes = [_p] * 10 + [_w, _w, _w, _w, _p]
lib.fa_cache_compact.restype = _i
lib.fa_cache_compact.argtypes = [_p] * 8 + [_w, _w, _w, _w, _w, _w, _w, _i, _w, _w, _p]
lib.fa_pages_resize.restype = _i
lib.fa_pages_resize.argtypes = [_p] * 5 + [_w, _w, _i, _w, _w, _p]
lib.fa_pages_fork.restype = _i
lib.fa_pages_fork.argtypes = [_p] * 9 + [_w] * 9 + [_p]
lib.fa_decode_append.restype = _i
lib.fa_decode_append.argtypes = [_p, _p, _p, _p, _p, _p, _i, _i, _i, _i, _i, _i, _f, _p, _sz, _p]
lib.fa_decode_append_workspace_bytes.restype = _sz
lib.fa_decode_append_workspace_bytes.argtypes = [_i, _i, _i, _i, _i, _i]
lib.fa_decode_fp8.restype = _i
lib.fa_decode_fp8.argtypes = [_p, _p, _p, _p, _p, _p, _i, _i, _i, _i, _i, _f, _f, _f, _p, _sz, _p]
lib.fa_decode_fp8_paged.restype = _i
lib.fa_decode_fp8_paged.argtypes = [_p, _p, _p, _p, _p, _p, _p, _i, _i, _i, _i, _i, _i, _i, _i, _f, _f, _f, _p, _sz, _p]
lib.fa_decode_fp8_bf16.restype = _i
lib.fa_decode_fp8_bf16.argtypes = lib.fa_decode_fp8.argtypes
lib.fa_decode_fp8_paged_bf16.restype = _i
lib.fa_decode_fp8_paged_bf16.argtypes = lib.fa_decode_fp8_paged.argtypes
lib.fa_forward_varlen_paged.restype = _i
lib.fa_forward_varlen_paged.argtypes = [_p, _p, _p, _p, _p, _p, _p, _p, _i, _i, _i, _i, _i, _i, _i, _i, _i, _i, _i, _i, _f,
                                        _i, _p]
lib.fa_decode_paged.restype = _i
lib.fa_decode_paged.argtypes = [_p, _p, _p, _p, _p, _p, _p, _i, _i, _i, _i, _i, _i, _i, _i, _f, _p, _sz, _p]
lib.fa_decode_noalloc.restype = _i
lib.fa_decode_noalloc.argtypes = [_p, _p, _p, _p, _p, _p, _i, _i, _i, _i, _i, _f, _p]
lib.fa_forward_host.restype = _i
lib.fa_forward_host.argtypes = [_p, _p, _p, _p, _p, _i, _i, _i, _i, _i, _i, _i, _f, _i, _p, _sz, _p]
lib.fa_forward_host_staging_bytes.restype = _sz
lib.fa_forward_host_staging_bytes.argtypes = [_i, _i, _i, _i, _i, _i]
lib.fa_device_status.restype = _i
lib.fa_device_status.argtypes = [ctypes.POINTER(ctypes.c_uint * 2)]
lib.fa_selftest_wait.restype = _i
lib.fa_selftest_wait.argtypes = [ctypes.c_uint, _p, _p]
lib.fa_selftest_decode_cut.restype = _i
lib.fa_selftest_decode_cut.argtypes = [_i, _i, _i, _i, _i, _i, _i, ctypes.POINTER(_i * 4)]
lib.fa_strerror.restype = ctypes.c_char_p
lib.fa_strerror.argtypes = [_i]
lib.fa_version.restype = _i
lib.fa_last_cuda_error.restype = _i

FA_DECODE_NOALLOC_BYTES = 4 << 20

EXPORTS = ["fa_forward", "fa_forward_bf16", "fa_forward_ex", "fa_forward_fp8", "fa_forward_proj", "fa_forward_proj_workspace_bytes", "fa_decode", "fa_decode_workspace_bytes",
           "fa_decode_noalloc", "fa_decode_paged", "fa_forward_varlen", "fa_decode_fp8", "fa_decode_fp8_paged", "fa_decode_fp8_bf16", "fa_decode_fp8_paged_bf16", "fa_decode_append", "fa_decode_append_workspace_bytes", "fa_decode_ex", "fa_forward_varlen_paged",
           "fa_decode_tree", "fa_decode_tree_workspace_bytes", "fa_spec_verify", "fa_cache_compact", "fa_pages_resize", "fa_pages_fork", "fa_rope", "fa_cache_append", "fa_forward_latent",
           "fa_decode_latent", "fa_decode_latent_workspace_bytes",
           "fa_forward_host", "fa_forward_host_staging_bytes", "fa_device_status", "fa_selftest_wait", "fa_selftest_decode_cut", "fa_strerror",
           "fa_version", "fa_last_cuda_error"]


class FaError(RuntimeError):
    def __init__(self, code: int, what: str):
        self.code = code
        super().__init__(f"{what}: {fa_strerror(code)} (code {code}, cuda {fa_last_cuda_error()})")


def fa_strerror(code: int) -> str:
    return lib.fa_strerror(int(code)).decode()


def fa_version() -> int:
    return int(lib.fa_version())


def fa_last_cuda_error() -> int:
    return int(lib.fa_last_cuda_error())


# The current stream's handle without building a torch.cuda.Stream object around it: a call on a few
# hundred keys is bound by what the host does for it, and the object took 3.4 us of its 10.5.  The
# function is torch's own and not promised: a torch without it (one without CUDA among them) takes the object.
_raw_stream, _device = getattr(torch._C, "_cuda_getCurrentRawStream", None), torch.cuda.current_device


def _stream() -> int:
    if _raw_stream is None:
        return int(torch.cuda.current_stream().cuda_stream)
    return _raw_stream(_device())


def _ptr(t) -> int:
    return 0 if t is None else int(t.data_ptr())


def _check(rc: int, what: str, raise_on_error: bool) -> int:
    if rc != FA_OK and raise_on_error:
        raise FaError(rc, what)
    return rc


def fa_forward(q, k, v, o, lse, causal: bool, scale: float, raise_on_error: bool = True) -> int:
    """``fa_forward`` / ``fa_forward_bf16`` on contiguous [B,S,H,d] device tensors (by dtype of q)."""
    B, Sq, Hq, d = q.shape
    _, Skv, Hkv, _ = k.shape
    fn = lib.fa_forward_bf16 if q.dtype == torch.bfloat16 else lib.fa_forward
    rc = fn(_ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse), B, Hq, Hkv, Sq, Skv, d, int(bool(causal)),
            float(scale), _stream())
    return _check(rc, "fa_forward", raise_on_error)


def fa_forward_ex(q, k, v, o, lse, causal: bool, scale: float, variant: int = 0,
                  raise_on_error: bool = True) -> int:
    """``fa_forward_ex``: q/k/v/o are [B,S,H,d] views with any batch/sequence/head strides
    (d contiguous); ``o`` may be fp32 to read the accumulator without the final rounding."""
    B, Sq, Hq, d = q.shape
    _, Skv, Hkv, _ = k.shape
    p = fa_params()
    p.q, p.k, p.v, p.o, p.lse = _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse)
    p.B, p.Hq, p.Hkv, p.Sq, p.Skv, p.d = B, Hq, Hkv, Sq, Skv, d
    p.causal, p.scale = int(bool(causal)), float(scale)
    p.dtype = FA_DTYPE_BF16 if q.dtype == torch.bfloat16 else FA_DTYPE_FP16
    p.o_dtype = FA_DTYPE_FP32 if o.dtype == torch.float32 else p.dtype
    for name, t in (("q_stride", q), ("k_stride", k), ("v_stride", v), ("o_stride", o)):
        arr = getattr(p, name)
        arr[0], arr[1], arr[2] = t.stride(0), t.stride(1), t.stride(2)
    p.variant = int(variant)
    rc = lib.fa_forward_ex(ctypes.byref(p), _stream())
    return _check(rc, "fa_forward_ex", raise_on_error)


def fa_forward_fp8(q, k, v, o, lse, causal: bool, scale: float, q_scale: float, k_scale: float, v_scale: float,
                   raise_on_error: bool = True) -> int:
    """``fa_forward_fp8``: q [B,Sq,Hq,d], k, v [B,Skv,Hkv,d] contiguous device tensors of FP8 e4m3
    (``torch.float8_e4m3fn`` or uint8 bit patterns) with one factor each; o fp16 or bf16."""
    B, Sq, Hq, d = q.shape
    _, Skv, Hkv, _ = k.shape
    dt = FA_DTYPE_BF16 if o.dtype == torch.bfloat16 else FA_DTYPE_FP16
    rc = lib.fa_forward_fp8(_ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse), B, Hq, Hkv, Sq, Skv, d, int(bool(causal)),
                            float(scale), float(q_scale), float(k_scale), float(v_scale), dt, _stream())
    return _check(rc, "fa_forward_fp8", raise_on_error)


def fa_forward_proj_workspace_bytes(B: int, Sq: int) -> int:
    return int(lib.fa_forward_proj_workspace_bytes(B, Sq))


def fa_forward_proj(q, k, v, w_o, o, lse, out, causal: bool, scale: float, fused: bool, workspace=None,
                    raise_on_error: bool = True) -> int:
    """``fa_forward_proj``: attention, then ``out = O.view(B, Sq, Hq*d) @ w_o`` with w_o [Hq*d, d_model];
    one launch (``fused``, needs a workspace of ``fa_forward_proj_workspace_bytes`` bytes) or two."""
    B, Sq, Hq, d = q.shape
    _, Skv, Hkv, _ = k.shape
    dt = FA_DTYPE_BF16 if q.dtype == torch.bfloat16 else FA_DTYPE_FP16
    wbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    rc = lib.fa_forward_proj(_ptr(q), _ptr(k), _ptr(v), _ptr(w_o), _ptr(o), _ptr(lse), _ptr(out), B, Hq, Hkv, Sq, Skv, d,
                             w_o.shape[1], int(bool(causal)), float(scale), dt, int(bool(fused)), _ptr(workspace), wbytes,
                             _stream())
    return _check(rc, "fa_forward_proj", raise_on_error)


def fa_forward_varlen(q, k, v, o, lse, cu_seqlens_q, cu_seqlens_k, max_seqlen_q: int, max_seqlen_k: int,
                      causal: bool, scale: float, raise_on_error: bool = True) -> int:
    """``fa_forward_varlen``: q, o [total_q,Hq,d], k, v [total_k,Hkv,d] contiguous device tensors,
    lse [Hq,total_q] or None, cu_seqlens_* int32 [B+1] on the device."""
    total_q, Hq, d = q.shape
    total_k, Hkv, _ = k.shape
    B = cu_seqlens_q.numel() - 1
    dt = FA_DTYPE_BF16 if q.dtype == torch.bfloat16 else FA_DTYPE_FP16
    rc = lib.fa_forward_varlen(_ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse), _ptr(cu_seqlens_q),
                               _ptr(cu_seqlens_k), B, Hq, Hkv, total_q, total_k, int(max_seqlen_q),
                               int(max_seqlen_k), d, int(bool(causal)), float(scale), dt, _stream())
    return _check(rc, "fa_forward_varlen", raise_on_error)


def fa_decode_workspace_bytes(B: int, Hq: int, Hkv: int, Skv_max: int, d: int) -> int:
    return int(lib.fa_decode_workspace_bytes(B, Hq, Hkv, Skv_max, d))


def fa_decode(q, k_cache, v_cache, o, lse, seqlens_k, scale: float, workspace,
              raise_on_error: bool = True) -> int:
    """``fa_decode``: q [B,1,Hq,d], caches [B,Smax,Hkv,d], seqlens_k int32 [B] on the device,
    workspace a device byte tensor of at least ``fa_decode_workspace_bytes`` bytes."""
    B, _, Hq, d = q.shape
    _, Smax, Hkv, _ = k_cache.shape
    wbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    rc = lib.fa_decode(_ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(o), _ptr(lse), _ptr(seqlens_k), B, Hq,
                       Hkv, Smax, d, float(scale), _ptr(workspace), wbytes, _stream())
    return _check(rc, "fa_decode", raise_on_error)


def fa_forward_varlen_paged(q, k_pages, v_pages, block_table, o, lse, cu_seqlens_q, seqlens_k, max_seqlen_q: int,
                            max_seqlen_k: int, causal: bool, scale: float, raise_on_error: bool = True) -> int:
    """``fa_forward_varlen_paged``: q, o [total_q,Hq,d] packed, K and V in page pools [num_pages,page_size,Hkv,d]
    behind block_table int32 [B,stride]; cu_seqlens_q int32 [B+1] and seqlens_k int32 [B] on the device."""
    total_q, Hq, d = q.shape
    num_pages, page_size, Hkv, _ = k_pages.shape
    B = cu_seqlens_q.numel() - 1
    dt = FA_DTYPE_BF16 if q.dtype == torch.bfloat16 else FA_DTYPE_FP16
    rc = lib.fa_forward_varlen_paged(_ptr(q), _ptr(k_pages), _ptr(v_pages), _ptr(block_table), _ptr(o), _ptr(lse),
                                     _ptr(cu_seqlens_q), _ptr(seqlens_k), B, Hq, Hkv, total_q, num_pages, page_size,
                                     block_table.shape[1], block_table.stride(0), int(max_seqlen_q), int(max_seqlen_k), d,
                                     int(bool(causal)), float(scale), dt, _stream())
    return _check(rc, "fa_forward_varlen_paged", raise_on_error)


def fa_decode_ex(q, k, v, o, lse, seqlens_k, scale: float, workspace, block_table=None, max_pages: int = None,
                 raise_on_error: bool = True) -> int:
    """``fa_decode_ex``: fp16 or bf16 (from q's dtype); q, o [B,Sq,Hq,d]; k, v the caches [B,Smax,Hkv,d] or, with a
    block table, the page pools [num_pages,page_size,Hkv,d]."""
    p = fa_decode_params()
    p.q, p.k, p.v, p.o, p.lse = _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse)
    p.seqlens_k, p.block_table = _ptr(seqlens_k), _ptr(block_table)
    p.B, p.Sq, p.Hq, p.d = q.shape
    p.Hkv = k.shape[2]
    p.dtype = FA_DTYPE_BF16 if q.dtype == torch.bfloat16 else FA_DTYPE_FP16
    if block_table is None:
        p.Skv_max = k.shape[1]
    else:
        p.num_pages, p.page_size = k.shape[0], k.shape[1]
        p.max_pages = block_table.shape[1] if max_pages is None else int(max_pages)
        p.table_stride = block_table.stride(0)
    p.scale = float(scale)
    p.workspace = _ptr(workspace)
    p.workspace_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    rc = lib.fa_decode_ex(ctypes.byref(p), _stream())
    return _check(rc, "fa_decode_ex", raise_on_error)


# The checks of the calls below: what the library cannot see of its pointers.  Types, layouts and sizes, as a tensor that is too
# small would be read or written past its end; vectors [B] may be longer than the batch.  (A step's calls are short, and bound by what the host
# does for them: a call first asks in one expression whether all is well, and looks for what is wrong only if not; parameter
# blocks are packed, not filled field by field.  fa_decode_tree 6.7 -> 3.8 us before the library, fa_cache_compact 10.3 -> 5.7.)
_INT, _HALF, _BF16, _FLOAT = torch.int32, torch.float16, torch.bfloat16, torch.float32


def _contiguous(what: str, *tensors) -> None:
    """The calls below take contiguous tensors; a view would be read as something else."""
    for t in tensors:
        if t is not None and not t.is_contiguous():
            raise ValueError(f"{what}: a tensor of shape {tuple(t.shape)} and strides {t.stride()} is not contiguous")


def _int32(what: str, *tensors) -> None:
    for t in tensors:
        if t is not None and t.dtype is not _INT:
            raise ValueError(f"{what}: index tensors are int32, not {t.dtype}")


def _shapes(what: str, **tensors) -> None:
    """The call's tensors do not go together: says how."""
    given = ", ".join(f"{name} {tuple(t.shape)}" for name, t in tensors.items() if t is not None)
    raise ValueError(f"{what}: shapes that do not go together, {given}")


def _table(what: str, t) -> int:
    """The stride of a block table, whose rows are contiguous."""
    stride, one = t.stride()
    if t.dtype is not _INT or (one != 1 and t.shape[1] > 1):
        raise ValueError(f"{what}: a block table is int32 [B,pages] with contiguous rows, not {t.dtype} of strides {t.stride()}")
    return stride


def tree_mask(parents):
    """The mask of ``fa_decode_tree`` for trees given by their parents, int32 [B,T] (or [T]; parents[i] < i, -1 for the root): each
    node sees itself and the nodes above it.  A number outside [0, i) is no parent, as for ``fa_spec_verify`` (entries past a tree's
    length may hold anything).  Made with torch operations on the parents' device, once per step."""
    T = parents.shape[-1]
    up = parents.long()
    up = torch.where(up < torch.arange(T, device=up.device), up, -1)
    see = torch.eye(T, dtype=torch.bool, device=parents.device).expand(*up.shape, T).clone()
    hop = up.clamp(min=0).unsqueeze(-1)
    for _ in range(max(1, (T - 1).bit_length())):   # what a node's ancestor sees, twice as far up each time
        live = (up >= 0).unsqueeze(-1)
        see = see | (torch.gather(see, -2, hop.expand_as(see)) & live)
        up = torch.where(up >= 0, torch.gather(up, -1, hop.squeeze(-1)), up)
        hop = up.clamp(min=0).unsqueeze(-1)
    W = (T + 31) // 32
    bits = torch.zeros(*see.shape[:-1], W * 32, dtype=torch.int64, device=see.device)
    bits[..., :T] = see
    words = (bits.view(*see.shape[:-1], W, 32) << torch.arange(32, device=see.device)).sum(-1)
    return torch.where(words >= 1 << 31, words - (1 << 32), words).to(torch.int32)


def fa_decode_tree_workspace_bytes(B: int, T: int, Hq: int, Hkv: int, Skv_max: int, d: int, variant: int = 0) -> int:
    return int(lib.fa_decode_tree_workspace_bytes(B, T, Hq, Hkv, Skv_max, d, variant))


def fa_decode_tree(q, k, v, o, lse, seqlens_k, mask, scale: float, workspace, tree_lens=None, block_table=None,
                   max_pages: int = None, variant: int = 0, raise_on_error: bool = True) -> int:
    """``fa_decode_tree``: q, o [B,T,Hq,d], the nodes of each sequence's tree, whose rows end its cache; mask int32
    [B,T,ceil(T/32)], or [T,ceil(T/32)] for one tree (see ``tree_mask``); k, v, block_table as for ``fa_decode_ex``; seqlens_k
    int32 [B] with the tree's rows, tree_lens int32 [B] or None."""
    dt = q.dtype
    if not (k.dtype is dt and v.dtype is dt and o.dtype is dt and (dt is _HALF or dt is _BF16)):
        raise ValueError("fa_decode_tree: q, k, v and o share one 16-bit type")
    if not (q.is_contiguous() and k.is_contiguous() and v.is_contiguous() and o.is_contiguous() and seqlens_k.dtype is _INT
            and seqlens_k.is_contiguous() and mask.dtype is _INT and mask.is_contiguous()
            and (tree_lens is None or (tree_lens.dtype is _INT and tree_lens.is_contiguous()))
            and (lse is None or (lse.is_contiguous() and lse.dtype is _FLOAT))):
        _contiguous("fa_decode_tree", q, k, v, o, lse, seqlens_k, mask, tree_lens)
        _int32("fa_decode_tree", seqlens_k, mask, tree_lens)
        raise ValueError("fa_decode_tree: lse is float32")
    B, T, Hq, d = shape = q.shape
    slabs, rows, Hkv, width = cache = k.shape
    seen = mask.shape
    if seen != (B, T, (T + 31) // 32) and seen != (T, (T + 31) // 32):
        raise ValueError(f"fa_decode_tree: a mask of shape {tuple(seen)} for T = {T}")
    if block_table is None:
        tables, sizes = slabs, (rows, d, _FA16[dt], 0, 0, 0, 0)
    else:
        tables, pages = block_table.shape
        sizes = (0, d, _FA16[dt], slabs, rows, pages if max_pages is None else max_pages, _table("fa_decode_tree", block_table))
    if not (o.shape == shape and v.shape == cache and width == d and tables >= B and seqlens_k.numel() >= B
            and (tree_lens is None or tree_lens.numel() >= B) and (lse is None or lse.numel() >= B * Hq * T)):
        _shapes("fa_decode_tree", q=q, o=o, k=k, v=v, seqlens_k=seqlens_k, tree_lens=tree_lens, lse=lse, block_table=block_table)
    p = _TREE.pack(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), 0 if lse is None else lse.data_ptr(), seqlens_k.data_ptr(),
                   0 if tree_lens is None else tree_lens.data_ptr(), mask.data_ptr(), 0 if block_table is None else block_table.data_ptr(),
                   B, T, Hq, Hkv, *sizes, variant, 0 if len(seen) == 2 else T * seen[2], scale,
                   0 if workspace is None else workspace.data_ptr(), 0 if workspace is None else workspace.nbytes)
    rc = lib.fa_decode_tree(p, _stream())
    return _check(rc, "fa_decode_tree", raise_on_error) if rc else rc


def fa_spec_verify(target_probs, draft_probs, tokens, parents, uniforms, noise, n_accept, path, out_tokens, tree_lens=None,
                   raise_on_error: bool = True) -> int:
    """``fa_spec_verify``: target_probs [B,T,V] (fp32, fp16 or bf16), draft_probs the same or None, tokens, parents int32 [B,T],
    uniforms float32 [B,T], noise float32 [B,V]; writes n_accept int32 [B], path and out_tokens int32 [B,T]."""
    dt = target_probs.dtype
    if dt not in _FA_PROBS or (draft_probs is not None and draft_probs.dtype is not dt):
        raise ValueError("fa_spec_verify: probabilities are fp32, fp16 or bf16, both of one type")
    if uniforms.dtype is not _FLOAT or noise.dtype is not _FLOAT:
        raise ValueError("fa_spec_verify: random numbers are float32")
    if not (target_probs.is_contiguous() and (draft_probs is None or draft_probs.is_contiguous()) and uniforms.is_contiguous() and noise.is_contiguous()
            and tokens.dtype is _INT and tokens.is_contiguous() and parents.dtype is _INT and parents.is_contiguous() and path.dtype is _INT
            and path.is_contiguous() and out_tokens.dtype is _INT and out_tokens.is_contiguous() and n_accept.dtype is _INT
            and n_accept.is_contiguous() and (tree_lens is None or (tree_lens.dtype is _INT and tree_lens.is_contiguous()))):
        _contiguous("fa_spec_verify", target_probs, draft_probs, tokens, parents, uniforms, noise, n_accept, path, out_tokens, tree_lens)
        _int32("fa_spec_verify", tokens, parents, n_accept, path, out_tokens, tree_lens)
    B, T, V = shape = target_probs.shape
    if not (tokens.numel() == parents.numel() == uniforms.numel() == path.numel() == out_tokens.numel() == B * T and noise.numel() == B * V
            and n_accept.numel() >= B and (draft_probs is None or draft_probs.shape == shape) and (tree_lens is None or tree_lens.numel() >= B)):
        _shapes("fa_spec_verify", target_probs=target_probs, draft_probs=draft_probs, tokens=tokens, parents=parents, uniforms=uniforms, noise=noise,
                n_accept=n_accept, path=path, out_tokens=out_tokens, tree_lens=tree_lens)
    rc = lib.fa_spec_verify(target_probs.data_ptr(), 0 if draft_probs is None else draft_probs.data_ptr(), tokens.data_ptr(), parents.data_ptr(),
                            0 if tree_lens is None else tree_lens.data_ptr(), uniforms.data_ptr(), noise.data_ptr(), n_accept.data_ptr(),
                            path.data_ptr(), out_tokens.data_ptr(), B, T, V, _FA_PROBS[dt], _stream())
    return _check(rc, "fa_spec_verify", raise_on_error) if rc else rc


def _planes(what: str, k, v):
    """(layers, slabs, rows of a slab, bytes between layers, bytes of a row) of caches [layers, slabs, rows, ...], each layer contiguous."""
    shape, stride = k.shape, k.stride()
    if v.shape != shape or k.dtype is not v.dtype or v.stride() != stride:
        raise ValueError(f"{what}: k and v are of one shape, type and layout")
    if not k.is_contiguous():
        _contiguous(what, k[0])
    size = k.element_size()
    # (the stride of an extent of 1 may be any number)
    layer = stride[0] if shape[0] > 1 else 0
    row = stride[2] if shape[2] > 1 else math.prod(shape[3:])
    return shape[0], shape[1], shape[2], layer * size, row * size


def fa_cache_compact(k, v, seqlens_k, path, n_accept, new_lens, tree_lens=None, block_table=None, max_pages: int = None,
                     raise_on_error: bool = True) -> int:
    """``fa_cache_compact``: k, v the caches of all layers, [L,B,Smax,Hkv,d], or with a block table the pools
    [L,num_pages,page_size,Hkv,d] (any element type); path int32 [B,T], n_accept int32 [B] as ``fa_spec_verify`` writes
    them; writes new_lens int32 [B]."""
    layers, slabs, rows, stride, row = _planes("fa_cache_compact", k, v)
    if not (seqlens_k.dtype is _INT and path.dtype is _INT and n_accept.dtype is _INT and new_lens.dtype is _INT and path.is_contiguous()
            and seqlens_k.is_contiguous() and n_accept.is_contiguous() and new_lens.is_contiguous()
            and (tree_lens is None or (tree_lens.dtype is _INT and tree_lens.is_contiguous()))):
        _contiguous("fa_cache_compact", seqlens_k, path, n_accept, new_lens, tree_lens)
        _int32("fa_cache_compact", seqlens_k, path, n_accept, new_lens, tree_lens)
    B, T = path.shape
    if block_table is None:
        tables, args = slabs, (rows, 0, 0, 0, 0)
    else:
        tables, pages = block_table.shape
        args = (0, slabs, rows, pages if max_pages is None else max_pages, _table("fa_cache_compact", block_table))
    if not (tables >= B and seqlens_k.numel() >= B and n_accept.numel() >= B and new_lens.numel() >= B and (tree_lens is None or tree_lens.numel() >= B)):
        _shapes("fa_cache_compact", k=k, path=path, seqlens_k=seqlens_k, n_accept=n_accept, new_lens=new_lens, tree_lens=tree_lens, block_table=block_table)
    rc = lib.fa_cache_compact(k.data_ptr(), v.data_ptr(), 0 if block_table is None else block_table.data_ptr(), seqlens_k.data_ptr(),
                              0 if tree_lens is None else tree_lens.data_ptr(), path.data_ptr(), n_accept.data_ptr(), new_lens.data_ptr(),
                              layers, stride, B, T, *args, row, _stream())
    return _check(rc, "fa_cache_compact", raise_on_error) if rc else rc


def fa_pages_resize(block_table, held, refs, want, n_short, page_size: int, raise_on_error: bool = True) -> int:
    """``fa_pages_resize``: block_table int32 [B,max_pages], held int32 [B], refs int32 [num_pages], want int32 [B] (rows);
    n_short int32 [1] counts the sequences that could not be served."""
    if not (held.dtype is _INT and refs.dtype is _INT and want.dtype is _INT and n_short.dtype is _INT and held.is_contiguous()
            and refs.is_contiguous() and want.is_contiguous() and n_short.is_contiguous()):
        _contiguous("fa_pages_resize", held, refs, want, n_short)
        _int32("fa_pages_resize", held, refs, want, n_short)
    B, pages = block_table.shape
    if not (held.numel() >= B and want.numel() >= B and n_short.numel() >= 1):
        _shapes("fa_pages_resize", block_table=block_table, held=held, want=want, n_short=n_short)
    if B == 0:   # (a call of the library that has nothing to do writes nothing)
        n_short.zero_()
    rc = lib.fa_pages_resize(block_table.data_ptr(), held.data_ptr(), refs.data_ptr(), want.data_ptr(), n_short.data_ptr(), B, refs.numel(),
                             page_size, pages, _table("fa_pages_resize", block_table), _stream())
    return _check(rc, "fa_pages_resize", raise_on_error) if rc else rc


def fa_pages_fork(k, v, block_table, held, seqlens_k, refs, src, dst, n_short, raise_on_error: bool = True) -> int:
    """``fa_pages_fork``: pools k, v [L,num_pages,page_size,Hkv,d] with the state of ``fa_pages_resize`` and seqlens_k int32
    [B]; sequence dst[i] becomes a copy of src[i] (int32 [n] each); n_short int32 [1] counts the pairs that got no page."""
    layers, slabs, rows, stride, row = _planes("fa_pages_fork", k, v)
    if not (held.dtype is _INT and held.is_contiguous() and seqlens_k.dtype is _INT and seqlens_k.is_contiguous() and refs.dtype is _INT
            and refs.is_contiguous() and src.dtype is _INT and src.is_contiguous() and dst.dtype is _INT and dst.is_contiguous()
            and n_short.dtype is _INT and n_short.is_contiguous()):
        _contiguous("fa_pages_fork", held, seqlens_k, refs, src, dst, n_short)
        _int32("fa_pages_fork", held, seqlens_k, refs, src, dst, n_short)
    if refs.numel() != slabs:
        raise ValueError("fa_pages_fork: refs has an entry for each of the pool's pages")
    B, pages = block_table.shape
    if not (held.numel() >= B and seqlens_k.numel() >= B and src.numel() == dst.numel() and n_short.numel() >= 1):
        _shapes("fa_pages_fork", block_table=block_table, held=held, seqlens_k=seqlens_k, src=src, dst=dst, n_short=n_short)
    if src.numel() == 0:
        n_short.zero_()
    rc = lib.fa_pages_fork(k.data_ptr(), v.data_ptr(), block_table.data_ptr(), held.data_ptr(), seqlens_k.data_ptr(), refs.data_ptr(),
                           src.data_ptr(), dst.data_ptr(), n_short.data_ptr(), src.numel(), layers, stride, B, slabs, rows, pages,
                           _table("fa_pages_fork", block_table), row, _stream())
    return _check(rc, "fa_pages_fork", raise_on_error) if rc else rc


def rope_frequencies(rot_dim: int, base: float = 10000.0, stretch: float = 1.0, trained: int = 0, slow: float = 1.0, fast: float = 32.0,
                     device="cuda"):
    """Radians per position of each pair of ``rot_dim`` rotated columns, float64: base^(-2 i / rot_dim).  ``stretch`` > 1 scales them for
    contexts so many times longer: all alike (positions drawn together), or, with ``trained`` the context a model was trained on,
    by parts: pairs that turn less than ``slow`` times over it are slowed down by stretch, those that turn more than ``fast`` times
    stay, in between it is a mixture of both, linear in the turns.  (A larger base is given as such.)"""
    w = float(base) ** (-torch.arange(0, rot_dim, 2, dtype=torch.float64, device=device) / rot_dim)
    if stretch == 1.0:
        return w
    if not trained:
        return w / stretch
    keep = ((trained * w / (2.0 * math.pi) - slow) / (fast - slow)).clamp(0.0, 1.0)
    return w * (keep + (1.0 - keep) / stretch)


def rope_turns(frequencies):
    """The ``turns`` of ``fa_rope`` and ``fa_cache_append`` for frequencies in radians per position (float64 [rot_dim / 2], see
    ``rope_frequencies``): shares of a full turn in 64-bit fixed point, int64 (its bits are what counts).  Made once for a model."""
    if frequencies.dtype is not torch.float64 or frequencies.dim() != 1:
        raise ValueError("rope_turns: frequencies are float64 [rot_dim / 2] (32 bits lose the angles of far positions)")
    share = frequencies / (2.0 * math.pi)
    share = share - share.round()
    return torch.where(share >= 0.5, share - 1.0, share).mul(2.0 ** 64).to(torch.int64)   # (half a turn either way is the same)


def _turns(what: str, t) -> int:
    if t.dtype is not torch.int64 or not t.is_contiguous() or t.dim() != 1:
        raise ValueError(f"{what}: turns are int64 [rot_dim / 2], contiguous (see rope_turns)")
    return 2 * t.shape[0]


def fa_rope(x, out, positions, turns, offset: int = 0, interleaved: bool = False, factor: float = 1.0, raise_on_error: bool = True) -> int:
    """``fa_rope``: x, out [n,H,d] (out may be x), fp16 or bf16, any strides of tokens and heads; positions int32 [n]; turns from
    ``rope_turns``, for the 2 * len(turns) columns of each head from ``offset`` on."""
    dt = x.dtype
    n, H, d = shape = x.shape
    xt, xh, xd = x.stride()
    ot, oh, od = out.stride()
    if not (out.dtype is dt and (dt is _HALF or dt is _BF16) and out.shape == shape and xd == 1 and od == 1 and positions.dtype is _INT
            and positions.numel() >= n and positions.is_contiguous()):
        if out.dtype is not dt or dt not in _FA16:
            raise ValueError("fa_rope: x and out share one 16-bit type")
        _contiguous("fa_rope", positions)
        _int32("fa_rope", positions)
        if xd != 1 or od != 1:
            raise ValueError("fa_rope: the columns of a head are contiguous")
        _shapes("fa_rope", x=x, out=out, positions=positions)
    rot = _turns("fa_rope", turns)
    if n <= 1:   # (the stride of an extent of 1 may be any number)
        xt = ot = 0
    if H <= 1:
        xh = oh = 0
    rc = lib.fa_rope(x.data_ptr(), out.data_ptr(), positions.data_ptr(), turns.data_ptr(), n, H, d, rot, offset, 1 if interleaved else 0, factor,
                     xt, xh, ot, oh, _FA16[dt], _stream())
    return _check(rc, "fa_rope", raise_on_error) if rc else rc


def _tokens(what: str, t):
    """(tokens, heads, width, stride of a token, stride of a head) of [n,H,d] or [B,T,H,d]."""
    shape = t.shape
    if len(shape) == 3 and t.is_contiguous():
        n, H, d = shape
        return n, H, d, H * d, d
    stride = t.stride()
    if stride[-1] != 1 and shape[-1] != 1:
        raise ValueError(f"{what}: the columns of a head are contiguous")
    if len(shape) == 3:
        n, H, d = shape
        return n, H, d, stride[0] if n > 1 else 0, stride[1] if H > 1 else 0
    B, T, H, d = shape
    if B > 1 and T > 1 and stride[0] != T * stride[1]:
        raise ValueError(f"{what}: the tokens of [B,T,H,d] are as far apart from one sequence to the next as inside it")
    return B * T, H, d, (stride[1] if T > 1 else stride[0]) if B * T > 1 else 0, stride[2] if H > 1 else 0


def _rows(what: str, cache, Hkv: int, d: int):
    """(slabs, rows of a slab, stride of a slab, stride of a row) of a cache [slabs,rows,Hkv,d], or [slabs,rows,d] for one head."""
    shape = cache.shape
    if len(shape) == 4 and shape[2] == Hkv and shape[3] == d and cache.is_contiguous():
        return shape[0], shape[1], shape[1] * Hkv * d, Hkv * d
    stride = cache.stride()
    if len(shape) == 4:
        slabs, rows, heads, width = shape
        good = stride[3] == 1 and (Hkv == 1 or stride[2] == d)
    else:
        slabs, rows, width = shape
        heads, good = 1, stride[2] == 1
    if heads != Hkv or width != d:
        raise ValueError(f"{what}: a cache of shape {tuple(shape)} for {Hkv} heads of {d}")
    if not good:
        raise ValueError(f"{what}: a row of a cache is contiguous, not of strides {stride[2:]}")
    return slabs, rows, stride[0] if slabs > 1 else 0, stride[1] if rows > 1 else 0


def fa_cache_append(q, q_out, k, v, k_cache, v_cache, first_rows, turns=None, positions=None, counts=None, cu_seqlens=None,
                    block_table=None, max_pages: int = None, offset: int = 0, interleaved: bool = False, factor: float = 1.0,
                    k_scale: float = 1.0, v_scale: float = 1.0, raise_on_error: bool = True) -> int:
    """``fa_cache_append``: q, q_out [n,Hq,d] (or None), k [n,Hkv,d], v [n,Hkv,dv] (or None), packed by cu_seqlens int32 [B+1], or
    without it [B,T,H,d] or the same tokens as [n,H,d]; first_rows int32 [B]; caches [B,Smax,Hkv,d] and [B,Smax,Hkv,dv], or with a block table
    [num_pages,page_size,...], of the inputs' type or FP8 e4m3 (``torch.float8_e4m3fn`` or uint8 bit patterns) with one factor
    each; turns from ``rope_turns`` (None: no rotation); positions int32 [n], counts int32 [B] or None."""
    what, dt = "fa_cache_append", k.dtype
    if not ((dt is _HALF or dt is _BF16) and (v is None or v.dtype is dt) and (q is None or (q.dtype is dt and q_out.dtype is dt))):
        raise ValueError(f"{what}: q, q_out, k and v share one 16-bit type")
    ct = k_cache.dtype
    f8 = ct is torch.float8_e4m3fn or ct is torch.uint8
    if not (f8 or ct is dt) or (v is not None and v_cache.dtype is not ct):
        raise ValueError(f"{what}: caches are of the inputs' type or e4m3, both of one type")
    if not (first_rows.dtype is _INT and first_rows.is_contiguous() and (positions is None or (positions.dtype is _INT and positions.is_contiguous()))
            and (counts is None or (counts.dtype is _INT and counts.is_contiguous()))
            and (cu_seqlens is None or (cu_seqlens.dtype is _INT and cu_seqlens.is_contiguous()))):
        _int32(what, first_rows, positions, counts, cu_seqlens)
        _contiguous(what, first_rows, positions, counts, cu_seqlens)
    n, Hkv, d, kt, kh = _tokens(what, k)
    slabs, rows, ks, kr = _rows(what, k_cache, Hkv, d)
    fits = True
    Hq = qt = qh = ot = oh = dv = vt = vh = vs = vr = 0
    if q is not None:
        nq, Hq, dq, qt, qh = _tokens(what, q)
        no, ho, do, ot, oh = _tokens(what, q_out)
        fits = nq == no == n and ho == Hq and dq == do == d
    if v is not None:
        nv, hv, dv, vt, vh = _tokens(what, v)
        slabs_v, rows_v, vs, vr = _rows(what, v_cache, Hkv, dv)
        fits = fits and nv == n and hv == Hkv and slabs_v == slabs and rows_v == rows
    B = first_rows.numel() if cu_seqlens is None else cu_seqlens.numel() - 1
    if cu_seqlens is None and k.dim() == 4:
        B = k.shape[0]
    T = 0 if cu_seqlens is not None or B == 0 else n // B
    if block_table is None:
        tables, sizes = slabs, (rows, 0, 0, 0, 0)
    else:
        tables, pages = block_table.shape
        sizes = (0, slabs, rows, pages if max_pages is None else max_pages, _table(what, block_table))
    if not (fits and tables >= B and first_rows.numel() >= B and (counts is None or counts.numel() >= B)
            and (positions is None or positions.numel() >= n) and (cu_seqlens is not None or B * T == n)):
        _shapes(what, q=q, q_out=q_out, k=k, v=v, k_cache=k_cache, v_cache=v_cache, first_rows=first_rows, positions=positions, counts=counts,
                cu_seqlens=cu_seqlens, block_table=block_table)
    rot = 0 if turns is None else _turns(what, turns)
    p = _APPEND.pack(0 if q is None else q.data_ptr(), 0 if q is None else q_out.data_ptr(), k.data_ptr(), 0 if v is None else v.data_ptr(),
                     k_cache.data_ptr(), 0 if v is None else v_cache.data_ptr(), 0 if turns is None else turns.data_ptr(),
                     0 if positions is None else positions.data_ptr(), first_rows.data_ptr(), 0 if counts is None else counts.data_ptr(),
                     0 if cu_seqlens is None else cu_seqlens.data_ptr(), 0 if block_table is None else block_table.data_ptr(),
                     qt, qh, ot, oh, kt, kh, vt, vh, ks, kr, vs, vr, n, B, T, Hq, Hkv, d, dv, rot, offset if rot else 0, 1 if interleaved else 0,
                     _FA16[dt], FA_DTYPE_E4M3 if f8 else _FA16[dt], *sizes, factor, k_scale, v_scale)
    rc = lib.fa_cache_append(p, _stream())
    return _check(rc, what, raise_on_error) if rc else rc


def fa_forward_latent(q, q_rope, k, k_rope, v, o, lse, cu_seqlens_q, cu_seqlens_k, max_seqlen_q: int, max_seqlen_k: int, causal: bool, scale: float,
                      raise_on_error: bool = True) -> int:
    """``fa_forward_latent``: a packed batch, q [total_q,H,128] and q_rope [total_q,H,64], k, v [total_k,H,128], k_rope [total_k,64] shared
    by the heads, all with any strides of tokens and heads; o [total_q,H,128] contiguous, lse [H,total_q] or None; cu_seqlens_* int32 [B+1]."""
    what, dt = "fa_forward_latent", q.dtype
    if not ((dt is _HALF or dt is _BF16) and q_rope.dtype is dt and k.dtype is dt and k_rope.dtype is dt and v.dtype is dt and o.dtype is dt):
        raise ValueError(f"{what}: q, q_rope, k, k_rope, v and o share one 16-bit type")
    if not (o.is_contiguous() and cu_seqlens_q.dtype is _INT and cu_seqlens_k.dtype is _INT and cu_seqlens_q.is_contiguous() and cu_seqlens_k.is_contiguous()
            and (lse is None or (lse.dtype is _FLOAT and lse.is_contiguous()))):
        _int32(what, cu_seqlens_q, cu_seqlens_k)
        _contiguous(what, o, lse, cu_seqlens_q, cu_seqlens_k)
        raise ValueError(f"{what}: lse is float32")
    n, H, d, qt, qh = _tokens(what, q)
    nr, hr, rope, rt, rh = _tokens(what, q_rope)
    m, hk, dk, kt, kh = _tokens(what, k)
    mv, hv, dv, vt, vh = _tokens(what, v)
    B = cu_seqlens_q.shape[0] - 1
    if not (nr == n and hr == hk == hv == H and dk == dv == d and mv == m and k_rope.shape == (m, rope) and o.shape == (n, H, d)
            and (lse is None or lse.numel() == H * n) and cu_seqlens_k.shape[0] == B + 1 >= 1):
        _shapes(what, q=q, q_rope=q_rope, k=k, k_rope=k_rope, v=v, o=o, lse=lse, cu_seqlens_q=cu_seqlens_q, cu_seqlens_k=cu_seqlens_k)
    if k_rope.stride(1) != 1:
        raise ValueError(f"{what}: the columns of k_rope are contiguous")
    p = _LATENT.pack(q.data_ptr(), q_rope.data_ptr(), k.data_ptr(), k_rope.data_ptr(), v.data_ptr(), o.data_ptr(), 0 if lse is None else lse.data_ptr(),
                     cu_seqlens_q.data_ptr(), cu_seqlens_k.data_ptr(), qt, qh, rt, rh, kt, kh, vt, vh, k_rope.stride(0) if m > 1 else 0,
                     B, H, n, m, max_seqlen_q, max_seqlen_k, d, rope, 1 if causal else 0, _FA16[dt], scale)
    rc = lib.fa_forward_latent(p, _stream())
    return _check(rc, what, raise_on_error) if rc else rc


def fa_decode_latent_workspace_bytes(B: int, T: int, H: int, Skv_max: int, d: int = 512) -> int:
    return int(lib.fa_decode_latent_workspace_bytes(B, T, H, Skv_max, d))


def fa_decode_latent(q, q_rope, cache, o, lse, seqlens_k, scale: float, workspace, block_table=None, max_pages: int = None,
                     raise_on_error: bool = True) -> int:
    """``fa_decode_latent``: q [B,T,H,512] and q_rope [B,T,H,64] of any strides (two parts of one tensor, for instance), cache [B,Smax,576] or with a
    block table the pool [num_pages,page_size,576]; o [B,T,H,512] contiguous, lse [B,H,T] or None; seqlens_k int32 [B], the T tokens included."""
    what, dt = "fa_decode_latent", q.dtype
    if not (q_rope.dtype is dt and cache.dtype is dt and o.dtype is dt and (dt is _HALF or dt is _BF16)):
        raise ValueError(f"{what}: q, q_rope, cache and o share one 16-bit type")
    if not (cache.is_contiguous() and o.is_contiguous() and seqlens_k.dtype is _INT and seqlens_k.is_contiguous()
            and (lse is None or (lse.is_contiguous() and lse.dtype is _FLOAT))):
        _contiguous(what, cache, o, lse, seqlens_k)
        _int32(what, seqlens_k)
        raise ValueError(f"{what}: lse is float32")
    B, T, H, d = shape = q.shape
    rope = q_rope.shape[3]
    slabs, rows, width = cache.shape
    qb, qt, qh, q1 = q.stride()
    rb, rt, rh, r1 = q_rope.stride()
    if q1 != 1 or r1 != 1:
        raise ValueError(f"{what}: the columns of a head are contiguous")
    if block_table is None:
        tables, Smax, sizes = slabs, rows, (0, 0, 0, 0)
    else:
        tables, pages = block_table.shape
        Smax, sizes = 0, (slabs, rows, pages if max_pages is None else max_pages, _table(what, block_table))
    if not (q_rope.shape[:3] == shape[:3] and o.shape == shape and width == d + rope and tables >= B and seqlens_k.numel() >= B
            and (lse is None or lse.numel() >= B * H * T)):
        _shapes(what, q=q, q_rope=q_rope, cache=cache, o=o, lse=lse, seqlens_k=seqlens_k, block_table=block_table)
    # (the stride of an extent of 1 may be any number)
    p = _LATENT_DECODE.pack(q.data_ptr(), q_rope.data_ptr(), cache.data_ptr(), o.data_ptr(), 0 if lse is None else lse.data_ptr(), seqlens_k.data_ptr(),
                            0 if block_table is None else block_table.data_ptr(), qb if B > 1 else 0, qt if T > 1 else 0, qh if H > 1 else 0,
                            rb if B > 1 else 0, rt if T > 1 else 0, rh if H > 1 else 0, B, T, H, Smax, d, rope, _FA16[dt], *sizes, scale,
                            0 if workspace is None else workspace.data_ptr(), 0 if workspace is None else workspace.nbytes)
    rc = lib.fa_decode_latent(p, _stream())
    return _check(rc, what, raise_on_error) if rc else rc


def fa_decode_append_workspace_bytes(B: int, Sq: int, Hq: int, Hkv: int, Skv_max: int, d: int) -> int:
    return int(lib.fa_decode_append_workspace_bytes(B, Sq, Hq, Hkv, Skv_max, d))


def fa_decode_append(q, k_cache, v_cache, o, lse, seqlens_k, scale: float, workspace, raise_on_error: bool = True) -> int:
    """``fa_decode_append``: q, o [B,Sq,Hq,d] (the last Sq positions of every sequence), lse [B,Hq,Sq],
    caches [B,Smax,Hkv,d], seqlens_k int32 [B] on the device (lengths including the Sq new tokens)."""
    B, Sq, Hq, d = q.shape
    _, Smax, Hkv, _ = k_cache.shape
    wbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    rc = lib.fa_decode_append(_ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(o), _ptr(lse), _ptr(seqlens_k), B, Sq, Hq,
                              Hkv, Smax, d, float(scale), _ptr(workspace), wbytes, _stream())
    return _check(rc, "fa_decode_append", raise_on_error)


def fa_decode_fp8(q, k_cache, v_cache, o, lse, seqlens_k, scale: float, k_scale: float, v_scale: float, workspace,
                  raise_on_error: bool = True) -> int:
    """``fa_decode_fp8``: q [B,1,Hq,d] fp16, caches [B,Smax,Hkv,d] of FP8 e4m3 (``torch.float8_e4m3fn`` or
    uint8 bit patterns) with one factor each, seqlens_k int32 [B] on the device."""
    B, _, Hq, d = q.shape
    _, Smax, Hkv, _ = k_cache.shape
    wbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    rc = lib.fa_decode_fp8(_ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(o), _ptr(lse), _ptr(seqlens_k), B, Hq, Hkv,
                           Smax, d, float(scale), float(k_scale), float(v_scale), _ptr(workspace), wbytes, _stream())
    return _check(rc, "fa_decode_fp8", raise_on_error)


def fa_decode_fp8_bf16(q, k_cache, v_cache, o, lse, seqlens_k, scale: float, k_scale: float, v_scale: float, workspace,
                       raise_on_error: bool = True) -> int:
    """``fa_decode_fp8_bf16``: as ``fa_decode_fp8`` with q and o in bf16."""
    B, _, Hq, d = q.shape
    _, Smax, Hkv, _ = k_cache.shape
    wbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    rc = lib.fa_decode_fp8_bf16(_ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(o), _ptr(lse), _ptr(seqlens_k), B, Hq, Hkv,
                                Smax, d, float(scale), float(k_scale), float(v_scale), _ptr(workspace), wbytes, _stream())
    return _check(rc, "fa_decode_fp8_bf16", raise_on_error)


def fa_decode_fp8_paged(q, k_pages, v_pages, block_table, o, lse, seqlens_k, scale: float, k_scale: float,
                        v_scale: float, workspace, max_pages: int = None, raise_on_error: bool = True) -> int:
    """``fa_decode_fp8_paged``: as ``fa_decode_paged`` with pools of FP8 e4m3 bytes and one factor per tensor."""
    B, _, Hq, d = q.shape
    num_pages, page_size, Hkv, _ = k_pages.shape
    stride = block_table.stride(0) if block_table.dim() == 2 else block_table.numel() // max(1, B)
    if max_pages is None:
        max_pages = block_table.shape[1]
    wbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    rc = lib.fa_decode_fp8_paged(_ptr(q), _ptr(k_pages), _ptr(v_pages), _ptr(block_table), _ptr(o), _ptr(lse),
                                 _ptr(seqlens_k), B, Hq, Hkv, num_pages, page_size, int(max_pages), int(stride), d,
                                 float(scale), float(k_scale), float(v_scale), _ptr(workspace), wbytes, _stream())
    return _check(rc, "fa_decode_fp8_paged", raise_on_error)


def fa_decode_fp8_paged_bf16(q, k_pages, v_pages, block_table, o, lse, seqlens_k, scale: float, k_scale: float,
                             v_scale: float, workspace, max_pages: int = None, raise_on_error: bool = True) -> int:
    """``fa_decode_fp8_paged_bf16``: as ``fa_decode_fp8_paged`` with q and o in bf16."""
    B, _, Hq, d = q.shape
    num_pages, page_size, Hkv, _ = k_pages.shape
    stride = block_table.stride(0) if block_table.dim() == 2 else block_table.numel() // max(1, B)
    if max_pages is None:
        max_pages = block_table.shape[1]
    wbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    rc = lib.fa_decode_fp8_paged_bf16(_ptr(q), _ptr(k_pages), _ptr(v_pages), _ptr(block_table), _ptr(o), _ptr(lse),
                                      _ptr(seqlens_k), B, Hq, Hkv, num_pages, page_size, int(max_pages), int(stride), d,
                                      float(scale), float(k_scale), float(v_scale), _ptr(workspace), wbytes, _stream())
    return _check(rc, "fa_decode_fp8_paged_bf16", raise_on_error)


def fa_decode_paged(q, k_pages, v_pages, block_table, o, lse, seqlens_k, scale: float, workspace,
                    max_pages: int = None, raise_on_error: bool = True) -> int:
    """``fa_decode_paged``: q [B,1,Hq,d], page pools [num_pages,page_size,Hkv,d], block_table int32
    [B,table_stride] and seqlens_k int32 [B] on the device; workspace of at least
    ``fa_decode_workspace_bytes(B, Hq, Hkv, max_pages * page_size, d)`` bytes."""
    B, _, Hq, d = q.shape
    num_pages, page_size, Hkv, _ = k_pages.shape
    stride = block_table.stride(0) if block_table.dim() == 2 else block_table.numel() // max(1, B)
    if max_pages is None:
        max_pages = block_table.shape[1]
    wbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    rc = lib.fa_decode_paged(_ptr(q), _ptr(k_pages), _ptr(v_pages), _ptr(block_table), _ptr(o), _ptr(lse),
                             _ptr(seqlens_k), B, Hq, Hkv, num_pages, page_size, int(max_pages), int(stride), d,
                             float(scale), _ptr(workspace), wbytes, _stream())
    return _check(rc, "fa_decode_paged", raise_on_error)


def fa_decode_noalloc(q, k_cache, v_cache, o, lse, seqlens_k, scale: float, raise_on_error: bool = True) -> int:
    """``fa_decode_noalloc``: decode for callers that may not allocate device memory.  Same
    arguments as ``fa_decode`` minus the workspace; the partial results live in a fixed
    ``FA_DECODE_NOALLOC_BYTES`` array inside the library, shared by all calls (do not overlap
    two calls on the GPU).  Problems whose partials do not fit are refused with FA_ERR_WORKSPACE."""
    B, _, Hq, d = q.shape
    _, Smax, Hkv, _ = k_cache.shape
    rc = lib.fa_decode_noalloc(_ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(o), _ptr(lse), _ptr(seqlens_k), B,
                               Hq, Hkv, Smax, d, float(scale), _stream())
    return _check(rc, "fa_decode_noalloc", raise_on_error)


def fa_forward_host_staging_bytes(B, Hq, Hkv, Sq, Skv, d) -> int:
    return int(lib.fa_forward_host_staging_bytes(B, Hq, Hkv, Sq, Skv, d))


def fa_forward_host(q_host, k_host, v_host, o_host, lse_host, causal: bool, scale: float, staging,
                    raise_on_error: bool = True) -> int:
    """``fa_forward_host``: q/k/v/o/lse are HOST tensors (pinned for asynchronous copies),
    ``staging`` is a device byte tensor of at least ``fa_forward_host_staging_bytes`` bytes."""
    B, Sq, Hq, d = q_host.shape
    _, Skv, Hkv, _ = k_host.shape
    dt = FA_DTYPE_BF16 if q_host.dtype == torch.bfloat16 else FA_DTYPE_FP16
    rc = lib.fa_forward_host(_ptr(q_host), _ptr(k_host), _ptr(v_host), _ptr(o_host), _ptr(lse_host), B, Hq,
                             Hkv, Sq, Skv, d, int(bool(causal)), float(scale), dt, _ptr(staging),
                             staging.numel() * staging.element_size(), _stream())
    return _check(rc, "fa_forward_host", raise_on_error)


def fa_selftest_wait(limit_us: int, gave_up, raise_on_error: bool = True) -> int:
    """``fa_selftest_wait``: one CTA runs a bounded wait that cannot be satisfied; ``gave_up`` is a zeroed
    uint32/int32 device tensor of one element that ends up holding the number of threads that gave up."""
    rc = lib.fa_selftest_wait(int(limit_us), _ptr(gave_up), _stream())
    return _check(rc, "fa_selftest_wait", raise_on_error)


def fa_device_status():
    """Synchronises, then returns (code, where, block) of the device-side status word and clears it."""
    detail = (ctypes.c_uint * 2)(0, 0)
    rc = int(lib.fa_device_status(ctypes.byref(detail)))
    return rc, int(detail[0]), int(detail[1])


def fa_selftest_decode_cut(B: int, Sq: int, Hq: int, Hkv: int, Skv_max: int, d: int, kv8: bool = False):
    """``fa_selftest_decode_cut``: (form, chunks, tiles of the longest chunk, tiles of a chunk of form 0) of a decode of these
    sizes; form 0: chunks of one length, 1: a sequence's chunks are one cluster, 2: cut by the lengths the device finds."""
    cut = (_i * 4)()
    _check(lib.fa_selftest_decode_cut(B, Sq, Hq, Hkv, Skv_max, d, int(kv8), ctypes.byref(cut)), "fa_selftest_decode_cut", True)
    return tuple(cut)
