"""ctypes binding of the serving operators of libmq.so (include/mq_serve.h): the names and argument orders of the C entry
points, torch CUDA tensors where C takes device pointers.  Marshalling only; tensors that are not on the current device are
refused here, because the library takes plain addresses and cannot tell.
"""
from __future__ import annotations

import ctypes

import torch

from .binding import _check, load_library
from .seq import _cache, _CKvCache, _here, _p

__all__ = ["MQ_ROWS8", "exported_serve_symbols", "mq_chunk_attention_ws_bytes", "mq_chunk_attention", "mq_kv_fork_ws_bytes",
           "mq_kv_fork", "mq_kv_compact_ws_bytes", "mq_kv_compact", "mq_add_rms_norm", "mq_add_rms_norm_rows8",
           "mq_add_rms_norm_pack8", "mq_w4_bytes", "mq_w4_pack", "mq_w4_prepare", "mq_w4_unpack", "mq_w4_product_ws_bytes",
           "mq_w4_product", "w4_pack", "w4_prepare"]

MQ_ROWS8 = 3


def exported_serve_symbols():
    """Names include/mq_serve.h declares; used by the CPU-only load test."""
    return ["mq_chunk_attention_ws_bytes", "mq_chunk_attention", "mq_kv_fork_ws_bytes", "mq_kv_fork", "mq_kv_compact_ws_bytes",
            "mq_kv_compact", "mq_add_rms_norm", "mq_add_rms_norm_rows8", "mq_add_rms_norm_pack8", "mq_w4_bytes", "mq_w4_pack",
            "mq_w4_prepare", "mq_w4_unpack", "mq_w4_product_ws_bytes", "mq_w4_product"]


_declared = None


def _lib():
    global _declared
    lib = load_library()
    if _declared is lib:
        return lib
    vp, sz, ci, cf = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int, ctypes.c_float
    cache = ctypes.POINTER(_CKvCache)
    for name, args in (("mq_chunk_attention_ws_bytes", [sz, sz, sz, ci, ci, sz]), ("mq_kv_fork_ws_bytes", [sz, sz, sz]),
                       ("mq_kv_compact_ws_bytes", [sz]), ("mq_w4_bytes", [sz, sz, ci]), ("mq_w4_product_ws_bytes", [sz, sz, sz])):
        getattr(lib, name).restype, getattr(lib, name).argtypes = sz, args
    lib.mq_chunk_attention.argtypes = [cache, vp, sz, vp, vp, sz, sz, sz, ci, vp, sz, ci, ci, cf, vp, sz, vp, sz, vp]
    lib.mq_kv_fork.argtypes = [cache, vp, vp, sz, vp, sz, vp, vp, sz, vp, vp, vp, vp, sz, vp]
    lib.mq_kv_compact.argtypes = [cache, vp, vp, sz, vp, sz, vp, vp, vp, vp, sz, vp]
    lib.mq_add_rms_norm.argtypes = [vp, sz, vp, sz, ci, vp, sz, sz, cf, vp, sz, vp, sz, vp]
    lib.mq_add_rms_norm_rows8.argtypes = [vp, sz, vp, sz, ci, vp, sz, sz, cf, vp, sz, vp, sz, vp, vp]
    lib.mq_add_rms_norm_pack8.argtypes = [vp, sz, vp, sz, ci, vp, sz, sz, cf, vp, sz, vp, vp, vp]
    lib.mq_w4_pack.argtypes = [vp, vp, vp, sz, sz, ci, vp, vp]
    lib.mq_w4_prepare.argtypes = [vp, sz, sz, ci, vp, vp]
    lib.mq_w4_unpack.argtypes = [vp, sz, sz, ci, vp, vp]
    lib.mq_w4_product.argtypes = [vp, sz, ci, vp, vp, sz, sz, sz, ci, vp, vp, sz, ci, vp, sz, vp]
    _declared = lib
    return lib


def mq_chunk_attention_ws_bytes(B, T, max_len, heads, kv_heads, head_dim) -> int:
    return int(_lib().mq_chunk_attention_ws_bytes(B, T, max_len, heads, kv_heads, head_dim))


def mq_chunk_attention(cache, table, table_width, first, lens, B, T, max_len, causal, q, ldq, heads, dtype, scale, out, ldo, ws,
                       ws_bytes, stream=None):
    """cache: a KvCache; everything else as in include/mq_serve.h."""
    c, at = _here(stream)
    _check(_lib().mq_chunk_attention(_cache(cache, c), _p(table, c), table_width, _p(first, c), _p(lens, c), B, T, max_len,
                                     int(causal), _p(q, c), ldq, heads, dtype, scale, _p(out, c), ldo, _p(ws, c), ws_bytes, at),
           "mq_chunk_attention")


def mq_kv_fork_ws_bytes(blocks, B_new, table_width) -> int:
    return int(_lib().mq_kv_fork_ws_bytes(blocks, B_new, table_width))


def mq_kv_fork(cache, keep, table, table_width, lens, B, parent, grow, B_new, table_new, lens_new, missing, ws, ws_bytes, stream=None):
    """cache: a KvCache; everything else as in include/mq_serve.h."""
    c, at = _here(stream)
    _check(_lib().mq_kv_fork(_cache(cache, c), _p(keep, c), _p(table, c), table_width, _p(lens, c), B, _p(parent, c), _p(grow, c), B_new,
                             _p(table_new, c), _p(lens_new, c), _p(missing, c), _p(ws, c), ws_bytes, at), "mq_kv_fork")


def mq_kv_compact_ws_bytes(blocks) -> int:
    return int(_lib().mq_kv_compact_ws_bytes(blocks))


def mq_kv_compact(cache, keep, table, table_width, lens, B, table_new, moved, used, ws, ws_bytes, stream=None):
    """cache: a KvCache; everything else as in include/mq_serve.h."""
    c, at = _here(stream)
    _check(_lib().mq_kv_compact(_cache(cache, c), _p(keep, c), _p(table, c), table_width, _p(lens, c), B, _p(table_new, c), _p(moved, c),
                                _p(used, c), _p(ws, c), ws_bytes, at), "mq_kv_compact")


def mq_add_rms_norm(x, ldx, r, ldr, dtype, gamma, M, d, eps, h, ldh, y, ldy, stream=None):
    c, at = _here(stream)
    _check(_lib().mq_add_rms_norm(_p(x, c), ldx, _p(r, c), ldr, dtype, _p(gamma, c), M, d, eps, _p(h, c), ldh, _p(y, c), ldy, at),
           "mq_add_rms_norm")


def mq_add_rms_norm_rows8(x, ldx, r, ldr, dtype, gamma, M, d, eps, h, ldh, q, ldq, scale, stream=None):
    c, at = _here(stream)
    _check(_lib().mq_add_rms_norm_rows8(_p(x, c), ldx, _p(r, c), ldr, dtype, _p(gamma, c), M, d, eps, _p(h, c), ldh, _p(q, c), ldq,
                                        _p(scale, c), at), "mq_add_rms_norm_rows8")


def mq_add_rms_norm_pack8(x, ldx, r, ldr, dtype, gamma, M, d, eps, h, ldh, s, packed, stream=None):
    c, at = _here(stream)
    _check(_lib().mq_add_rms_norm_pack8(_p(x, c), ldx, _p(r, c), ldr, dtype, _p(gamma, c), M, d, eps, _p(h, c), ldh, _p(s, c),
                                        _p(packed, c), at), "mq_add_rms_norm_pack8")


def mq_w4_bytes(N, K, group) -> int:
    return int(_lib().mq_w4_bytes(N, K, group))


def mq_w4_pack(codes, scales, zeros, N, K, group, packed, stream=None):
    c, at = _here(stream)
    _check(_lib().mq_w4_pack(_p(codes, c), _p(scales, c), _p(zeros, c), N, K, group, _p(packed, c), at), "mq_w4_pack")


def mq_w4_prepare(w, N, K, group, packed, stream=None):
    c, at = _here(stream)
    _check(_lib().mq_w4_prepare(_p(w, c), N, K, group, _p(packed, c), at), "mq_w4_prepare")


def mq_w4_unpack(packed, N, K, group, w, stream=None):
    c, at = _here(stream)
    _check(_lib().mq_w4_unpack(_p(packed, c), N, K, group, _p(w, c), at), "mq_w4_unpack")


def mq_w4_product_ws_bytes(M, N, K) -> int:
    return int(_lib().mq_w4_product_ws_bytes(M, N, K))


def mq_w4_product(x, ldx, xtype, row_scale, packed, M, N, K, group, bias, y, ldy, ytype, ws, ws_bytes, stream=None):
    c, at = _here(stream)
    _check(_lib().mq_w4_product(_p(x, c), ldx, xtype, _p(row_scale, c), _p(packed, c), M, N, K, group, _p(bias, c), _p(y, c), ldy,
                                ytype, _p(ws, c), ws_bytes, at), "mq_w4_product")


def _packed4(N, K, group, device):
    size = mq_w4_bytes(N, K, group)
    if size == 0:
        raise ValueError(f"no packed parameter of {N} x {K} elements in groups of {group}")
    return torch.empty(size, dtype=torch.uint8, device=device)


def w4_pack(codes: torch.Tensor, scales: torch.Tensor, zeros, group: int, stream=None) -> torch.Tensor:
    """Allocate and fill the packed form of codes uint8 [N, K], scales float32 and zeros uint8 (or None) [N, groups]."""
    N, K = codes.shape
    groups = -(-K // group) if group > 0 else 0
    if codes.dtype != torch.uint8 or scales.dtype != torch.float32 or (zeros is not None and zeros.dtype != torch.uint8):
        raise ValueError("codes and zeros are uint8, scales float32")
    if tuple(scales.shape) != (N, groups) or (zeros is not None and tuple(zeros.shape) != (N, groups)):
        raise ValueError(f"scales and zeros are [{N}, {groups}]")
    if not (codes.is_contiguous() and scales.is_contiguous() and (zeros is None or zeros.is_contiguous())):
        raise ValueError("codes, scales and zeros are contiguous")
    packed = _packed4(N, K, group, codes.device)
    mq_w4_pack(codes, scales, zeros, N, K, group, packed, stream)
    return packed


def w4_prepare(w: torch.Tensor, group: int, stream=None) -> torch.Tensor:
    """Allocate and fill the packed form of a float32 parameter [N, K]."""
    if w.dtype != torch.float32 or not w.is_contiguous():
        raise ValueError("a parameter is float32 and contiguous")
    N, K = w.shape
    packed = _packed4(N, K, group, w.device)
    mq_w4_prepare(w, N, K, group, packed, stream)
    return packed
