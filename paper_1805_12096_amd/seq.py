"""ctypes binding of the sequence operators of libmq.so (include/mq_seq.h): the names and argument orders of the C entry
points, torch CUDA tensors where C takes device pointers.  Marshalling only; tensors that are not on the current device are
refused here, because the library takes plain addresses and cannot tell.
"""
from __future__ import annotations

import ctypes

import torch

from . import binding
from .binding import _check, _stream, load_library

__all__ = ["MQ_F32", "MQ_F16", "MQ_BF16", "MQ_KV_BLOCK", "KvCache", "kv_cache", "dtype_code", "exported_seq_symbols",
           "mq_kv_key_bytes", "mq_kv_value_bytes", "mq_kv_append", "mq_cached_attention_ws_bytes", "mq_cached_attention",
           "mq_prompt_attention_ws_bytes", "mq_prompt_attention", "mq_token_logprob_ws_bytes", "mq_gemm_token_logprob_packed"]

MQ_F32, MQ_F16, MQ_BF16 = 0, 1, 2
MQ_KV_BLOCK = 64
_CODES = {torch.float32: MQ_F32, torch.float16: MQ_F16, torch.bfloat16: MQ_BF16}


class _CKvCache(ctypes.Structure):
    _fields_ = [("keys", ctypes.c_void_p), ("values", ctypes.c_void_p), ("amax", ctypes.c_void_p), ("blocks", ctypes.c_size_t),
                ("kv_heads", ctypes.c_int), ("head_dim", ctypes.c_size_t)]


def exported_seq_symbols():
    """Names include/mq_seq.h declares; used by the CPU-only load test."""
    return ["mq_kv_key_bytes", "mq_kv_value_bytes", "mq_kv_append", "mq_cached_attention_ws_bytes", "mq_cached_attention",
            "mq_prompt_attention_ws_bytes", "mq_prompt_attention", "mq_token_logprob_ws_bytes", "mq_gemm_token_logprob_packed"]


_declared = None


def _lib():
    global _declared
    lib = load_library()
    if _declared is lib:
        return lib
    vp, sz, ci, cf = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int, ctypes.c_float
    cache = ctypes.POINTER(_CKvCache)
    for name in ("mq_kv_key_bytes", "mq_kv_value_bytes"):
        getattr(lib, name).restype, getattr(lib, name).argtypes = sz, [sz, ci, sz]
    lib.mq_kv_append.argtypes = [cache, vp, sz, vp, vp, sz, sz, vp, sz, vp, sz, vp, sz, ci, ci, vp, sz, ci, vp, vp, vp]
    lib.mq_cached_attention_ws_bytes.restype = sz
    lib.mq_cached_attention_ws_bytes.argtypes = [sz, sz, ci, ci, sz]
    lib.mq_cached_attention.argtypes = [cache, vp, sz, vp, sz, sz, vp, sz, ci, ci, cf, vp, sz, vp, sz, vp]
    lib.mq_prompt_attention_ws_bytes.restype = sz
    lib.mq_prompt_attention_ws_bytes.argtypes = [ci, sz, sz, ci, sz]
    lib.mq_prompt_attention.argtypes = [vp, sz, vp, sz, vp, sz, ci, vp, vp, sz, sz, sz, ci, ci, sz, ci, cf, vp, sz, vp, sz, vp]
    lib.mq_token_logprob_ws_bytes.restype = sz
    lib.mq_token_logprob_ws_bytes.argtypes = [sz, sz, ci]
    lib.mq_gemm_token_logprob_packed.argtypes = [vp, vp, sz, sz, sz, vp, vp, vp, ci, vp, vp, vp, vp, vp, sz, vp]
    _declared = lib
    return lib


def _p(t, current=-2):
    """Device address of a tensor on the current device (None -> NULL); raw ints pass through."""
    if t is None or isinstance(t, int):
        return t
    if t.get_device() != current:                    # (-1 for host memory)
        raise ValueError(f"a tensor on {t.device} was passed: the library takes memory of the current device")
    return t.data_ptr()


def _here(stream):
    """The current device (-2, where no tensor is, while nothing has touched a device yet) and the stream's handle, asked for
    once a call: a decode-sized call's host time shows."""
    if not torch.cuda.is_initialized():
        return -2, 0 if stream is None else _stream(stream)
    if binding._device is None or binding._raw_stream is None:
        return torch.cuda.current_device(), _stream(stream)
    current = binding._device()
    return current, binding._raw_stream(current) if stream is None else _stream(stream)


def dtype_code(dtype: torch.dtype) -> int:
    """The mq_dtype of a torch type."""
    if dtype not in _CODES:
        raise ValueError(f"{dtype} is none of float32, float16, bfloat16")
    return _CODES[dtype]


class KvCache:
    """The C struct of a cache plus the tensors that keep its device memory alive (layout: include/mq_seq.h)."""

    def __init__(self, keys: torch.Tensor, values: torch.Tensor, amax: torch.Tensor, blocks: int, kv_heads: int, head_dim: int):
        if keys.dtype != torch.int8 or values.dtype != torch.int8 or amax.dtype != torch.float32:
            raise ValueError("keys and values are int8, amax is float32")
        if not (keys.is_contiguous() and values.is_contiguous() and amax.is_contiguous()):
            raise ValueError("a cache is contiguous")
        if (keys.numel() != mq_kv_key_bytes(blocks, kv_heads, head_dim) or keys.numel() == 0
                or values.numel() != mq_kv_value_bytes(blocks, kv_heads, head_dim) or amax.numel() != 2 * blocks * kv_heads):
            raise ValueError("tensors do not have the sizes of a cache of that many blocks and heads")
        self.keys, self.values, self.amax = keys, values, amax
        self.blocks, self.kv_heads, self.head_dim = blocks, kv_heads, head_dim
        self.device = keys.get_device() if keys.is_cuda and values.device == keys.device == amax.device else -1
        self.c = _CKvCache(keys.data_ptr(), values.data_ptr(), amax.data_ptr(), blocks, kv_heads, head_dim)


def kv_cache(blocks: int, kv_heads: int, head_dim: int, device="cuda") -> KvCache:
    """Allocate a cache of `blocks` blocks of MQ_KV_BLOCK tokens (all zero)."""
    dk, dv = -(-head_dim // 64) * 64, -(-head_dim // 16) * 16
    return KvCache(torch.zeros((blocks, kv_heads, MQ_KV_BLOCK, dk), dtype=torch.int8, device=device),
                   torch.zeros((blocks, kv_heads, dv, MQ_KV_BLOCK), dtype=torch.int8, device=device),
                   torch.zeros((blocks, kv_heads, 2), dtype=torch.float32, device=device), blocks, kv_heads, head_dim)


def _cache(cache, current):
    if cache.device != current:
        raise ValueError("a cache that is not on the current device")
    return ctypes.byref(cache.c)


def mq_kv_key_bytes(blocks, kv_heads, head_dim) -> int:
    return int(_lib().mq_kv_key_bytes(blocks, kv_heads, head_dim))


def mq_kv_value_bytes(blocks, kv_heads, head_dim) -> int:
    return int(_lib().mq_kv_value_bytes(blocks, kv_heads, head_dim))


def mq_kv_append(cache, table, table_width, first, held, B, T, k, ldk, v, ldv, q, ldq, heads, dtype, freq, rot, interleaved,
                 k_out=None, q_out=None, stream=None):
    """cache: a KvCache; everything else as in include/mq_seq.h."""
    c, at = _here(stream)
    _check(_lib().mq_kv_append(_cache(cache, c), _p(table, c), table_width, _p(first, c), _p(held, c), B, T, _p(k, c), ldk,
                               _p(v, c), ldv, _p(q, c), ldq, heads, dtype, _p(freq, c), rot, int(interleaved), _p(k_out, c),
                               _p(q_out, c), at), "mq_kv_append")


def mq_cached_attention_ws_bytes(B, max_len, heads, kv_heads, head_dim) -> int:
    return int(_lib().mq_cached_attention_ws_bytes(B, max_len, heads, kv_heads, head_dim))


def mq_cached_attention(cache, table, table_width, lens, B, max_len, q, ldq, heads, dtype, scale, out, ldo, ws, ws_bytes,
                        stream=None):
    """cache: a KvCache; everything else as in include/mq_seq.h."""
    c, at = _here(stream)
    _check(_lib().mq_cached_attention(_cache(cache, c), _p(table, c), table_width, _p(lens, c), B, max_len, _p(q, c), ldq, heads,
                                      dtype, scale, _p(out, c), ldo, _p(ws, c), ws_bytes, at),
           "mq_cached_attention")


def mq_prompt_attention_ws_bytes(dtype, B, Tk, kv_heads, head_dim) -> int:
    return int(_lib().mq_prompt_attention_ws_bytes(dtype, B, Tk, kv_heads, head_dim))


def mq_prompt_attention(q, ldq, k, ldk, v, ldv, dtype, q_first, k_first, B, Tq, Tk, heads, kv_heads, head_dim, causal, scale,
                        out, ldo, ws, ws_bytes, stream=None):
    c, at = _here(stream)
    _check(_lib().mq_prompt_attention(_p(q, c), ldq, _p(k, c), ldk, _p(v, c), ldv, dtype, _p(q_first, c), _p(k_first, c), B, Tq,
                                      Tk, heads, kv_heads, head_dim, int(causal), scale, _p(out, c), ldo, _p(ws, c), ws_bytes,
                                      at), "mq_prompt_attention")


def mq_token_logprob_ws_bytes(M, N, k) -> int:
    return int(_lib().mq_token_logprob_ws_bytes(M, N, int(k)))


def mq_gemm_token_logprob_packed(packedA, packedW, M, N, K, sA, sW, target, k, logprob, entropy, tok, alt_logprob, ws, ws_bytes,
                                 stream=None):
    c, at = _here(stream)
    _check(_lib().mq_gemm_token_logprob_packed(_p(packedA, c), _p(packedW, c), M, N, K, _p(sA, c), _p(sW, c), _p(target, c),
                                               int(k), _p(logprob, c), _p(entropy, c), _p(tok, c), _p(alt_logprob, c), _p(ws, c),
                                               ws_bytes, at), "mq_gemm_token_logprob_packed")
