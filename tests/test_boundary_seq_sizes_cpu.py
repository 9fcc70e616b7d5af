"""CPU-only: calls of the sequence operators that would need a launch of 2^32 threads or more are refused before anything is enqueued."""
import ctypes

import pytest
import torch

from paper_1805_12096_amd import seq

SHAPE, G, BIG = 2, 1 << 20, 1 << 62     # a well aligned device pointer that is never dereferenced; a large workspace


def cache(kv_heads, head_dim):
    return ctypes.byref(seq._CKvCache(G, G, G, 4, kv_heads, head_dim))


def append(B, T, hk, dim, heads=0, first=G):
    q = G if heads else None
    return "mq_kv_append", (cache(hk, dim), G, 4, first, G, B, T, G, hk * dim, G, hk * dim, q, heads * dim, heads, 0, None, 0, 0, None,
                            q, None)


def cached(B, hk, heads, dim, max_len):
    return "mq_cached_attention", (cache(hk, dim), G, 1 << 20, G, B, max_len, G, heads * dim, heads, 0, 1.0, G, heads * dim, G, BIG, None)


def prompt(dtype, B, Tq, Tk, heads, hk, dim):
    return "mq_prompt_attention", (G, heads * dim, G, hk * dim, G, hk * dim, dtype, G, G, B, Tq, Tk, heads, hk, dim, 1, 1.0, G, heads * dim,
                                   G, BIG, None)


def score(M, N, K, k):
    return "mq_gemm_token_logprob_packed", (G, G, M, N, K, G, G, G, k, G, G, G, G, G, BIG, None)


CALLS = [
    append(1 << 23, 1 << 23, 8, 64),                     # a wave to a block
    append(1 << 23, 1 << 23, 8, 64, first=None),
    append(1 << 21, 1 << 21, 8, 33),                     # element by element
    append(1, 1 << 30, 1, 64),                           # four waves to a block
    append(1, 1 << 26, 1, 16, heads=1),                  # queries
    cached(1 << 23, 8, 8, 64, 64),
    cached(1 << 22, 8, 8, 64, 200),
    prompt(0, 1 << 26, 1 << 26, 1 << 26, 1, 1, 16),      # one launch
    prompt(2, 1, 1000, 1 << 29, 1, 1, 64),               # the keys' and values' packing
    prompt(0, 1, 1 << 30, 1000, 2, 2, 64),               # the attention behind it, two groups of waves
    prompt(2, 1, 1 << 30, 1000, 4, 2, 64),
    score(1 << 26, 64, 64, 4),
]


@pytest.mark.skipif(torch.cuda.is_available(), reason="the addresses are none")
@pytest.mark.parametrize("i", range(len(CALLS)))
def test_launches_that_are_none_are_refused(i):
    name, args = CALLS[i]
    assert getattr(seq._lib(), name)(*args) == SHAPE
