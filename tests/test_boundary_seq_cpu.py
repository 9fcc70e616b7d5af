"""CPU-only checks of the sequence operators' boundary (include/mq_seq.h): symbols, sizes, refusals before anything is enqueued."""
import ctypes
import os
import re

import pytest
import torch

import paper_1805_12096_amd as mq
from paper_1805_12096_amd import seq

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NULL, SHAPE, DTYPE, ALIGN, WS, UNSUP = 1, 2, 3, 4, 5, 6
G, BIG = 1 << 20, 1 << 40          # a well aligned device pointer that is never dereferenced; a large workspace


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(mq.lib_path()):
        from paper_1805_12096_amd import build
        build.build()
    return seq._lib()


def test_header_symbols_are_exported(lib):
    header = open(os.path.join(ROOT, "include", "mq_seq.h")).read()
    body = re.sub(r"/\*.*?\*/", "", header, flags=re.S)
    declared = set(re.findall(r"\b(mq_[a-z0-9_]+)\s*\(", body))
    assert declared == set(mq.exported_seq_symbols())
    for name in declared:
        assert hasattr(lib, name), name
        assert callable(getattr(mq, name)), name


def test_size_queries(lib):
    assert mq.mq_kv_key_bytes(3, 2, 80) == 3 * 2 * 64 * 128
    assert mq.mq_kv_value_bytes(3, 2, 80) == 3 * 2 * 64 * 80
    assert mq.mq_kv_value_bytes(3, 2, 33) == 3 * 2 * 64 * 48
    # past 32 bits
    assert mq.mq_kv_key_bytes(1 << 20, 8, 128) == (1 << 20) * 8 * 64 * 128
    for bad in ((0, 1, 64), (1, 0, 64), (1, 1, 0), (1, 1, 257), (1 << 31, 1, 64), (1, 1025, 64)):
        assert mq.mq_kv_key_bytes(*bad) == 0 and mq.mq_kv_value_bytes(*bad) == 0
    assert mq.mq_cached_attention_ws_bytes(4, 1000, 8, 8, 64) > 0
    for bad in ((0, 1, 8, 8, 64), (1, 0, 8, 8, 64), (1, 1, 8, 3, 64), (1, 1, 0, 1, 64), (1, 1, 8, 8, 300)):
        assert mq.mq_cached_attention_ws_bytes(*bad) == 0
    assert mq.mq_prompt_attention_ws_bytes(mq.MQ_F32, 2, 100, 4, 64) > mq.mq_prompt_attention_ws_bytes(mq.MQ_BF16, 2, 100, 4, 64)
    # every sequence may end inside a unit: one token each takes as many units as there are sequences
    assert mq.mq_prompt_attention_ws_bytes(mq.MQ_BF16, 100, 100, 1, 32) >= 100 * 32 * 32 * 2 * 2
    for bad in ((3, 1, 1, 1, 64), (0, 0, 1, 1, 64), (0, 1, 0, 1, 64), (0, 1, 1, 0, 64), (0, 1, 1, 1, 0)):
        assert mq.mq_prompt_attention_ws_bytes(*bad) == 0
    assert mq.mq_token_logprob_ws_bytes(5, 1000, 4) > 0
    for bad in ((0, 5, 0), (5, 0, 0), (5, 5, -1), (5, 5, 9)):
        assert mq.mq_token_logprob_ws_bytes(*bad) == 0


def _cache(keys=G, values=G, amax=G, blocks=4, kv_heads=2, head_dim=64):
    return ctypes.byref(seq._CKvCache(keys, values, amax, blocks, kv_heads, head_dim))


# name -> valid arguments by name (None of the calls with them is made), in the order of the C entry point
def _valid():
    return {
        "mq_kv_append": dict(cache=_cache(), table=G, table_width=4, first=G, held=G, B=3, T=9, k=G, ldk=128, v=G, ldv=128, q=G,
                             ldq=256, heads=4, dtype=0, freq=G, rot=64, interleaved=0, k_out=G, q_out=G, stream=None),
        "mq_cached_attention": dict(cache=_cache(), table=G, table_width=4, lens=G, B=3, max_len=256, q=G, ldq=256, heads=4,
                                    dtype=0, scale=0.125, out=G, ldo=256, ws=G, ws_bytes=BIG, stream=None),
        "mq_prompt_attention": dict(q=G, ldq=256, k=G, ldk=128, v=G, ldv=128, dtype=0, q_first=G, k_first=G, B=3, Tq=9, Tk=9,
                                    heads=4, kv_heads=2, head_dim=64, causal=1, scale=0.125, out=G, ldo=256, ws=G,
                                    ws_bytes=BIG, stream=None),
        "mq_gemm_token_logprob_packed": dict(packedA=G, packedW=G, M=4, N=16, K=64, sA=G, sW=G, target=G, k=2, logprob=G,
                                             entropy=G, tok=G, alt_logprob=G, ws=G, ws_bytes=BIG, stream=None),
    }


CACHE_REFUSALS = [(dict(cache=None), NULL), (dict(table=None), NULL), (dict(keys=None), NULL), (dict(values=None), NULL),
                  (dict(amax=None), NULL), (dict(blocks=0), SHAPE), (dict(blocks=1 << 31), SHAPE), (dict(kv_heads=0), SHAPE),
                  (dict(kv_heads=-1), SHAPE), (dict(head_dim=0), SHAPE), (dict(head_dim=257), SHAPE), (dict(kv_heads=3), SHAPE),
                  (dict(table_width=0), SHAPE), (dict(keys=G + 8), ALIGN), (dict(values=G + 4), ALIGN), (dict(amax=G + 4), ALIGN),
                  (dict(table=G + 2), ALIGN), (dict(dtype=3), DTYPE), (dict(dtype=-1), DTYPE), (dict(B=0), SHAPE),
                  (dict(B=(1 << 30) + 1), SHAPE), (dict(heads=0), SHAPE), (dict(heads=5), SHAPE), (dict(heads=2048), SHAPE),
                  (dict(ldq=255), SHAPE), (dict(q=G + 2), ALIGN), (dict(ldq=1 << 41), SHAPE)]
REFUSALS = {
    "mq_kv_append": CACHE_REFUSALS + [
        (dict(held=None), NULL), (dict(k=None), NULL), (dict(v=None), NULL), (dict(q=None), NULL), (dict(q_out=None), NULL),
        (dict(freq=None), NULL), (dict(T=0), SHAPE), (dict(first=None), SHAPE), (dict(rot=63), SHAPE), (dict(rot=66), SHAPE),
        (dict(ldk=127), SHAPE), (dict(ldv=127), SHAPE), (dict(held=G + 1), ALIGN), (dict(first=G + 2), ALIGN),
        (dict(k=G + 2), ALIGN), (dict(v=G + 1), ALIGN), (dict(k_out=G + 2), ALIGN), (dict(q_out=G + 2), ALIGN),
        (dict(freq=G + 2), ALIGN), (dict(dtype=1, v=G + 1), ALIGN)],
    "mq_cached_attention": CACHE_REFUSALS + [
        (dict(lens=None), NULL), (dict(q=None), NULL), (dict(out=None), NULL), (dict(ws=None), NULL), (dict(max_len=0), SHAPE),
        (dict(max_len=257), SHAPE), (dict(ldo=255), SHAPE), (dict(lens=G + 2), ALIGN), (dict(out=G + 2), ALIGN),
        (dict(ws=G + 8), ALIGN), (dict(ws_bytes=15), WS)],
    "mq_prompt_attention": [
        (dict(dtype=7), DTYPE), (dict(q=None), NULL), (dict(k=None), NULL), (dict(v=None), NULL), (dict(q_first=None), NULL),
        (dict(k_first=None), NULL), (dict(out=None), NULL), (dict(ws=None), NULL), (dict(B=0), SHAPE), (dict(Tq=0), SHAPE),
        (dict(Tk=0), SHAPE), (dict(heads=3), SHAPE), (dict(kv_heads=0), SHAPE), (dict(head_dim=0), SHAPE),
        (dict(head_dim=257, ldq=2000, ldk=2000, ldv=2000, ldo=2000), SHAPE), (dict(ldq=255), SHAPE), (dict(ldk=127), SHAPE),
        (dict(ldv=127), SHAPE), (dict(ldo=255), SHAPE), (dict(Tq=(1 << 30) + 1), SHAPE), (dict(q=G + 2), ALIGN),
        (dict(k=G + 2), ALIGN), (dict(v=G + 2), ALIGN), (dict(out=G + 2), ALIGN), (dict(q_first=G + 2), ALIGN),
        (dict(k_first=G + 1), ALIGN), (dict(ws=G + 128), ALIGN), (dict(ws_bytes=1000), WS)],
    "mq_gemm_token_logprob_packed": [
        (dict(packedA=None), NULL), (dict(packedW=None), NULL), (dict(sA=None), NULL), (dict(sW=None), NULL),
        (dict(target=None), NULL), (dict(logprob=None), NULL), (dict(ws=None), NULL), (dict(tok=None), NULL),
        (dict(alt_logprob=None), NULL), (dict(M=0), SHAPE), (dict(N=0), SHAPE), (dict(K=0), SHAPE), (dict(k=-1), SHAPE),
        (dict(k=9), SHAPE), (dict(k=8, N=7), SHAPE), (dict(M=1 << 30, N=1 << 20), SHAPE), (dict(K=1025), UNSUP),
        (dict(N=(1 << 24) + 1), UNSUP), (dict(packedA=G + 8), ALIGN), (dict(packedW=G + 8), ALIGN), (dict(sA=G + 2), ALIGN),
        (dict(sW=G + 2), ALIGN), (dict(target=G + 2), ALIGN), (dict(logprob=G + 2), ALIGN), (dict(entropy=G + 1), ALIGN),
        (dict(tok=G + 2), ALIGN), (dict(alt_logprob=G + 2), ALIGN), (dict(ws=G + 8), ALIGN), (dict(ws_bytes=16), WS)],
}


@pytest.mark.parametrize("name", sorted(REFUSALS))
def test_bad_arguments_are_refused(lib, name):
    inside = ("keys", "values", "amax", "blocks", "kv_heads", "head_dim")
    for change, status in REFUSALS[name]:
        args = _valid()[name]
        in_cache = {k: v for k, v in change.items() if "cache" in args and k in inside}
        if in_cache:
            args["cache"] = _cache(**in_cache)
        args.update({k: v for k, v in change.items() if k not in in_cache})
        assert set(args) == set(_valid()[name]), change
        assert getattr(lib, name)(*args.values()) == status, change


def test_every_entry_point_has_refusals():
    queries = {n for n in mq.exported_seq_symbols() if n.endswith("_bytes")}
    assert set(REFUSALS) | queries == set(mq.exported_seq_symbols())


def test_binding_refuses_host_tensors_and_other_types(lib):
    x = torch.zeros(64)
    with pytest.raises(ValueError):
        seq._p(x)
    assert seq._p(None) is None and seq._p(7) == 7
    assert [mq.dtype_code(t) for t in (torch.float32, torch.float16, torch.bfloat16)] == [0, 1, 2]
    with pytest.raises(ValueError):
        mq.dtype_code(torch.float64)
    k, v, a = torch.zeros((2, 1, 64, 64), dtype=torch.int8), torch.zeros((2, 1, 48, 64), dtype=torch.int8), torch.zeros((2, 1, 2))
    cache = mq.KvCache(k, v, a, 2, 1, 40)
    with pytest.raises(ValueError):
        mq.mq_kv_append(cache, G, 1, None, G, 1, 1, G, 40, G, 40, None, 0, 1, 0, None, 0, False)
    for bad in ((k, v, a, 3, 1, 40), (k, v, a, 2, 1, 64), (k, v[:1], a, 2, 1, 40), (k.float(), v, a, 2, 1, 40), (k, v, a.half(), 2, 1, 40),
                (k.transpose(2, 3), v, a, 2, 1, 40), (k, v, a, 0, 1, 40)):
        with pytest.raises(ValueError):
            mq.KvCache(*bad)
