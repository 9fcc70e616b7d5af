"""CPU-only checks of the serving operators' boundary (include/mq_serve.h): symbols, sizes, refusals before anything is enqueued."""
import ctypes
import os
import re

import pytest
import torch

import paper_1805_12096_amd as mq
from paper_1805_12096_amd import seq, serve

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NULL, SHAPE, DTYPE, ALIGN, WS = 1, 2, 3, 4, 5
G, BIG = 1 << 20, 1 << 50          # a well aligned device pointer that is never dereferenced; a large workspace


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(mq.lib_path()):
        from paper_1805_12096_amd import build
        build.build()
    return serve._lib()


def test_header_symbols_are_exported(lib):
    header = open(os.path.join(ROOT, "include", "mq_serve.h")).read()
    body = re.sub(r"/\*.*?\*/", "", header, flags=re.S)
    declared = set(re.findall(r"\b(mq_[a-z0-9_]+)\s*\(", body))
    assert declared == set(mq.exported_serve_symbols())
    for name in declared:
        assert hasattr(lib, name), name
        assert callable(getattr(mq, name)), name


def test_size_queries(lib):
    assert mq.mq_chunk_attention_ws_bytes(4, 9, 1000, 8, 8, 64) > 0
    for bad in ((0, 9, 9, 8, 8, 64), (1, 0, 9, 8, 8, 64), (1, 9, 0, 8, 8, 64), (1, 9, 9, 8, 3, 64), (1, 9, 9, 0, 1, 64), (1, 9, 9, 8, 8, 257),
                (1, (1 << 30) + 1, 9, 8, 8, 64)):
        assert mq.mq_chunk_attention_ws_bytes(*bad) == 0, bad
    assert mq.mq_kv_fork_ws_bytes(100, 5, 3) > 0 and mq.mq_kv_compact_ws_bytes(100) > 0
    for bad in ((0, 5, 3), (100, 0, 3), (100, 5, 0), (1 << 30, 5, 3), (100, (1 << 30) + 1, 3)):
        assert mq.mq_kv_fork_ws_bytes(*bad) == 0, bad
    assert mq.mq_kv_compact_ws_bytes(0) == 0 and mq.mq_kv_compact_ws_bytes(1 << 30) == 0
    # four bits an element, a word for each group of a row, in tiles of 16 rows x 128 elements
    assert mq.mq_w4_bytes(16, 128, 128) == 1024 + 64
    assert mq.mq_w4_bytes(17, 129, 32) == 4 * 1024 + 2 * 8 * 64
    assert mq.mq_w4_bytes(1 << 20, 1 << 14, 64) == (1 << 33) + (1 << 30)            # past 32 bits
    for bad in ((0, 5, 32), (5, 0, 32), (5, 5, 0), (5, 5, 16), (5, 5, 96), (5, 5, -32), ((1 << 24) + 1, 5, 32), (5, (1 << 24) + 1, 32),
                (1 << 22, 1 << 22, 32)):
        assert mq.mq_w4_bytes(*bad) == 0, bad
    assert mq.mq_w4_product_ws_bytes(3, 100, 100) > 0
    for bad in ((0, 5, 5), (5, 0, 5), (5, 5, 0), (1 << 30, 1 << 20, 5), (1 << 30, 5, 1 << 20)):
        assert mq.mq_w4_product_ws_bytes(*bad) == 0, bad


def _cache(keys=G, values=G, amax=G, blocks=4, kv_heads=2, head_dim=64):
    return ctypes.byref(seq._CKvCache(keys, values, amax, blocks, kv_heads, head_dim))


NORM = dict(x=G, ldx=64, r=G, ldr=64, dtype=0, gamma=G, M=3, d=64, eps=1e-6, h=G, ldh=64)


# name -> valid arguments by name (None of the calls with them is made), in the order of the C entry point
def _valid():
    return {
        "mq_chunk_attention": dict(cache=_cache(), table=G, table_width=4, first=G, lens=G, B=3, T=9, max_len=256, causal=1, q=G,
                                   ldq=256, heads=4, dtype=0, scale=0.125, out=G, ldo=256, ws=G, ws_bytes=BIG, stream=None),
        "mq_kv_fork": dict(cache=_cache(), keep=G, table=G, table_width=4, lens=G, B=3, parent=G, grow=G, B_new=5, table_new=G,
                           lens_new=G, missing=G, ws=G, ws_bytes=BIG, stream=None),
        "mq_kv_compact": dict(cache=_cache(), keep=G, table=G, table_width=4, lens=G, B=3, table_new=G, moved=G, used=G, ws=G,
                              ws_bytes=BIG, stream=None),
        "mq_add_rms_norm": dict(**NORM, y=G, ldy=64, stream=None),
        "mq_add_rms_norm_rows8": dict(**NORM, q=G, ldq=64, scale=G, stream=None),
        "mq_add_rms_norm_pack8": dict(**NORM, s=G, packed=G, stream=None),
        "mq_w4_pack": dict(codes=G, scales=G, zeros=G, N=5, K=70, group=32, packed=G, stream=None),
        "mq_w4_prepare": dict(w=G, N=5, K=70, group=32, packed=G, stream=None),
        "mq_w4_unpack": dict(packed=G, N=5, K=70, group=32, w=G, stream=None),
        "mq_w4_product": dict(x=G, ldx=70, xtype=0, row_scale=None, packed=G, M=3, N=5, K=70, group=32, bias=G, y=G, ldy=5, ytype=0,
                              ws=G, ws_bytes=BIG, stream=None),
    }


CACHE_REFUSALS = [(dict(cache=None), NULL), (dict(table=None), NULL), (dict(keys=None), NULL), (dict(values=None), NULL),
                  (dict(amax=None), NULL), (dict(blocks=0), SHAPE), (dict(blocks=1 << 31), SHAPE), (dict(kv_heads=0), SHAPE),
                  (dict(kv_heads=-1), SHAPE), (dict(head_dim=0), SHAPE), (dict(head_dim=257), SHAPE), (dict(table_width=0), SHAPE),
                  (dict(keys=G + 8), ALIGN), (dict(values=G + 4), ALIGN), (dict(amax=G + 4), ALIGN), (dict(table=G + 2), ALIGN),
                  (dict(B=0), SHAPE), (dict(B=(1 << 30) + 1), SHAPE), (dict(lens=None), NULL), (dict(ws=None), NULL),
                  (dict(lens=G + 2), ALIGN), (dict(ws=G + 8), ALIGN), (dict(ws_bytes=4), WS)]
TABLE_REFUSALS = CACHE_REFUSALS + [(dict(blocks=1 << 30), SHAPE), (dict(table_new=None), NULL), (dict(table_new=G + 2), ALIGN),
                                   (dict(keep=G + 1), ALIGN), (dict(table_width=(1 << 24) + 1), SHAPE),
                                   (dict(B=1 << 24, table_width=1 << 20), SHAPE)]
NORM_REFUSALS = [(dict(dtype=3), DTYPE), (dict(dtype=-1), DTYPE), (dict(x=None), NULL), (dict(gamma=None), NULL), (dict(M=0), SHAPE),
                 (dict(M=(1 << 30) + 1), SHAPE), (dict(d=0), SHAPE), (dict(d=16385, ldx=20000, ldr=20000, ldh=20000), SHAPE),
                 (dict(ldx=63), SHAPE), (dict(ldr=63), SHAPE), (dict(ldh=63), SHAPE), (dict(eps=-1.0), SHAPE),
                 (dict(eps=float("nan")), SHAPE), (dict(eps=float("inf")), SHAPE), (dict(x=G + 2), ALIGN), (dict(r=G + 2), ALIGN),
                 (dict(h=G + 2), ALIGN), (dict(gamma=G + 2), ALIGN), (dict(dtype=1, x=G + 1), ALIGN)]
W4_REFUSALS = [(dict(packed=None), NULL), (dict(N=0), SHAPE), (dict(K=0), SHAPE), (dict(group=0), SHAPE), (dict(group=48), SHAPE),
               (dict(N=(1 << 24) + 1), SHAPE), (dict(K=(1 << 24) + 1), SHAPE), (dict(packed=G + 8), ALIGN)]
REFUSALS = {
    "mq_chunk_attention": CACHE_REFUSALS + [
        (dict(dtype=3), DTYPE), (dict(dtype=-1), DTYPE), (dict(first=None), NULL), (dict(q=None), NULL), (dict(out=None), NULL),
        (dict(T=0), SHAPE), (dict(T=(1 << 30) + 1), SHAPE), (dict(max_len=0), SHAPE), (dict(max_len=257), SHAPE),
        (dict(heads=0), SHAPE), (dict(heads=5), SHAPE), (dict(heads=2048), SHAPE), (dict(kv_heads=3), SHAPE), (dict(ldq=255), SHAPE),
        (dict(ldo=255), SHAPE), (dict(ldq=1 << 41), SHAPE), (dict(first=G + 2), ALIGN), (dict(q=G + 2), ALIGN), (dict(out=G + 2), ALIGN),
        (dict(dtype=2, q=G + 1), ALIGN), (dict(ws_bytes=15), WS),
        # launches of 2^32 threads
        (dict(B=1 << 23), SHAPE), (dict(T=1 << 28, ldq=256, ldo=256), SHAPE)],
    "mq_kv_fork": TABLE_REFUSALS + [
        (dict(parent=None), NULL), (dict(grow=None), NULL), (dict(lens_new=None), NULL), (dict(missing=None), NULL),
        (dict(B_new=0), SHAPE), (dict(B_new=(1 << 30) + 1), SHAPE), (dict(B_new=1 << 29), SHAPE), (dict(B_new=1 << 10, table_width=1 << 22), SHAPE), (dict(parent=G + 2), ALIGN),
        (dict(grow=G + 1), ALIGN), (dict(lens_new=G + 2), ALIGN), (dict(missing=G + 2), ALIGN)],
    "mq_kv_compact": TABLE_REFUSALS + [
        (dict(moved=None), NULL), (dict(used=None), NULL), (dict(moved=G + 2), ALIGN), (dict(used=G + 2), ALIGN),
        (dict(B=1 << 29), SHAPE)],
    "mq_add_rms_norm": NORM_REFUSALS + [(dict(y=None), NULL), (dict(ldy=63), SHAPE), (dict(y=G + 2), ALIGN),
                                        (dict(M=1 << 30, d=1 << 12, ldx=1 << 12), SHAPE)],
    "mq_add_rms_norm_rows8": NORM_REFUSALS + [(dict(q=None), NULL), (dict(scale=None), NULL), (dict(ldq=63), SHAPE), (dict(scale=G + 1), ALIGN)],
    "mq_add_rms_norm_pack8": NORM_REFUSALS + [(dict(s=None), NULL), (dict(packed=None), NULL), (dict(s=G + 2), ALIGN), (dict(packed=G + 8), ALIGN)],
    "mq_w4_pack": W4_REFUSALS + [(dict(codes=None), NULL), (dict(scales=None), NULL), (dict(scales=G + 2), ALIGN)],
    "mq_w4_prepare": W4_REFUSALS + [(dict(w=None), NULL), (dict(w=G + 2), ALIGN)],
    "mq_w4_unpack": W4_REFUSALS + [(dict(w=None), NULL), (dict(w=G + 2), ALIGN)],
    "mq_w4_product": W4_REFUSALS + [
        (dict(x=None), NULL), (dict(y=None), NULL), (dict(ws=None), NULL), (dict(row_scale=G), NULL), (dict(xtype=3), NULL),
        (dict(xtype=4), DTYPE), (dict(xtype=-1), DTYPE), (dict(ytype=3), DTYPE), (dict(M=0), SHAPE), (dict(M=(1 << 30) + 1), SHAPE),
        (dict(ldx=69), SHAPE), (dict(ldy=4), SHAPE), (dict(ldy=1 << 41), SHAPE), (dict(x=G + 2), ALIGN), (dict(y=G + 2), ALIGN),
        (dict(bias=G + 2), ALIGN), (dict(xtype=3, row_scale=G + 2), ALIGN), (dict(ws=G + 8), ALIGN), (dict(ws_bytes=0), WS),
        (dict(M=1 << 30), SHAPE)],
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
    queries = {n for n in mq.exported_serve_symbols() if n.endswith("_bytes")}
    assert set(REFUSALS) | queries == set(mq.exported_serve_symbols())


def test_binding_refuses_host_tensors_and_other_types(lib):
    x = torch.zeros(64)
    with pytest.raises(ValueError):
        mq.mq_add_rms_norm(x, 64, None, 64, 0, x, 1, 64, 1e-6, None, 64, x, 64)
    k, v, a = torch.zeros((2, 1, 64, 64), dtype=torch.int8), torch.zeros((2, 1, 48, 64), dtype=torch.int8), torch.zeros((2, 1, 2))
    cache = mq.KvCache(k, v, a, 2, 1, 40)
    with pytest.raises(ValueError):
        mq.mq_kv_compact(cache, None, G, 1, G, 1, G, G, G, G, BIG)
    codes, scales, zeros = torch.zeros((5, 70), dtype=torch.uint8), torch.zeros((5, 3)), torch.zeros((5, 3), dtype=torch.uint8)
    for bad in ((codes.float(), scales, zeros, 32), (codes, scales.half(), zeros, 32), (codes, scales, zeros.int(), 32),
                (codes, scales[:, :2], zeros, 32), (codes, scales, zeros[:4], 32), (codes, scales, None, 64), (codes, scales, None, 0),
                (codes.t(), scales, zeros, 32), (codes, scales, None, -32), (codes, scales, None, 30)):
        with pytest.raises(ValueError):
            mq.w4_pack(*bad)
    for bad in ((codes, 32), (scales.t(), 32), (scales, 33)):
        with pytest.raises(ValueError):
            mq.w4_prepare(*bad)
