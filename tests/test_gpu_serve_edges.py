"""Corners of the serving operators' ranges (include/mq_serve.h) on the GPU, against the same formulas in 64 bits.

Tolerances come from the number formats, before any run: a rounding to a type is off by at most half a step, and where operands or
sums are whole multiples of a power of two that fit the 24 bits of binary32, products and sums are exact.
"""
import math

import numpy as np
import pytest
import torch

import paper_1805_12096_amd as mq
from test_gpu_serve import (BF16, BLOCK, DEV, EPS32, F16, F32, PARTS, TYPES, check_chunk, chunk_call, chunk_expected, gen, half_step, i32,
                            normal, product_tolerance, random_cache, tables, w4_inputs)

pytestmark = pytest.mark.gpu


# ---- attention of new tokens: scales of the values ----------------------------------------------------------------------------

# new tokens, tokens in the cache with them, heads, kv heads, width, columns that the table has more: few rows, one workgroup a tile;
# few rows in equal shares; many rows
FORMS = {"few": ([3, 20], [320, 300], 4, 2, 64, 0), "shares": ([3, 20], [640, 1300], 4, 2, 64, 100), "many": ([300, 170], [700, 1300], 8, 2, 64, 2000),
         "few wide": ([5], [384], 4, 2, 200, 0), "many wide": ([400], [1500], 4, 1, 128, 2000), "many widest": ([200], [900], 8, 2, 256, 2000)}


def a_call(form, seed):
    """(cache, table, first, lens, width of the table, queries in 64 bits, heads) of a form."""
    new, lens, heads, kv_heads, dim, room = FORMS[form]
    g = gen(seed)
    need = sum(-(-n // BLOCK) for n in lens)
    cache = random_cache(g, need, kv_heads, dim)
    width = max(-(-n // BLOCK) for n in lens) + room
    return cache, tables(g, lens, width, need), np.concatenate([[0], np.cumsum(new)]), lens, width, normal(g, sum(new), heads * dim), heads


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("power", [-130, -127, -120, -119, -118, -110, -100, -90, -70, -61, -53, -52, -30])
def test_weights_of_small_values_count(form, dtype, power):
    """Blocks whose values are very small beside ordinary ones: their tokens' weights stand in the denominator all the same.  (The
    smallest powers are those of amax; a value is a whole number of 127th of it.)"""
    cache, table, first, lens, width, q, heads = a_call(form, 30)
    cache.amax[:, :, 1] *= 2.0 ** power
    for b in range(len(lens)):                               # an ordinary block in four
        for j in range(b, -(-lens[b] // BLOCK), 4):
            cache.amax[table[b][j], :, 1] = 1.5
    q, scale = q.to(dtype).to(DEV), 0.7 * cache.head_dim ** -0.5
    args = cache, i32(table), i32(first), i32(lens), width * BLOCK
    check_chunk(chunk_call(*args, True, q, heads, scale), *chunk_expected(cache, table, first, lens, width * BLOCK, True, q, heads, scale, dtype))


@pytest.mark.parametrize("form", ["few", "shares", "many"])
@pytest.mark.parametrize("dtype", TYPES)
def test_weights_of_values_of_every_size(form, dtype):
    """Scales that change from block to block, from none to large, and scores over 20 binary orders."""
    cache, table, first, lens, width, q, heads = a_call(form, 31)
    powers = [0.0] + [2.0 ** p for p in (-140, -119, 3, -60, -118, 8 if dtype == F16 else 30, -90, -54, -53, -52, 5, -20)]
    for e in range(cache.blocks):
        cache.amax[e, :, 1] = powers[e % len(powers)] * 1.3
    q, scale = q.to(dtype).to(DEV), 1.2 * cache.head_dim ** -0.5
    args = cache, i32(table), i32(first), i32(lens), width * BLOCK
    check_chunk(chunk_call(*args, True, q, heads, scale), *chunk_expected(cache, table, first, lens, width * BLOCK, True, q, heads, scale, dtype))


@pytest.mark.parametrize("form", ["few", "shares", "many"])
@pytest.mark.parametrize("power", [-100, -80, -55, -50])
def test_values_that_are_small_throughout(form, power):
    """Results are as exact in proportion where all values are small (bfloat16 and binary32 have them)."""
    cache, table, first, lens, width, q, heads = a_call(form, 32)
    cache.amax[:, :, 1] *= 2.0 ** power
    for dtype in (BF16, F32):
        x, scale = q.to(dtype).to(DEV), cache.head_dim ** -0.5
        args = cache, i32(table), i32(first), i32(lens), width * BLOCK
        check_chunk(chunk_call(*args, False, x, heads, scale), *chunk_expected(cache, table, first, lens, width * BLOCK, False, x, heads, scale, dtype))


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_queries_next_to_the_largest_number(form, dtype):
    """Rows whose largest element lies between 2^127 and the type's largest number, beside keys and a scale that are small."""
    cache, table, first, lens, width, q, heads = a_call(form, 33)
    cache.amax[:, :, 0] *= 2.0 ** -8
    d, T = cache.head_dim, len(q)
    q = q.double().view(T, heads, d).clamp(-3, 3) * 2.0 ** 125
    at = torch.arange(T * heads).view(T, heads)
    q.scatter_(2, (at % d)[..., None], ((1 - 2 * (at % 2)) * (1 + at % 50 / 51) * 2.0 ** 127)[..., None].double())
    q = q.to(dtype).view(T, heads * d).to(DEV)
    assert torch.isfinite(q).all() and (q.view(T, heads, d).abs().amax(-1) >= 2.0 ** 127).all()
    args, scale = (cache, i32(table), i32(first), i32(lens), width * BLOCK), 2.0 ** -119
    check_chunk(chunk_call(*args, True, q, heads, scale), *chunk_expected(cache, table, first, lens, width * BLOCK, True, q, heads, scale, dtype))


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_probabilities_of_short_types_hold_sixteen_bits(form, dtype):
    """Queries that see a few tokens, scores of about 1: results are off by their own rounding and 2^-15 of the largest value, as those
    of a type whose probabilities enter in two parts."""
    new, lens, heads, kv_heads, dim, room = FORMS[form]
    g = gen(34)
    lens = list(new) if len(new) * new[0] > 100 else [n + 4 for n in new]
    cache = random_cache(g, 40, kv_heads, dim)
    width = max(-(-n // BLOCK) for n in lens) + room
    table, first = tables(g, lens, width, 40), np.concatenate([[0], np.cumsum(new)])
    q, scale = normal(g, sum(new), heads * dim).to(dtype).to(DEV), 0.3 * dim ** -0.5
    args = cache, i32(table), i32(first), i32(lens), width * BLOCK
    want, tol = chunk_expected(cache, table, first, lens, width * BLOCK, True, q, heads, scale, F16)
    tol = tol - half_step(F16, want) + half_step(dtype, want)
    check_chunk(chunk_call(*args, True, q, heads, scale), want, tol)


@pytest.mark.parametrize("form", ["few", "shares", "many"])
@pytest.mark.parametrize("dtype,bits", [(F32, 18), (F16, 10)])
def test_every_bit_of_a_query_counts(form, dtype, bits):
    """Two elements that differ in their last bit, against keys of 1 and -1: all sums are multiples of 2^-bits below 4, so scores are
    exact but for their factor (of four roundings): the lowest bit decides between two tokens.  A query without its last part
    would give both the same weight."""
    new, lens, heads, kv_heads, dim, room = FORMS[form]
    g = gen(35)
    T, need = sum(new), sum(-(-n // BLOCK) for n in lens)
    cache = random_cache(g, need, kv_heads, dim)
    width = max(-(-n // BLOCK) for n in lens) + room
    table, first = tables(g, lens, width, need), np.concatenate([[0], np.cumsum(new)])
    cache.keys.zero_()
    cache.keys[:, :, ::2, 0], cache.keys[:, :, ::2, dim - 1] = 1, -1
    cache.amax[:, :, 0] = 127.0
    q = torch.zeros(T, heads, dim)
    q[..., 0], q[..., dim - 1] = 1 + 2.0 ** -9 + 2.0 ** -bits, 1 + 2.0 ** -9
    if bits == 10:
        q[..., 0], q[..., dim - 1] = 1 + 2.0 ** -10, 1
    q = q.view(T, -1).to(dtype).to(DEV)
    scale = 2.0 ** bits                                      # scores are 1 and 0 by turns
    want, _ = chunk_expected(cache, table, first, lens, width * BLOCK, True, q, heads, scale, dtype)
    out = chunk_call(cache, i32(table), i32(first), i32(lens), width * BLOCK, True, q, heads, scale)
    # weights are off by 8 eps32 and their parts, sums of up to n of them by (n + 64) eps32; values are up to 2.5 and the result rounded
    off = (8 * EPS32 + 2.0 ** (-15 if dtype == F16 else -23) + (max(lens) + 64) * EPS32) * 2.5
    check_chunk(out, want, off + half_step(dtype, want))


# ---- norm -----------------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [40, 512, 1000])
@pytest.mark.parametrize("power", [-149, -130, -125, -121, -119, -110])
def test_multipliers_of_very_small_rows_are_finite(dtype, d, power):
    """127 / max |y| where that is a number, the largest number where it would be past it; a row that is all zeros has 1."""
    g, M = gen(d), 5
    x, gamma = normal(g, M, d).to(dtype).to(DEV), torch.full((d,), 2.0 ** power, device=DEV)
    x[3] = 0
    z = x.double()
    y = z / torch.sqrt((z * z).mean(-1, keepdim=True) + 1e-5) * gamma.double()
    q, scale = torch.empty((M, d), dtype=torch.int8, device=DEV), torch.empty(M, device=DEV)
    mq.mq_add_rms_norm_rows8(x, d, None, d, mq.dtype_code(dtype), gamma, M, d, 1e-5, None, d, q, d, scale)
    assert scale[3] == 1 and not q[3].any()
    rows, most = [0, 1, 2, 4], torch.finfo(F32).max
    assert torch.isfinite(scale).all()
    # y is off by 43 eps32 in proportion (sums of squares) or by half of 2^-149, whichever is more, its largest element likewise
    top = y[rows].abs().amax(-1)
    off = 43 * EPS32 * top + 2.0 ** -150
    low, high = 127 / (top + off) * (1 - EPS32), torch.where(top > off, 127 / (top - off) * (1 + EPS32), torch.full_like(top, math.inf))
    s = scale[rows].double()
    if power > -149:                                         # (there a row may be zeros altogether)
        assert ((s >= low.clamp(max=most)) & (s <= high.clamp(max=most))).all()
        assert ((q[rows].double() - y[rows] * s[:, None]).abs() <= 0.5 + (off * s)[:, None] + 127 * EPS32).all()


# ---- products with 4-bit parameters -------------------------------------------------------------------------------------------

def product(x, packed, N, group, out, rs=None, bias=None, K=None):
    """y of an x of which K columns count."""
    M, K = len(x), K or x.shape[1]
    y = torch.full((M, N), 7.0, dtype=out, device=DEV)
    ws = torch.full((mq.mq_w4_product_ws_bytes(M, N, K),), 255, dtype=torch.uint8, device=DEV)
    mq.mq_w4_product(x, x.stride(0), mq.MQ_ROWS8 if rs is not None else mq.dtype_code(x.dtype), rs, packed, M, N, K, group, bias, y, N,
                     mq.dtype_code(out), ws, ws.numel())
    return y


@pytest.mark.parametrize("M", [1, 5, 8, 9, 70])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("K", [32, 300, 1000])
def test_zeros_next_to_codes_cost_no_bits(M, group, K):
    """Binary32 rows with one element each, codes and zeros that differ by 1: the result is that element times the scale, rounded
    (a power of two here: not even that), however large codes and zeros are."""
    g, N = gen(M), 40
    groups = -(-K // group)
    zeros = torch.randint(0, 15, (N, groups), generator=g).to(torch.uint8)
    codes = (zeros[:, torch.arange(K) // group] + 1).to(torch.uint8)
    scales = 2.0 ** torch.randint(-3, 4, (N, groups), generator=g).float()
    packed = mq.w4_pack(codes.to(DEV), scales.to(DEV), zeros.to(DEV), group)
    x, at = torch.zeros(M, K), torch.randint(0, K, (M,), generator=g)
    x[torch.arange(M), at] = normal(g, M)
    want = x[torch.arange(M), at][:, None] * scales[:, at // group].T
    y = product(x.to(DEV), packed, N, group, F32).cpu()
    assert ((y.double() - want.double()).abs() <= EPS32 * want.abs()).all(), float(((y - want) / want).abs().max()) / EPS32


@pytest.mark.parametrize("M", [1, 6, 9, 16, 40])
@pytest.mark.parametrize("xtype", [F32, F16, BF16])
def test_every_bit_of_x_counts(M, xtype):
    """Rows with one element each and codes 15 off their zeros: 15 times the element, off by few roundings of 31 times it.  The last
    of its parts is about 2^-18 (binary32), 2^-9 (binary16) of it."""
    g, N, K, group = gen(M), 33, 512, 64
    packed = mq.w4_pack(torch.full((N, K), 15, dtype=torch.uint8, device=DEV), torch.ones((N, K // group), device=DEV),
                        torch.zeros((N, K // group), dtype=torch.uint8, device=DEV), group)
    x, at = torch.zeros(M, K, dtype=xtype), torch.randint(0, K, (M,), generator=g)
    # values whose parts are all there: bits at the top, in the middle and at the end
    x[torch.arange(M), at] = (1 + 2.0 ** -9 * 1.3333334 * (1 + torch.arange(M) / 50)).to(xtype) * (2.0 ** torch.randint(-9, 9, (M,), generator=g)).to(xtype)
    want = 15 * x[torch.arange(M), at].double()[:, None].expand(M, N)
    y = product(x.to(DEV), packed, N, group, F32).double().cpu()
    assert ((y - want).abs() <= 31 * 8 * EPS32 / 2 * want.abs() / 15).all(), float(((y - want) / want).abs().max())


# rows, width; few rows of whole pieces: of one and two row tiles, fragments fewer and more than waves ahead, ragged ends
FEW = [(17, 128), (24, 336), (31, 624), (32, 2192), (18, 4096), (32, 16), (29, 8208), (9, 384), (16, 2064), (12, 80), (3, 2304), (8, 5120), (1, 10000),
       (5, 48), (7, 640)]


@pytest.mark.parametrize("M,K", FEW)
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("xtype", ["rows8", F32, F16, BF16])
def test_few_rows_of_whole_pieces(M, K, group, xtype):
    """Every form for few rows (binary16 and binary32 take it up to 16 and 8 rows, so others here see the form for many)."""
    g, N = gen(M * K + group), 16 * (M % 3 + 1) + M % 5
    codes, s, z, w = w4_inputs(g, N, K, group, M % 2 == 0)
    packed = mq.w4_pack(codes, s, z, group)
    bias = normal(g, N).to(DEV) if M % 4 else None
    ld, rs = K + 16 * (M % 2), None
    if xtype == "rows8":
        x = torch.full((M, ld), 55, dtype=torch.int8, device=DEV)
        x[:, :K] = torch.randint(-127, 128, (M, K), generator=g).to(torch.int8)
        rs, out = (5 + 10 * torch.rand(M, generator=g)).to(DEV), BF16 if group == 64 else F32
        x64 = x[:, :K].double().cpu() / rs.double().cpu()[:, None]
    else:
        x, out = torch.full((M, ld), math.nan, dtype=xtype, device=DEV), xtype if group == 64 else F32
        x[:, :K] = normal(g, M, K).to(xtype)
        x64 = x[:, :K].double().cpu()
    want = x64 @ w.T + (0 if bias is None else bias.double().cpu())
    w31 = (62.0 * s.double().cpu())[:, torch.arange(K) // group]
    tol = product_tolerance(x64, w31, K, group, 1 if xtype == "rows8" else PARTS[xtype], out, want)
    off = (product(x, packed, N, group, out, rs, bias, K).double().cpu() - want).abs()
    assert (off <= tol).all(), float((off / tol).max())
    if xtype == "rows8" and out == F32 and bias is None:
        # whole numbers: sums of a group are exact; its fused operation, the join of up to four waves and the quotient are off by
        # half a step each of something that is at most sum |x| |w|
        assert (off <= (-(-K // group) + 4 + 1) * EPS32 / 2 * (x64.abs() @ w.abs().T)).all()


@pytest.mark.parametrize("xtype,M", [(F32, 65535 * 32 + 33), (BF16, 65535 * 64 + 65)])
def test_millions_of_rows(xtype, M):
    """More rows than one axis of a launch has workgroups for; each row is the product of its own."""
    g, N, K, group = gen(41), 3, 4, 32
    codes, s, z, w = w4_inputs(g, N, K, group)
    packed = mq.w4_pack(codes, s, z, group)
    x = (torch.arange(M, device=DEV)[:, None] * torch.tensor([1, 3, 7, 11], device=DEV) % 251 - 125).to(xtype)
    y = product(x, packed, N, group, F32)
    # whole numbers below 2^7 by whole numbers below 2^4, times a scale: one rounding each for it, the zero's product and the sum
    want = x.double() @ w.T.contiguous().to(DEV)
    assert ((y.double() - want).abs() <= 4 * EPS32 * 4 * 125 * 62 * s.max()).all()


def test_more_short_sequences_than_a_join_would_have_places():
    """Single launches are bounded by their own workgroups: 131072 sequences of one new token, 32 heads.  Held against calls of a
    quarter of them."""
    g, B, heads, dim, blocks = gen(42), 131072 + 96, 32, 8, 600
    cache = random_cache(g, blocks, heads, dim)
    table = torch.randint(0, blocks, (B, 2), generator=g, dtype=torch.int32).to(DEV)
    lens = torch.randint(0, 129, (B,), generator=g, dtype=torch.int32).to(DEV)
    q = normal(g, B, heads * dim).to(BF16).to(DEV)

    def call(at, n):
        return chunk_call(cache, table[at:at + n], torch.arange(n + 1, dtype=torch.int32, device=DEV), lens[at:at + n], 128, True, q[at:at + n], heads, 0.3)
    assert mq.mq_chunk_attention_ws_bytes(B, B, 128, heads, heads, dim) > 0
    whole = call(0, B)
    step = B // 4
    for at in range(0, B, step):
        assert torch.equal(whole[at:at + step], call(at, step))


# ---- the form for many rows: what the other forms are held to elsewhere --------------------------------------------------------

MANY = [f for f in FORMS if f.startswith("many")]


@pytest.mark.parametrize("form", MANY)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [None, 40, 57, 130])
def test_many_rows(form, dtype, dim):
    """Whole tiles and ragged ends, with and without a mask; widths that are no whole pieces."""
    new, lens, heads, kv_heads, d, room = FORMS[form]
    d, g = dim or d, gen(50)
    new, lens = [*new, max(new) - 13, 0], [*lens, 500, 10]
    need = sum(-(-n // BLOCK) for n in lens)
    cache = random_cache(g, need, kv_heads, d)
    width = max(-(-n // BLOCK) for n in lens) + 4 * room
    table, first = tables(g, lens, width, need), np.concatenate([[0], np.cumsum(new)])
    q = normal(g, sum(new), heads * d).to(dtype).to(DEV)
    for causal in (True, False):
        out = chunk_call(cache, i32(table), i32(first), i32(lens), width * BLOCK, causal, q, heads, d ** -0.5)
        check_chunk(out, *chunk_expected(cache, table, first, lens, width * BLOCK, causal, q, heads, d ** -0.5, dtype))


@pytest.mark.parametrize("form", MANY)
@pytest.mark.parametrize("dtype", TYPES)
def test_many_rows_with_other_scales(form, dtype):
    cache, table, first, lens, width, q, heads = a_call(form, 51)
    q = q.to(dtype).to(DEV)
    for scale in (-0.1, 0.0):
        out = chunk_call(cache, i32(table), i32(first), i32(lens), width * BLOCK, True, q, heads, scale)
        want, _ = chunk_expected(cache, table, first, lens, width * BLOCK, True, q, heads, scale, dtype)
        _, tol = chunk_expected(cache, table, first, lens, width * BLOCK, True, q, heads, -scale, dtype)     # (depends on its magnitude)
        check_chunk(out, want, tol + half_step(dtype, want))


@pytest.mark.parametrize("form", MANY)
@pytest.mark.parametrize("dtype", TYPES)
def test_many_rows_keep_bad_queries_apart(form, dtype):
    cache, table, first, lens, width, good, heads = a_call(form, 52)
    T, d, good = len(good), cache.head_dim, good.to(dtype)
    q = good.clone()
    q[3, 5], q[25, d + d - 1], q[T - 1, 2 * d + 8], q[30, :d] = math.nan, math.inf, -math.inf, math.inf
    args = cache, i32(table), i32(first), i32(lens), width * BLOCK, True
    out, clean = (chunk_call(*args, x.to(DEV), heads, 0.1).view(T, heads, d) for x in (q, good))
    bad = (~torch.isfinite(q)).view(T, heads, d).any(-1).to(DEV)
    assert torch.isnan(out[bad]).all() and torch.equal(out[~bad], clean[~bad])


@pytest.mark.parametrize("form", MANY)
def test_many_rows_with_bad_lists_and_tables(form):
    """Lists that descend or leave their range, lengths out of theirs, entries that are no block: nothing outside the rows is written."""
    cache, table, _, lens, width, q, heads = a_call(form, 53)
    T, B = len(q), len(lens)
    table[:, 1::3], q = cache.blocks + 5, q.to(BF16).to(DEV)
    store = torch.full((T + 20, q.shape[1]), 7.0, dtype=BF16, device=DEV)
    for first in ([5, 2, T], [T, 0, T], [-9, T + 5, 3]):
        for n in ([1 << 30, -5], [300, 900]):
            chunk_call(cache, i32(table), i32(first[:B + 1]), i32(n[:B]), width * BLOCK, True, q, heads, 0.1, store[10:10 + T])
            assert (store[:10] == 7.0).all() and (store[10 + T:] == 7.0).all() and not torch.isnan(store).any()


@pytest.mark.parametrize("form", MANY)
@pytest.mark.parametrize("dtype", TYPES)
def test_many_rows_in_place_captured_and_beside_another_stream(form, dtype):
    cache, table, first, lens, width, q, heads = a_call(form, 54)
    g, q = gen(55), q.to(dtype).to(DEV)
    args = cache, i32(table), i32(first), i32(lens), width * BLOCK, True, q, heads, 0.09
    want = chunk_call(*args)
    again = q.clone()
    chunk_call(*args[:6], again, *args[7:], out=again)
    assert torch.equal(again, want)
    out = torch.zeros_like(q)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph):
        chunk_call(*args, out=out)
    for i in range(3):
        q.copy_(normal(g, *q.shape).to(dtype))
        out.zero_()
        beside = torch.zeros_like(q)
        want = chunk_call(*args)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            chunk_call(*args, out=beside)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(beside, want), i


@pytest.mark.parametrize("group", [32, 128])
def test_an_infinity_costs_its_group_and_nothing_else(group):
    """A scale that holds an infinity is one: the group comes out as NaN, as the header says; other groups and rows are what they were."""
    g, N, K = gen(60), 20, 300
    w = normal(g, N, K)
    bad = w.clone()
    bad[3, group + 5], bad[17, 299] = math.inf, -math.inf
    back = [torch.empty((N, K), device=DEV) for _ in range(2)]
    for x, y in zip((w, bad), back):
        mq.mq_w4_unpack(mq.w4_prepare(x.to(DEV), group), N, K, group, y)
    lost = torch.zeros((N, K), dtype=torch.bool, device=DEV)
    lost[3, group:2 * group], lost[17, 299 // group * group:] = True, True
    assert torch.isnan(back[1][lost]).all() and torch.equal(back[1][~lost], back[0][~lost])
