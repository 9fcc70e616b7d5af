"""The serving operators (include/mq_serve.h) on the GPU against plain implementations in 64 bits.

Tolerances come from the number formats, before any run.  With eps = torch.finfo(type).eps a rounding to the type is off by at
most eps / 2 of the value; values below the smallest normal one are eps times that apart, whatever they are (binary16: steps of
2^-24 below 2^-14), and a rounding there is off by at most half of it.
"""
import math

import numpy as np
import pytest
import torch

import paper_1805_12096_amd as mq

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
BLOCK = mq.MQ_KV_BLOCK
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
TYPES = [F32, F16, BF16]
EPS32 = torch.finfo(F32).eps
PARTS = {F32: 3, F16: 2, BF16: 1}
PLACES = [16 * ((t // 4) % 4) + 4 * (t // 16) + t % 4 for t in range(BLOCK)]


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def normal(g, *shape):
    return torch.randn(shape, generator=g)


def half_step(t, value):
    """How far a rounding of `value` to the type may be off."""
    f = torch.finfo(t)
    return f.eps / 2 * value.abs().clamp(min=f.smallest_normal)


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def random_cache(g, blocks, heads, dim):
    c = mq.kv_cache(blocks, heads, dim, DEV)
    c.keys[..., :dim] = torch.randint(-127, 128, c.keys[..., :dim].shape, generator=g, dtype=torch.int8).to(DEV)
    c.values[:, :, :dim] = torch.randint(-127, 128, c.values[:, :, :dim].shape, generator=g, dtype=torch.int8).to(DEV)
    c.amax.copy_((0.5 + torch.rand(c.amax.shape, generator=g)) * 2)
    return c


def cached(cache, row, n):
    """(keys, values, whether there) of a sequence's first n tokens in 64 bits, on the host: [heads, n, dim]."""
    d, hk = cache.head_dim, cache.kv_heads
    k, v, there = torch.zeros(2, hk, n, d, dtype=torch.float64).unbind(0) + (torch.zeros(n, dtype=torch.bool),)
    for t0 in range(0, n, BLOCK):
        e, m = int(row[t0 // BLOCK]), min(BLOCK, n - t0)
        if not 0 <= e < cache.blocks:
            continue
        a = cache.amax[e].double().cpu() / 127
        k[:, t0:t0 + m] = cache.keys[e][:, :m, :d].double().cpu() * a[:, 0, None, None]
        v[:, t0:t0 + m] = cache.values[e].double().cpu()[:, :d].transpose(1, 2)[:, PLACES][:, :m] * a[:, 1, None, None]
        there[t0:t0 + m] = True
    return k, v, there


# ---- chunk attention ----------------------------------------------------------------------------------------------------

def chunk_expected(cache, table, first, lens, max_len, causal, q, heads, scale, dtype):
    """(outputs, tolerances) by token row; rows of nobody are NaN.

    A score of d products in NP parts, added in binary32, is off by at most (d NP + 8) eps32 sum |q| |k|, its factor and the
    difference to the maximum included; the exponential, its product with the values' scale in as many parts as the type has,
    8 bits each, by 4 eps32 + 2^-(8 NP) in proportion; sums over n values (of magnitude up to the largest) and their rescaling by
    (n + 64) eps32.  The result is rounded to the type once."""
    T, d, hk = q.shape[0], cache.head_dim, cache.kv_heads
    per, np_ = heads // hk, PARTS[dtype]
    out, tol = torch.full((T, heads, d), math.nan, dtype=torch.float64), torch.zeros(T, heads, d, dtype=torch.float64)
    first = [min(max(int(f), 0), T) for f in first]
    for b in range(len(lens)):
        n, new = min(max(int(lens[b]), 0), max_len), first[b + 1] - first[b]
        if new <= 0:
            continue
        k, v, there = cached(cache, table[b], n)
        x = q[first[b]:first[b + 1]].double().cpu().view(new, hk, per, d).permute(1, 2, 0, 3)          # [hk, per, new, d]
        seen = there[None, :].expand(new, n)
        if causal:
            seen = seen & (torch.arange(n)[None, :] <= torch.arange(new)[:, None] + n - new)
        s = (x.reshape(hk, per * new, d) @ k.transpose(1, 2)).view(hk, per, new, n) * scale
        s = s.masked_fill(~seen, -math.inf)
        m = s.amax(-1, keepdim=True) if n else torch.full((hk, per, new, 1), -math.inf, dtype=torch.float64)
        p = torch.exp(s - torch.where(m > -math.inf, m, torch.zeros_like(m)))
        total = p.sum(-1, keepdim=True)
        o = (p.view(hk, per * new, n) @ v).view(hk, per, new, d) / torch.where(total > 0, total, torch.ones_like(total))
        big = (x.abs().reshape(hk, per * new, d) @ k.abs().transpose(1, 2)).view(hk, per, new, n).amax(-1) * scale if n else torch.zeros(hk, per, new)
        vmax = v.abs().amax(1) if n else torch.zeros(hk, d)
        off = (torch.exp(2 * (d * np_ + 8) * EPS32 * big) - 1 + 8 * EPS32 + 2.0 ** (-8 * np_ + 1) + (n + 64) * EPS32)[..., None] * vmax[:, None, None]
        out[first[b]:first[b + 1]] = o.permute(2, 0, 1, 3).reshape(new, heads, d)
        tol[first[b]:first[b + 1]] = (off + half_step(dtype, o)).permute(2, 0, 1, 3).reshape(new, heads, d)
    return out.view(T, -1), tol.view(T, -1)


def chunk_call(cache, table, first, lens, max_len, causal, q, heads, scale, out=None, stream=None):
    T = q.shape[0]
    B = len(lens)
    if out is None:
        out = torch.full((T, heads * cache.head_dim), 7.0, dtype=q.dtype, device=DEV)
    ws = torch.full((mq.mq_chunk_attention_ws_bytes(B, T, max_len, heads, cache.kv_heads, cache.head_dim),), 255, dtype=torch.uint8, device=DEV)
    mq.mq_chunk_attention(cache, table, table.shape[1], first, lens, B, T, max_len, causal, q, q.stride(0), heads, mq.dtype_code(q.dtype),
                          scale, out, out.stride(0), ws, ws.numel(), stream)
    return out


def check_chunk(out, expected, tol):
    got = out.double().cpu()
    nobody = torch.isnan(expected)
    assert (got[nobody] == 7.0).all(), "rows of nobody were written"
    off = (got - expected).abs()[~nobody]
    assert (off <= tol[~nobody]).all(), float((off / tol[~nobody]).max())


def tables(g, lens, width, blocks):
    order = torch.randperm(blocks, generator=g).tolist()
    table = np.full((len(lens), width), -1, np.int32)
    for b, n in enumerate(lens):
        for j in range(-(-n // BLOCK)):
            table[b, j] = order.pop()
    return table


CHUNKS = [
    # new tokens, tokens in the cache with them, heads, kv heads, width
    ([1], [1], 1, 1, 64),
    ([1, 0, 3, 64], [1, 5, 64, 65], 4, 2, 64),
    ([5, 2, 1, 1, 70], [5, 200, 63, 129, 71], 8, 8, 80),
    ([33], [1000], 8, 1, 128),
    ([4, 3, 6, 5], [900, 1300, 64, 77], 8, 2, 128),
    ([17, 300], [2000, 301], 6, 3, 33),
    ([2, 9], [130, 500], 16, 1, 256),
    ([40, 1], [41, 190], 5, 5, 160),
    ([130, 257, 1], [700, 257, 3], 12, 3, 96),
    ([1, 1, 1], [4500, 33, 0], 7, 1, 64),
    # many rows (and tables so wide that there may be much to do): whole tiles and ragged ends, parts of tiles
    ([300, 0, 77], [300, 10, 2500], 4, 2, 64),
    ([513, 70], [5000, 90], 4, 1, 128),
    ([200], [4400], 3, 3, 192),
    ([129, 260], [131, 2300], 2, 1, 250),
    ([64], [64], 16, 2, 40),
    # and few rows of a call that may be long
    ([3, 1, 0, 20], [1200, 64, 7, 3000], 8, 2, 128),
    ([2], [4097], 4, 4, 256),
    # more tiles, and more heads, than workgroups plan for; tiles of one head that fit a share each, and that do not
    ([1 + i % 3 for i in range(210)], [1 + i * 37 % 300 for i in range(210)], 2, 1, 64),
    ([3, 1], [700, 70], 200, 200, 16),
    ([3, 0, 2], [130, 5, 64], 1024, 1024, 8),
    ([4, 4, 4], [1500, 900, 1501], 8, 2, 64),
    ([2] * 24, [100 + 53 * i for i in range(24)], 4, 4, 64),
]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("case,room", [(c, 0 if c < 10 else 2000 if c < 17 else 30) for c in range(len(CHUNKS))] + [(c, 60) for c in range(10)])
def test_chunk(dtype, causal, case, room):
    """room: columns that the table has more than it needs, for calls that say only that sequences may be as long as it is."""
    new, lens, heads, kv_heads, dim = CHUNKS[case]
    g = gen(case)
    T = sum(new)
    need = sum(-(-n // BLOCK) for n in lens) + 2
    cache = random_cache(g, need, kv_heads, dim)
    width = max(1, max(-(-n // BLOCK) for n in lens)) + case % 2 + room
    table = tables(g, lens, width, need)
    first = np.concatenate([[0], np.cumsum(new)])
    q = normal(g, T, heads * dim).to(dtype).to(DEV)
    max_len = width * BLOCK if room else max(1, max(lens))
    out = chunk_call(cache, i32(table), i32(first), i32(lens), max_len, causal, q, heads, dim ** -0.5)
    check_chunk(out, *chunk_expected(cache, table, first, lens, max_len, causal, q, heads, dim ** -0.5, dtype))


@pytest.mark.parametrize("dtype", TYPES)
def test_chunk_lists_tables_and_rows_that_are_odd(dtype):
    """Rows in front of the first sequence and behind the last, lengths outside their range, fewer tokens than queries, entries
    that are no block, rows apart, bases that are aligned to an element only, NaN in what nobody reads."""
    g = gen(5)
    heads, kv_heads, dim, scale = 6, 2, 72, 0.2
    lens, first = [300, -4, 10, 5000, 64], [3, 40, 45, 60, 61, 75]
    T, max_len = 80, 320
    cache = random_cache(g, 30, kv_heads, dim)
    table = tables(g, [320] * 5, 5, 30)
    table[0, 1], table[3, 4], table[4, 0], table[0, 4] = -1, 30, -7, 2 ** 30
    spare = [e for e in range(30) if e not in table]
    cache.amax[spare] = math.nan
    store = torch.full((T * 500 + 1,), math.nan, dtype=dtype, device=DEV)
    q = store[1:].view(T, 500)[:, 3:3 + heads * dim]
    values = normal(g, T, heads * dim).to(dtype)
    values[first[0] + 2, dim:2 * dim] *= 1e4 if dtype != F16 else 10
    q[first[0]:first[-1]] = values[first[0]:first[-1]].to(DEV)
    out = torch.full((T, 477), 7.0, dtype=dtype, device=DEV)[:, 1:1 + heads * dim]
    for causal in (True, False):
        out.fill_(7.0)
        chunk_call(cache, i32(table), i32(first), i32(lens), max_len, causal, q, heads, scale, out)
        check_chunk(out, *chunk_expected(cache, table, first, lens, max_len, causal, q, heads, scale, dtype))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("max_len", [1200, 4096])
def test_chunk_bad_queries_stay_with_themselves(dtype, max_len):
    g = gen(6)
    heads, kv_heads, dim = 4, 2, 64
    new, lens = [20, 30], [100, 1200]
    cache = random_cache(g, 24, kv_heads, dim)
    table, first = tables(g, lens, 64, 24), np.array([0, 20, 50])
    q = normal(g, 50, heads * dim).to(dtype)
    good = q.clone()
    q[3, 5], q[25, 64 + 63], q[49, 200], q[30, :64] = math.nan, math.inf, -math.inf, math.inf
    args = cache, i32(table), i32(first), i32(lens), max_len, True
    out, clean = (chunk_call(*args, x.to(DEV), heads, 0.125) for x in (q, good))
    bad = torch.isnan(q) | torch.isinf(q)
    bad = bad.view(50, heads, dim).any(-1)
    assert torch.isnan(out.view(50, heads, dim)[bad.to(DEV)]).all()
    assert torch.equal(out.view(50, heads, dim)[~bad.to(DEV)], clean.view(50, heads, dim)[~bad.to(DEV)])
    # queries with nothing to see give zeros, whatever they hold
    out = chunk_call(cache, i32(table), i32(first), i32([2, 0]), max_len, True, q.to(DEV), heads, 0.125)
    assert (out[:18] == 0).all() and (out[20:] == 0).all() and not torch.isnan(out[18:20]).any()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("max_len,new", [(320, [3, 40]), (6400, [3, 40]), (64000, [300, 40])])
def test_chunk_negative_and_zero_scales(dtype, max_len, new):
    g = gen(15)
    heads, kv_heads, dim, lens = 6, 2, 48, [300, 171]
    cache = random_cache(g, 12, kv_heads, dim)
    table, first = tables(g, lens, 1000, 12), np.concatenate([[0], np.cumsum(new)])
    q = normal(g, sum(new), heads * dim).to(dtype).to(DEV)
    for scale in (-0.1, 0.0):
        out = chunk_call(cache, i32(table), i32(first), i32(lens), max_len, True, q, heads, scale)
        expected, _ = chunk_expected(cache, table, first, lens, max_len, True, q, heads, scale, dtype)
        _, tol = chunk_expected(cache, table, first, lens, max_len, True, q, heads, -scale, dtype)     # (depends on its magnitude)
        # (the rounding of the result itself, which is another one for the other sign)
        check_chunk(out, expected, tol + half_step(dtype, expected))


@pytest.mark.parametrize("max_len", [320, 6400, 64000])
def test_chunk_with_a_bad_list_stays_inside_its_rows(max_len):
    g = gen(16)
    heads, kv_heads, dim, T = 4, 2, 64, 700
    cache = random_cache(g, 12, kv_heads, dim)
    table, lens = tables(g, [300] * 2, 1000, 12), [300, 300, 1 << 30, -5, 17]
    table = np.concatenate([table, table, table[:1]])
    store = torch.full((T + 20, heads * dim), 7.0, device=DEV)
    q = normal(g, T, heads * dim).to(DEV)
    for first in ([5, 2, 600, 7, 1000, -3], [700, 0, 700, 0, 700, 0], [-9, 300, 299, 298, 2 ** 31 - 1, 5]):
        chunk_call(cache, i32(table), i32(first), i32(lens), max_len, True, q, heads, 0.1, store[10:10 + T])
        assert (store[:10] == 7.0).all() and (store[10 + T:] == 7.0).all()
        assert not torch.isnan(store).any()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("max_len", [400, 4096])
def test_chunk_large_and_small_magnitudes(dtype, max_len):
    """Scales of blocks that differ by 2^80, queries of any magnitude: references move, nothing overflows on the way."""
    g = gen(7)
    heads, kv_heads, dim = 2, 1, 64
    new, lens = [10], [400]
    cache = random_cache(g, 8, kv_heads, dim)
    cache.amax[:, 0, 1] = torch.tensor([2.0 ** (20 * (i % 5) - 40) for i in range(8)], device=DEV)
    cache.amax[3, 0, 1] = 0
    table, first = tables(g, lens, 64, 8), np.array([0, 10])
    for power in (-100, -20, 0, 60):
        q = (normal(g, 10, heads * dim) * 2.0 ** power).to(dtype).to(DEV)
        scale = 2.0 ** -(power + 3)
        out = chunk_call(cache, i32(table), i32(first), i32(lens), max_len, True, q, heads, scale)
        check_chunk(out, *chunk_expected(cache, table, first, lens, max_len, True, q, heads, scale, dtype))


def test_chunk_of_one_token_is_cached_attention():
    """One new token per sequence: the formula of mq_cached_attention."""
    g = gen(8)
    heads, kv_heads, dim, lens = 8, 2, 128, [1, 64, 65, 700, 1900]
    cache = random_cache(g, 60, kv_heads, dim)
    table = tables(g, lens, 30, 60)
    q = normal(g, 5, heads * dim).to(DEV)
    out = chunk_call(cache, i32(table), i32(range(6)), i32(lens), 1900, True, q, heads, 0.09)
    ws = torch.empty(mq.mq_cached_attention_ws_bytes(5, 1900, heads, kv_heads, dim), dtype=torch.uint8, device=DEV)
    want = torch.empty_like(out)
    mq.mq_cached_attention(cache, i32(table), 30, i32(lens), 5, 1900, q, q.stride(0), heads, mq.MQ_F32, 0.09, want, want.stride(0), ws, ws.numel())
    assert torch.allclose(out, want, rtol=0, atol=1e-4)         # (both are held to 64 bits elsewhere)


def test_chunk_in_place_and_captured():
    """out is q; the same call replayed between eager work gives the same bits."""
    g = gen(9)
    heads, kv_heads, dim, new, lens = 8, 2, 64, [7, 30, 1], [2500, 90, 1]
    cache = random_cache(g, 60, kv_heads, dim)
    table, first = i32(tables(g, lens, 40, 60)), i32(np.concatenate([[0], np.cumsum(new)]))
    n = i32(lens)
    q = normal(g, 38, heads * dim).to(BF16).to(DEV)
    want = chunk_call(cache, table, first, n, 2500, True, q, heads, 0.125)
    again = q.clone()
    chunk_call(cache, table, first, n, 2500, True, again, heads, 0.125, out=again)
    assert torch.equal(again, want)
    out = torch.zeros_like(q)
    ws = torch.empty(mq.mq_chunk_attention_ws_bytes(3, 38, 2500, heads, kv_heads, dim), dtype=torch.uint8, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mq.mq_chunk_attention(cache, table, 40, first, n, 3, 38, 2500, True, q, q.stride(0), heads, mq.MQ_BF16, 0.125, out,
                              out.stride(0), ws, ws.numel())
    for i in range(4):
        q.copy_(normal(g, 38, heads * dim).to(BF16))
        out.zero_()
        want = chunk_call(cache, table, first, n, 2500, True, q, heads, 0.125)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want), i


@pytest.mark.parametrize("dtype", TYPES)
def test_chunk_of_many_rows_captured_beside_another_stream(dtype):
    """The form for many rows from a graph, replayed while the same call runs on another stream with a workspace of its own."""
    g = gen(19)
    heads, kv_heads, dim, new, lens = 8, 2, 128, [300, 170], [4000, 900]
    T, width = sum(new), 100
    cache = random_cache(g, 90, kv_heads, dim)
    table, first, n = i32(tables(g, lens, width, 90)), i32(np.concatenate([[0], np.cumsum(new)])), i32(lens)
    q = normal(g, T, heads * dim).to(dtype).to(DEV)
    args = cache, table, first, n, width * BLOCK, True, q, heads, 0.09
    chunk_call(*args)
    out = torch.zeros_like(q)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph):
        chunk_call(*args, out=out)
    for i in range(3):
        q.copy_(normal(g, T, heads * dim).to(dtype))
        out.zero_()
        beside = torch.zeros_like(q)
        want = chunk_call(*args)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            chunk_call(*args, out=beside)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(beside, want), i


# ---- fork and compact -----------------------------------------------------------------------------------------------------

def fork_expected(keep, table, lens, parent, grow, blocks):
    """The rules, entry after entry: (table, lens, missing, copies as (from, to))."""
    B, width = table.shape
    rows, readers, writers = [], set(i for i in range(blocks) if keep is not None and keep[i]), {}
    for b in range(len(parent)):
        known = 0 <= parent[b] < B
        n = min(max(int(lens[parent[b]]), 0), width * BLOCK) if known else 0
        held = -(-n // BLOCK)
        entries = [int(e) if 0 <= e < blocks else -1 for e in (table[parent[b]][:held] if known else [])]
        more = max(int(grow[b]), 0)
        rows.append((n, entries, min(-(-(n + more) // BLOCK), width)))
        for j, e in enumerate(entries):
            if e >= 0:
                if j == held - 1 and n % BLOCK and more:
                    writers.setdefault(e, []).append(b)
                else:
                    readers.add(e)
    free = [i for i in range(blocks) if i not in readers and i not in writers]
    out, copies, missing = np.full((len(parent), width), -1, np.int32), [], 0
    for b, (n, entries, end) in enumerate(rows):
        for j in range(max(end, len(entries))):
            if j < len(entries):
                e = entries[j]
                if e < 0 or b not in writers.get(e, []) or j != len(entries) - 1 or (e not in readers and writers[e][0] == b):
                    out[b, j] = e
                    continue
            if free:
                out[b, j] = free.pop(0)
                if j < len(entries):
                    copies.append((entries[j], int(out[b, j])))
            else:
                missing += 1
    return out, np.array([r[0] for r in rows], np.int32), missing, copies


def fork_call(cache, keep, table, lens, parent, grow, stream=None):
    B, n, width = len(lens), len(parent), table.shape[1]
    new = torch.full((n, width), 99, dtype=torch.int32, device=DEV)
    lens_new, missing = torch.full((n,), 99, dtype=torch.int32, device=DEV), torch.full((1,), 99, dtype=torch.int32, device=DEV)
    ws = torch.full((mq.mq_kv_fork_ws_bytes(cache.blocks, n, width),), 170, dtype=torch.uint8, device=DEV)
    mq.mq_kv_fork(cache, keep, table, width, lens, B, parent, grow, n, new, lens_new, missing, ws, ws.numel(), stream)
    return new, lens_new, missing


def contents(cache):
    return [t.clone() for t in (cache.keys, cache.values, cache.amax)]


def moved_contents(before, copies):
    after = [t.clone() for t in before]
    for at, to in copies:
        for x, y in zip(after, before):
            x[to] = y[at]
    return after


@pytest.mark.parametrize("seed", range(12))
@pytest.mark.parametrize("room", ["plenty", "scarce", "large"])
def test_fork(seed, room):
    """large: more blocks, or larger tables, than one workgroup does alone."""
    g = gen(100 + seed)
    rnd = np.random.RandomState(seed)
    B, width = rnd.randint(1, 40), rnd.randint(1, 9)
    n = rnd.randint(1, 90)
    if room == "large" and seed % 2:
        width, n = width + 200, n + 80
    lens = rnd.randint(-3, width * BLOCK + 10, B)
    lens[rnd.rand(B) < 0.3] //= BLOCK
    lens[rnd.rand(B) < 0.3] *= BLOCK
    lens = np.clip(lens, -5, 2 ** 20)
    blocks = rnd.randint(1, 5) if room == "scarce" and seed % 3 == 0 else B * width + (3 * n if room == "plenty" else n // 3)
    if room == "large":
        blocks = B * width + n + (0 if seed % 2 else 17000)
    # tables with shared, repeated and absent blocks
    table = rnd.randint(-2, blocks + 2, (B, width)) if seed % 2 else rnd.permutation(max(blocks, B * width))[:B * width].reshape(B, width)
    parent = rnd.randint(-2, B + 2, n)
    grow = rnd.randint(-1, 130, n) * (rnd.rand(n) < 0.8)
    keep = (rnd.rand(blocks) < 0.2).astype(np.int32) * 5 if seed % 4 else None
    heads, dim = [(1, 64), (2, 33), (3, 128), (1, 256)][seed % 4] if room != "large" else (1, 20)
    cache = random_cache(g, blocks, heads, dim)
    before = contents(cache)
    got = fork_call(cache, None if keep is None else i32(keep), i32(table), i32(lens), i32(parent), i32(grow))
    want, lens_new, missing, copies = fork_expected(keep, table, lens, parent, grow, blocks)
    assert np.array_equal(got[0].cpu().numpy(), want)
    assert np.array_equal(got[1].cpu().numpy(), lens_new)
    assert int(got[2]) == missing
    for x, y in zip(contents(cache), moved_contents(before, copies)):
        assert torch.equal(x, y)


def test_fork_many_rows_and_blocks():
    """More rows and blocks than a workgroup counts at once, tables longer than a wave."""
    rnd = np.random.RandomState(1)
    B, n, width = 300, 2500, 150
    lens = rnd.randint(0, width * BLOCK, B)
    blocks = 60000
    table = rnd.permutation(blocks)[:B * width].reshape(B, width)
    parent, grow = rnd.randint(0, B, n), rnd.randint(0, 200, n)
    keep = (rnd.rand(blocks) < 0.01).astype(np.int32)
    cache = random_cache(gen(1), blocks, 1, 16)
    before = contents(cache)
    got = fork_call(cache, i32(keep), i32(table), i32(lens), i32(parent), i32(grow))
    want, lens_new, missing, copies = fork_expected(keep, table, lens, parent, grow, blocks)
    assert len(copies) > 2000 and missing == 0
    assert np.array_equal(got[0].cpu().numpy(), want) and np.array_equal(got[1].cpu().numpy(), lens_new) and int(got[2]) == 0
    after = moved_contents(before, copies)
    for x, y in zip(contents(cache), after):
        assert torch.equal(x, y)


def compact_expected(keep, table, lens, blocks):
    B, width = table.shape
    held = [-(-min(max(int(x), 0), width * BLOCK) // BLOCK) for x in lens]
    used = [keep is not None and bool(keep[i]) for i in range(blocks)]
    for b in range(B):
        for e in table[b, :held[b]]:
            if 0 <= e < blocks:
                used[e] = True
    count = sum(used)
    holes, late = [i for i in range(count) if not used[i]], [i for i in range(count, blocks) if used[i]]
    moved = np.array([i if used[i] else -1 for i in range(blocks)], np.int32)
    moved[late] = holes
    out = np.full((B, width), -1, np.int32)
    for b in range(B):
        for j, e in enumerate(table[b, :held[b]]):
            out[b, j] = moved[e] if 0 <= e < blocks else -1
    return out, moved, count, list(zip(late, holes))


@pytest.mark.parametrize("seed", range(16))
def test_compact(seed):
    """The last four with more blocks, or a larger table, than one workgroup does alone."""
    g = gen(200 + seed)
    rnd = np.random.RandomState(50 + seed)
    B, width = rnd.randint(1, 60), rnd.randint(1, 9)
    blocks = [1, 7, 1023, 1024, 1025, 5000][seed % 6]
    if seed >= 12:
        B, width, blocks = [(40, 5, 20000), (130, 130, 3000), (1, 1, 16385), (700, 30, 700)][seed - 12]
    lens = rnd.randint(-3, width * BLOCK + 10, B)
    table = rnd.randint(-2, blocks + 2, (B, width))
    keep = (rnd.rand(blocks) < [0.05, 0.5, 0.0][seed % 3]).astype(np.int32) if seed % 4 else None
    heads, dim = [(1, 64), (2, 33), (3, 128), (1, 256)][seed % 4] if seed < 12 else (2, 20)
    cache = random_cache(g, blocks, heads, dim)
    before = contents(cache)
    t = i32(table)
    new = t if seed % 2 else torch.full_like(t, 99)          # in place, too
    moved, used = torch.full((blocks,), 99, dtype=torch.int32, device=DEV), torch.full((1,), 99, dtype=torch.int32, device=DEV)
    ws = torch.full((mq.mq_kv_compact_ws_bytes(blocks),), 170, dtype=torch.uint8, device=DEV)
    mq.mq_kv_compact(cache, None if keep is None else i32(keep), t, width, i32(lens), B, new, moved, used, ws, ws.numel())
    want, at, count, copies = compact_expected(keep, table, lens, blocks)
    assert int(used) == count
    assert np.array_equal(moved.cpu().numpy(), at)
    assert np.array_equal(new.cpu().numpy(), want)
    for x, y in zip(contents(cache), moved_contents(before, copies)):
        assert torch.equal(x, y)


def test_blocks_past_four_gigabytes():
    """Copies, moves and attention at offsets that 32 bits do not hold."""
    heads, dim, blocks = 16, 256, 20000                      # 512 KB a block
    cache = mq.kv_cache(blocks, heads, dim, DEV)
    g = gen(3)
    for e in (19998, 19990):
        cache.keys[e] = torch.randint(-127, 128, cache.keys[e].shape, generator=g, dtype=torch.int8).to(DEV)
        cache.values[e] = torch.randint(-127, 128, cache.values[e].shape, generator=g, dtype=torch.int8).to(DEV)
        cache.amax[e] = 1.5
    table = np.array([[19990, 19998]], np.int32)
    keep = np.ones(blocks, np.int32)
    keep[[19999, 19990, 19998]] = 0
    keep[:3] = 0
    q = normal(g, 3, heads * dim).to(BF16).to(DEV)
    out = chunk_call(cache, i32(table), i32([0, 3]), i32([100]), 100, True, q, heads, 0.06)
    check_chunk(out, *chunk_expected(cache, table, [0, 3], [100], 100, True, q, heads, 0.06, BF16))
    keep[:3] = 1
    new, _, missing = fork_call(cache, i32(keep), i32(table), i32([100]), i32([0, 0]), i32([1, 1]))
    assert new.tolist() == [[19990, 19998], [19990, 19999]] and int(missing) == 0
    assert torch.equal(cache.keys[19999], cache.keys[19998]) and torch.equal(cache.values[19999], cache.values[19998])
    second = torch.empty_like(new)
    moved, used = torch.empty(blocks, dtype=torch.int32, device=DEV), torch.empty(1, dtype=torch.int32, device=DEV)
    ws = torch.empty(mq.mq_kv_compact_ws_bytes(blocks), dtype=torch.uint8, device=DEV)
    mq.mq_kv_compact(cache, None, new, 2, i32([100, 100]), 2, second, moved, used, ws, ws.numel())
    assert second.tolist() == [[0, 1], [0, 2]] and int(used) == 3
    again = chunk_call(cache, second[:1], i32([0, 3]), i32([100]), 100, True, q, heads, 0.06)
    assert torch.equal(again, out)


# ---- norm ---------------------------------------------------------------------------------------------------------------

def norm_expected(x, r, gamma, eps):
    h = x if r is None else (x.double() + r.double()).to(x.dtype)       # (one rounding: binary32 holds sums of 16-bit types well enough)
    if r is not None and x.dtype != F32:
        h = (x.float() + r.float()).to(x.dtype)
    z = h.double()
    return h, z / torch.sqrt((z * z).mean(-1, keepdim=True) + eps) * gamma.double()


NORMS = [(1, 1), (3, 8), (5, 33), (4, 512), (7, 513), (2, 777), (65, 1024), (3, 2048), (3, 2056), (9, 4096), (2, 5000), (2, 8192), (3, 16384), (1, 16383)]


def norm_inputs(g, M, d, dtype, residual, apart):
    """Rows with a pitch and an offset of their own where `apart`."""
    def rows(scale):
        if not apart:
            return (normal(g, M, d) * scale).to(dtype).to(DEV)
        store = torch.full((M * (d + 5) + 1,), math.nan, dtype=dtype, device=DEV)
        view = store[1:].view(M, d + 5)[:, :d]
        view.copy_((normal(g, M, d) * scale).to(dtype))
        return view
    return rows(1.0), rows(3.0) if residual else None, (0.5 + torch.rand(d, generator=g)).to(DEV)


# Sums of up to 64 squares one after the other and of 256 threads in a tree: (64 + 12) roundings, half of it after the root; the
# mean, the root, the quotient and two products one each.
NORM_REL = (76 / 2 + 5) * EPS32


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("residual,apart", [(True, False), (False, False), (True, True)])
@pytest.mark.parametrize("M,d", NORMS)
def test_norm(dtype, residual, apart, M, d):
    g = gen(M * 100003 + d)
    x, r, gamma = norm_inputs(g, M, d, dtype, residual, apart)
    code, ld = mq.dtype_code(dtype), x.stride(0) if M > 1 else max(d, x.stride(0))
    h_want, y_want = norm_expected(x, r, gamma, 1e-5)
    h = torch.full((M, d), 7.0, dtype=dtype, device=DEV)
    y = torch.full((M, d + 3), 7.0, dtype=dtype, device=DEV)
    mq.mq_add_rms_norm(x, ld, r, ld, code, gamma, M, d, 1e-5, h, d, y, d + 3)
    assert torch.equal(h, h_want.contiguous())
    assert (y[:, d:] == 7.0).all()
    off = (y[:, :d].double() - y_want).abs()
    assert (off <= y_want.abs() * NORM_REL + half_step(dtype, y_want)).all()
    # 8-bit rows
    h.fill_(7.0)
    q = torch.full((M, d + 3), 99, dtype=torch.int8, device=DEV)
    scale = torch.full((M,), 7.0, device=DEV)
    mq.mq_add_rms_norm_rows8(x, ld, r, ld, code, gamma, M, d, 1e-5, h, d, q, d + 3, scale)
    assert torch.equal(h, h_want.contiguous()) and (q[:, d:] == 99).all()
    s_want = 127 / y_want.abs().amax(-1)
    assert ((scale.double() - s_want).abs() <= s_want * (NORM_REL + 2 * EPS32)).all()
    assert ((q[:, :d].double() - y_want * s_want[:, None]).abs() <= 0.5 + 127 * (2 * NORM_REL + 4 * EPS32)).all()
    assert (q[:, :d].abs().amax(-1) == 127).all()
    # a packed operand
    s = torch.tensor([31.0], device=DEV)
    packed = torch.full((mq.mq_packed_bytes(8, M, d),), 99, dtype=torch.uint8, device=DEV)
    mq.mq_add_rms_norm_pack8(x, ld, r, ld, code, gamma, M, d, 1e-5, None, d, s, packed)
    ints = torch.empty((M, d), dtype=torch.int8, device=DEV)
    mq.mq_unpack_weight(packed, 8, M, d, ints)
    want = (y_want * 31.0).clamp(-127, 127)
    assert ((ints.double() - want).abs() <= 0.5 + 127 * (NORM_REL + 2 * EPS32)).all()
    clean = torch.empty_like(packed)
    mq.mq_quantize_pack_f32(ints.float(), M, d, 8, torch.ones(1, device=DEV), clean)
    assert torch.equal(packed, clean)                        # padding included


@pytest.mark.parametrize("dtype", TYPES)
def test_norm_of_odd_rows_and_in_place(dtype):
    g = gen(11)
    M, d, code = 6, 1000, mq.dtype_code(dtype)
    x, r, gamma = norm_inputs(g, M, d, dtype, True, False)
    x[1, 5], x[2, 999], r[3, 7] = math.nan, math.inf, -math.inf
    x[4], r[4] = 0, 0
    q, scale = torch.empty((M, d), dtype=torch.int8, device=DEV), torch.empty(M, device=DEV)
    mq.mq_add_rms_norm_rows8(x, d, r, d, code, gamma, M, d, 1e-5, None, d, q, d, scale)
    assert torch.isnan(scale[1:4]).all() and not q[1:5].any() and scale[4] == 1 and not torch.isnan(scale[[0, 5]]).any()
    y = torch.empty_like(x)
    mq.mq_add_rms_norm(x, d, r, d, code, gamma, M, d, 1e-5, None, d, y, d)
    h = (x.float() + r.float()).to(dtype)
    assert torch.isnan(y[1]).all() and torch.isnan(y[2, 999]) and torch.isnan(y[3, 7]) and (y[2, :999] == 0).all() and (y[4] == 0).all()
    # h over r, y over x
    x2, r2 = x.clone(), r.clone()
    mq.mq_add_rms_norm(x2, d, r2, d, code, gamma, M, d, 1e-5, r2, d, x2, d)
    assert torch.equal(r2.nan_to_num(3.0), h.nan_to_num(3.0)) and torch.equal(x2.nan_to_num(3.0), y.nan_to_num(3.0))


# ---- 4-bit parameters -------------------------------------------------------------------------------------------------------

def w4_inputs(g, N, K, group, zeros=True):
    groups = -(-K // group)
    codes = torch.randint(0, 16, (N, K), generator=g).to(torch.uint8)
    z = torch.randint(0, 16, (N, groups), generator=g).to(torch.uint8) if zeros else None
    s = ((0.2 + torch.rand((N, groups), generator=g)) / 8).bfloat16().float()
    at = torch.arange(K) // group
    w = (codes.double() - (z.double()[:, at] if zeros else 8)) * s.double()[:, at]
    return codes.to(DEV), s.to(DEV), None if z is None else z.to(DEV), w


@pytest.mark.parametrize("N,K,group,zeros", [(1, 1, 32, True), (16, 128, 128, False), (17, 129, 64, True), (100, 1000, 32, True), (33, 4096, 128, True)])
def test_w4_pack_and_unpack(N, K, group, zeros):
    codes, s, z, w = w4_inputs(gen(N + K), N, K, group, zeros)
    back = torch.empty((N, K), device=DEV)
    mq.mq_w4_unpack(mq.w4_pack(codes, s, z, group), N, K, group, back)
    assert torch.equal(back.cpu(), w.float())                # small whole numbers times bfloat16 scales: exact
    # the upper four bits of a code do not count; scales are rounded to 20 bits of mantissa, to nearest, ties to even
    mq.mq_w4_unpack(mq.w4_pack(codes + 48, s, z, group), N, K, group, back)
    assert torch.equal(back.cpu(), w.float())
    fine = s * (1 + torch.rand(s.shape, generator=gen(1)).to(DEV) * 0.1)
    one = torch.full_like(codes, 9)
    mq.mq_w4_unpack(mq.w4_pack(one, fine, None, group), N, K, group, back)
    bits = fine.cpu().numpy().view(np.uint32).astype(np.uint64)
    held = ((bits + 7 + (bits >> 4 & 1)) & 0xfffffff0).astype(np.uint32).view(np.float32)
    assert np.array_equal(back.cpu().numpy(), held[:, np.arange(K) // group])


@pytest.mark.parametrize("N,K,group", [(1, 1, 32), (16, 128, 128), (35, 200, 64), (100, 1000, 32)])
def test_w4_prepare(N, K, group):
    w = normal(gen(N), N, K)
    w[0, 0] = 0
    if N > 1:
        w[1] = 0
        w[2, 5] = math.nan
    back = torch.empty((N, K), device=DEV)
    mq.mq_w4_unpack(mq.w4_prepare(w.to(DEV), group), N, K, group, back)
    want = np.zeros((N, K), np.float32)
    for k in range(0, K, group):
        x = np.nan_to_num(w.numpy()[:, k:k + group], nan=0.0)
        bits = (np.abs(x).max(-1) / np.float32(7)).astype(np.float32).view(np.uint32)
        s = ((bits + 7 + (bits >> 4 & 1)) & 0xfffffff0).astype(np.uint32).view(np.float32)
        with np.errstate(all="ignore"):
            c = np.where(s[:, None] > 0, np.clip(np.rint(x / s[:, None]), -8, 7), 0)
        want[:, k:k + group] = c * s[:, None]
    assert np.array_equal(back.cpu().numpy(), want)


def product_tolerance(x, w_abs31, K, group, parts, out_type, y):
    """Operands and products are exact.  A group's sums, (16 + c) x and x, have up to group x parts terms, a result up to
    groups of them and the joins of up to 64 parts: roundings in binary32 of magnitudes up to sum |x| (16 + 15 + 16 + 15) s."""
    n = group * parts + -(-K // group) + 64
    return 2 * n * EPS32 / 2 * 2 * (x.abs() @ w_abs31.T) + half_step(out_type, y)


PRODUCTS = [
    # rows, words, width, group
    (1, 1, 1, 32), (1, 64, 4096, 128), (3, 100, 129, 64), (16, 48, 1000, 32), (17, 130, 777, 128), (5, 33, 5000, 64), (64, 256, 512, 128),
    (65, 31, 250, 32), (150, 65, 2048, 64), (2, 5000, 96, 32), (31, 16, 20000, 128), (200, 1000, 320, 64), (8, 1024, 11008, 128),
]


@pytest.mark.parametrize("xtype", ["rows8", F32, F16, BF16])
@pytest.mark.parametrize("case", range(len(PRODUCTS)))
def test_w4_product(xtype, case):
    M, N, K, group = PRODUCTS[case]
    g = gen(300 + case)
    codes, s, z, w = w4_inputs(g, N, K, group, case % 2 == 0)
    packed = mq.w4_pack(codes, s, z, group)
    bias = normal(g, N).to(DEV) if case % 3 else None
    ld = K + (0, 3, 8)[case % 3]
    if xtype == "rows8":
        x = torch.full((M, ld), 55, dtype=torch.int8, device=DEV)
        x[:, :K] = torch.randint(-127, 128, (M, K), generator=g).to(torch.int8)
        rs = (5 + 10 * torch.rand(M, generator=g)).to(DEV)
        x64 = x[:, :K].double().cpu() / rs.double().cpu()[:, None]
        code, parts, out_types = mq.MQ_ROWS8, 1, TYPES
    else:
        x = torch.full((M, ld), math.nan, dtype=xtype, device=DEV)
        x[:, :K] = normal(g, M, K).to(xtype)
        rs, x64, code, parts = None, x[:, :K].double().cpu(), mq.dtype_code(xtype), PARTS[xtype]
        out_types = [xtype, F32]
    y64 = x64 @ w.T + (0 if bias is None else bias.double().cpu())
    w31 = (62.0 * s.double().cpu())[:, torch.arange(K) // group]
    ws = torch.full((mq.mq_w4_product_ws_bytes(M, N, K),), 255, dtype=torch.uint8, device=DEV)
    for t in out_types:
        y = torch.full((M, N + 2), 7.0, dtype=t, device=DEV)
        mq.mq_w4_product(x, ld, code, rs, packed, M, N, K, group, bias, y, N + 2, mq.dtype_code(t), ws, ws.numel())
        assert (y[:, N:] == 7.0).all()
        off, tol = (y[:, :N].double().cpu() - y64).abs(), product_tolerance(x64, w31, K, group, parts, t, y64)
        assert (off <= tol).all(), float((off / tol).max())


def test_w4_product_keeps_bad_rows_apart():
    g = gen(12)
    M, N, K, group = 20, 70, 300, 64
    codes, s, z, _ = w4_inputs(g, N, K, group)
    packed = mq.w4_pack(codes, s, z, group)
    ws = torch.empty(mq.mq_w4_product_ws_bytes(M, N, K), dtype=torch.uint8, device=DEV)

    def product(x):
        y = torch.empty((M, N), dtype=x.dtype, device=DEV)
        mq.mq_w4_product(x, K, mq.dtype_code(x.dtype), None, packed, M, N, K, group, None, y, N, mq.dtype_code(x.dtype), ws, ws.numel())
        return y
    for t in TYPES:
        x = normal(g, M, K).to(t).to(DEV)
        good = product(x)
        x[3, 299], x[17, 0] = math.nan, math.inf
        bad = product(x)
        rest = [m for m in range(M) if m not in (3, 17)]
        assert torch.isnan(bad[3]).all() and not torch.isfinite(bad[17]).any() and torch.equal(bad[rest], good[rest])


@pytest.mark.parametrize("xtype", TYPES)
@pytest.mark.parametrize("M", [3, 40])
def test_w4_product_captured(xtype, M):
    g = gen(20)
    N, K, group = 200, 1024, 64
    codes, s, z, _ = w4_inputs(g, N, K, group)
    packed = mq.w4_pack(codes, s, z, group)
    ws = torch.full((2, mq.mq_w4_product_ws_bytes(M, N, K)), 255, dtype=torch.uint8, device=DEV)
    code, x = mq.dtype_code(xtype), torch.zeros((M, K), dtype=xtype, device=DEV)

    def product(y, ws):
        mq.mq_w4_product(x, K, code, None, packed, M, N, K, group, None, y, N, mq.MQ_F32, ws, ws.numel())
        return y
    out = product(torch.zeros((M, N), device=DEV), ws[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        product(out, ws[0])
    for i in range(3):
        x.copy_(normal(g, M, K).to(xtype))
        want = product(torch.zeros((M, N), device=DEV), ws[1])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and bool(out.any()), i


# ---- together -----------------------------------------------------------------------------------------------------------------

class Layer:
    """A decoder layer with everything in the library: norm to 8-bit rows, 4-bit products, the cache, attention of the new tokens."""

    def __init__(self, g, d, heads, kv_heads, dim, f, group):
        self.d, self.heads, self.kv_heads, self.dim, self.f, self.group = d, heads, kv_heads, dim, f, group
        self.width = (heads + 2 * kv_heads) * dim
        self.float = [normal(g, n, k) / math.sqrt(k) for n, k in ((self.width, d), (d, heads * dim), (f, d), (d, f))]
        self.packed = [mq.w4_prepare(w.to(DEV), group) for w in self.float]
        self.held = []
        for p, w in zip(self.packed, self.float):
            back = torch.empty(w.shape, device=DEV)
            mq.mq_w4_unpack(p, w.shape[0], w.shape[1], group, back)
            self.held.append(back.double().cpu())
        self.gamma = [(0.5 + torch.rand(d, generator=g)).to(DEV) for _ in range(2)]

    def run(self, x, cache, table, first, held, lens, B, max_len, stream=None):
        """x: float32 [T, d].  Only library calls and allocations."""
        T, d, dim = x.shape[0], self.d, self.dim

        def product(i, a, scale):
            n, k = self.float[i].shape
            y = torch.empty((T, n), device=DEV)
            ws = torch.empty(mq.mq_w4_product_ws_bytes(T, n, k), dtype=torch.uint8, device=DEV)
            mq.mq_w4_product(a, k, mq.MQ_F32 if scale is None else mq.MQ_ROWS8, scale, self.packed[i], T, n, k, self.group, None, y, n,
                             mq.MQ_F32, ws, ws.numel(), stream)
            return y

        def norm(a, r, gamma, h):
            q, s = torch.empty((T, d), dtype=torch.int8, device=DEV), torch.empty(T, device=DEV)
            mq.mq_add_rms_norm_rows8(a, d, r, d, mq.MQ_F32, gamma, T, d, 1e-6, h, d, q, d, s, stream)
            return q, s
        qkv = product(0, *norm(x, None, self.gamma[0], None))
        nq, nk = self.heads * dim, self.kv_heads * dim
        q, k, v = qkv[:, :nq], qkv[:, nq:nq + nk], qkv[:, nq + nk:]
        mq.mq_kv_append(cache, table, table.shape[1], first, held, B, T, k, self.width, v, self.width, None, self.width, self.heads,
                        mq.MQ_F32, None, 0, False, None, None, stream)
        ctx = torch.empty((T, nq), device=DEV)
        ws = torch.empty(mq.mq_chunk_attention_ws_bytes(B, T, max_len, self.heads, self.kv_heads, dim), dtype=torch.uint8, device=DEV)
        mq.mq_chunk_attention(cache, table, table.shape[1], first, lens, B, T, max_len, True, q, self.width, self.heads, mq.MQ_F32,
                              dim ** -0.5, ctx, nq, ws, ws.numel(), stream)
        h = torch.empty((T, d), device=DEV)
        mid = product(2, *norm(product(1, ctx, None), x, self.gamma[1], h)).relu_()
        return h + product(3, mid, None), q, k, v


def layer_expected(layer, x, past, first):
    """The same in 64 bits without the cache's rounding: (outputs, keys and values by sequence)."""
    W, d, dim, hk, per = layer.held, layer.d, layer.dim, layer.kv_heads, layer.heads // layer.kv_heads
    norm = lambda a, gamma: a / torch.sqrt((a * a).mean(-1, keepdim=True) + 1e-6) * gamma.double().cpu()  # noqa: E731
    qkv = norm(x, layer.gamma[0]) @ W[0].T
    nq, nk = layer.heads * dim, hk * dim
    ctx, now = torch.zeros(len(x), layer.heads, dim, dtype=torch.float64), []
    for b in range(len(first) - 1):
        rows = slice(first[b], first[b + 1])
        k, v = (torch.cat([old, new.reshape(-1, hk, dim)]) for old, new in zip(past[b], (qkv[rows, nq:nq + nk], qkv[rows, nq + nk:])))
        now.append((k, v))
        n, m = first[b + 1] - first[b], len(k)
        q = qkv[rows, :nq].view(n, layer.heads, dim)
        for h in range(layer.heads):
            s = q[:, h] @ k[:, h // per].T / math.sqrt(dim)
            s = s.masked_fill(torch.arange(m)[None, :] > torch.arange(n)[:, None] + m - n, -math.inf)
            ctx[rows, h] = torch.softmax(s, dim=-1) @ v[:, h // per]
    h = x + ctx.view(len(x), -1) @ W[1].T
    return h + torch.relu(norm(h, layer.gamma[1]) @ W[2].T) @ W[3].T, now


def test_decoding_with_forks_and_compaction():
    """Prompts in two pieces, three hypotheses begun to each, reordered, moved to the cache's front, continued: the outputs follow the
    layer in 64 bits.  8-bit rows and caches are off by half a step of 127 of the largest element each, about 1 % of a typical
    one; through two products that average them and a softmax the outputs stay within 5 % of their size in the 2-norm."""
    g = gen(13)
    heads, kv_heads, dim, d, f = 8, 2, 64, 256, 512
    layer = Layer(g, d, heads, kv_heads, dim, f, 64)
    blocks, width = 64, 4
    cache = mq.kv_cache(blocks, kv_heads, dim, DEV)
    table = torch.full((2, width), -1, dtype=torch.int32, device=DEV)
    lens = i32([0, 0])
    past = [(torch.zeros(0, kv_heads, dim, dtype=torch.float64),) * 2 for _ in range(2)]
    lengths = [0, 0]

    def step(parents, news):
        """One call of everything for rows that continue `parents` with so many new tokens."""
        nonlocal table, lens, past, lengths
        table, held, missing = fork_call(cache, None, table, lens, i32(parents), i32(news))
        assert int(missing) == 0
        lengths = [lengths[p] for p in parents]
        past = [past[p] for p in parents]
        assert held.tolist() == lengths
        first = np.concatenate([[0], np.cumsum(news)])
        x = normal(g, int(first[-1]), d).to(DEV)
        lens = held + i32(news)
        lengths = [a + n for a, n in zip(lengths, news)]
        out, *_ = layer.run(x, cache, table, i32(first), held, lens, len(news), width * BLOCK)
        want, past = layer_expected(layer, x.double().cpu(), past, first.tolist())
        off = float(torch.linalg.norm(out.double().cpu() - want) / torch.linalg.norm(want))
        assert off <= 0.05, off

    step([0, 1], [70, 41])
    step([0, 1], [30, 23])                                   # 100 and 64 tokens
    step([0, 0, 0, 1, 1, 1], [1] * 6)                        # three of each
    step([2, 0, 2, 3, 5], [1, 2, 1, 1, 3])                   # reordered, one dropped
    used, moved = torch.empty(1, dtype=torch.int32, device=DEV), torch.empty(blocks, dtype=torch.int32, device=DEV)
    ws = torch.empty(mq.mq_kv_compact_ws_bytes(blocks), dtype=torch.uint8, device=DEV)
    mq.mq_kv_compact(cache, None, table, width, lens, 5, table, moved, used, ws, ws.numel())
    assert int(table.max()) == int(used) - 1
    step([0, 1, 2, 3, 4], [1, 1, 1, 1, 1])
    step([4, 4, 1], [2, 5, 1])


def test_a_captured_step_and_two_streams():
    """Fork, append, attention and products of a step in one graph, replayed; another stream works beside it."""
    g = gen(14)
    heads, kv_heads, dim, d, f = 8, 2, 64, 256, 512
    layer = Layer(g, d, heads, kv_heads, dim, f, 32)
    B, width, blocks = 6, 3, 40
    start = random_cache(g, blocks, kv_heads, dim)
    table0, lens0 = i32(tables(g, [100, 64, 1, 130, 63, 128], width, blocks)), i32([100, 64, 1, 130, 63, 128])
    x, parent, grow, first = torch.zeros((2 * B, d), device=DEV), i32(range(B)), i32([2] * B), i32(range(0, 2 * B + 1, 2))

    def one(cache):
        table, held, missing = fork_call(cache, None, table0, lens0, parent, grow)
        out, *_ = layer.run(x, cache, table, first, held, held + 2, B, width * BLOCK)
        return out, table, missing

    def fresh():
        c = mq.kv_cache(blocks, kv_heads, dim, DEV)
        for a, b in zip((c.keys, c.values, c.amax), contents(start)):
            a.copy_(b)
        return c
    cache = fresh()
    one(cache)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held_out = one(cache)
    side = torch.cuda.Stream()
    for i in range(4):
        x.copy_(normal(g, 2 * B, d))
        parent.copy_(torch.randint(0, B, (B,), generator=g).to(torch.int32))
        clean, other = fresh(), fresh()
        want = one(clean)
        for a, b in zip((cache.keys, cache.values, cache.amax), contents(start)):
            a.copy_(b)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            beside = one(other)
        graph.replay()
        torch.cuda.synchronize()
        for got in (held_out, beside):
            for a, b in zip(got, want):
                assert torch.equal(a, b), i
        for c in (cache, other):
            for a, b in zip(contents(c), contents(clean)):
                assert torch.equal(a, b), i
