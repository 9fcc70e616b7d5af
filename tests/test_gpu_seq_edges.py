"""The sequence operators (include/mq_seq.h) on the GPU where memory holds anything, where a softmax's reference moves, where
probabilities are subnormal, and in replays that find nothing of an earlier run.  Tolerances as in test_gpu_seq.py.
"""
import math

import pytest
import torch

import paper_1805_12096_amd as mq
import test_gpu_seq as base

pytestmark = pytest.mark.gpu

DEV, BLOCK = base.DEV, base.BLOCK
F32, F16, BF16 = base.F32, base.F16, base.BF16
TYPES = base.TYPES


# ---- the cache ----------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("held", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("heads,hk,dim", [(8, 8, 64), (4, 1, 128), (2, 2, 33), (4, 2, 256)])
@pytest.mark.parametrize("lens", [[100, 200, 64, 190], [2000], [9000, 700, 0, 64], [300, 190]])
def test_cached_attention_reads_nothing_of_blocks_that_are_not_there(lens, heads, hk, dim, held, dtype):
    # memory as it was allocated: block 0 belongs to nobody and has never been written
    g = base.gen(dim + len(lens))
    B = len(lens)
    need = [-(-n // BLOCK) for n in lens]
    c = base.filled_cache(g, sum(need) + 1, hk, dim)
    order = (torch.randperm(sum(need), generator=g) + 1).tolist()
    table = torch.full((B, max(need)), -1, dtype=torch.int32)
    for b in range(B):
        for i in range(need[b]):
            table[b, i] = order.pop()
    # entries that are no block: the first of a sequence, one further on, a whole sequence's
    table[0, 0] = -1
    table[0, need[0] - 1] = c.blocks
    if need[0] > 20:
        table[0, 10:17] = 1 << 30
    if B > 2:
        table[2] = -1
    q = base.normal(g, B, heads * dim).to(dtype)
    want, tol = base.cached_reference(c, table, lens, max(lens), q, heads, dim ** -0.5)
    c.amax[0] = held
    c.keys[0], c.values[0] = -128, -128
    got = base.cached(c, table.to(DEV), base.i32(lens), max(lens), q.to(DEV), heads, dim ** -0.5).cpu().double()
    assert ((got - want).abs() <= tol).all()
    if B > 2:
        assert (got[2] == 0).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_cached_attention_of_more_blocks_than_a_wave_reads_at_once(dtype):
    # many sequences of which one is long: it stays in one run, and a wave of it has more than 64 blocks
    g = base.gen(71)
    B, hk, dim, n = 520, 1, 64, 20_000
    lens = [3] * B
    lens[300], lens[301], lens[302] = n, n - 1, 64 * 256 + 1
    c = base.filled_cache(g, 400, hk, dim)
    table = torch.randint(0, 400, (B, -(-n // BLOCK)), generator=g, dtype=torch.int32)
    q = base.normal(g, B, 2 * dim).to(dtype)
    want, tol = base.cached_reference(c, table, lens, n, q, 2, dim ** -0.5)
    got = base.cached(c, table.to(DEV), base.i32(lens), n, q.to(DEV), 2, dim ** -0.5).cpu().double()
    assert ((got - want).abs() <= tol).all()


@pytest.mark.parametrize("lens", [[100, 0, 64], [9000, 33]])       # one launch, two
def test_cached_attention_in_place(lens):
    g = base.gen(72)
    heads, hk, dim = 20, 1, 128
    blocks = 160
    c = base.filled_cache(g, blocks, hk, dim)
    table = torch.randint(0, blocks, (len(lens), -(-max(lens) // BLOCK)), generator=g, dtype=torch.int32)
    q = base.normal(g, len(lens), heads * dim)
    want, tol = base.cached_reference(c, table, lens, max(lens), q, heads, 0.1)
    qd, ld = q.to(DEV), heads * dim
    n = mq.mq_cached_attention_ws_bytes(len(lens), max(lens), heads, hk, dim)
    ws = torch.full((n,), 255, dtype=torch.uint8, device=DEV)
    mq.mq_cached_attention(c, table.to(DEV), table.shape[1], base.i32(lens), len(lens), max(lens), qd, ld, heads, 0, 0.1, qd, ld, ws, n)
    assert ((qd.cpu().double() - want).abs() <= tol).all()


# ---- packed sequences ---------------------------------------------------------------------------------------------------

FORMS = [(150, 7), (300, 0), (1600, 0)]          # queries and keys, empty sequences behind: one launch, packed, long


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,others", FORMS)
@pytest.mark.parametrize("scale", [0.125, -0.125])
def test_prompt_attention_of_infinite_queries_is_nan(n, others, scale, dtype):
    # an infinite element makes every score infinite; scores of which all are minus infinity have no softmax either
    g = base.gen(51)
    heads, hk, dim = 2, 1, 64
    q, k, v = (base.normal(g, n, h * dim).to(dtype) for h in (heads, hk, hk))
    k[:, 3] = k[:, 3].abs() + 1
    for row, x in ((0, math.inf), (20, -math.inf), (n - 1, -math.inf), (n - 2, math.inf)):
        q[row, 3] = x
    ends = [0] + [n] * (1 + others)
    for causal in (True, False):
        got = base.prompt(q.to(DEV), k.to(DEV), v.to(DEV), ends, ends, heads, hk, dim, causal, scale).cpu()
        for row in (0, 20, n - 1, n - 2):
            assert torch.isnan(got[row, :dim]).all(), (row, causal)
            assert torch.isfinite(got[row, dim:]).all()
        assert torch.isfinite(got[1:20]).all() and torch.isfinite(got[21:n - 2]).all()
    # queries that see nothing give zeros, whatever they hold
    kends = [0] + [n - 30] * (1 + others)
    got = base.prompt(q.to(DEV), k.to(DEV), v.to(DEV), ends, kends, heads, hk, dim, True, scale).cpu()
    assert (got[:30] == 0).all() and torch.isnan(got[n - 2:, :dim]).all()


def grown(g, n, dim, jumps, dtype):
    """Queries, keys and values [n, dim] whose scores move by whole steps of about 8 (natural logarithm) at the units of 32
    keys named by `jumps`, up for some queries, down for others, hardly for the rest."""
    q, k, v = (base.normal(g, n, dim) for _ in range(3))
    q[:, 0] = torch.tensor([1.0, -1.0, 0.5, 0.02, 1.0])[torch.arange(n) % 5]
    level = torch.zeros(n)
    for unit in jumps:
        level[32 * unit:] += 8.0
    k[:, 0] = level * math.sqrt(dim)
    return q.to(dtype), k.to(dtype), v.to(dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [32, 64, 96, 128])
@pytest.mark.parametrize("jumps", [[1, 2, 3, 10, 21], [1, 4, 5, 36], [2, 47, 48, 49]])
@pytest.mark.parametrize("causal", [False, True])
def test_prompt_attention_of_growing_scores(causal, jumps, dim, dtype):
    # the reference of the softmax moves by far more than its slack at odd and even units, and what is held so far with it
    g = base.gen(dim + len(jumps))
    for n in (1601, 600):
        q, k, v = grown(g, n, dim, jumps, dtype)
        want, tol = base.prompt_reference(q, k, v, [0, n], [0, n], 1, 1, dim, causal, dim ** -0.5)
        got = base.prompt(q.to(DEV), k.to(DEV), v.to(DEV), [0, n], [0, n], 1, 1, dim, causal, dim ** -0.5).cpu().double()
        assert ((got - want).abs() <= tol).all(), n


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [32, 128])
@pytest.mark.parametrize("strong", [0, 1000, 1599])
@pytest.mark.parametrize("n,others", FORMS)
def test_prompt_attention_small_probabilities_of_a_long_run(n, others, strong, dim, dtype):
    # one key far above all others, whose probabilities are 2^-15 .. 2^-22 of its (subnormal as binary16) and whose values are all
    # there is.  Half a step of a subnormal binary16 is 2^-25, of a sum of at least 1.
    strong = min(strong, n - 1)
    m = n
    q, k, v = torch.zeros(n, dim), torch.zeros(m, dim), torch.ones(m, dim)
    q[:, 0] = torch.linspace(15, 22, n) * math.log(2)
    k[strong, 0] = 1
    v[strong] = 0
    q, k, v = (x.to(dtype) for x in (q, k, v))
    ends = [0] + [n] * (1 + others)
    want, tol = base.prompt_reference(q, k, v, ends, ends, 1, 1, dim, False, 1.0)
    # values are all alike, so an output is as far off, in proportion, as a probability: half a step of the type, or 2^-25 as
    # subnormal binary16; half a step for the output's own rounding; binary32 sums, of at most m terms above (m EPS32 / 2 of the
    # result, additions of at most half a step of a partial sum each) and m / 2 in a lane below (m EPS32 / 4); exponents of up to 22
    # after three roundings (22 ln 2 3 EPS32 / 2 = 23 EPS32), and the exponential's and the quotient's own
    tol = (torch.finfo(dtype).eps + (m + 64) * base.EPS32) * want.abs() + (m * 2.0 ** -25 if dtype == F16 else 0)
    got = base.prompt(q.to(DEV), k.to(DEV), v.to(DEV), ends, ends, 1, 1, dim, False, 1.0).cpu().double()
    assert ((got - want).abs() <= tol).all(), float(((got - want).abs() / want.abs()).max())


# ---- many sequences, and all of it together -------------------------------------------------------------------------------

def test_more_sequences_than_two_steps_of_the_search():
    # 64 x 64 entries are two steps of the search for a row's sequence; here it takes three
    B, dim = 270_000, 16
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    x = torch.randn(B, 3 * dim, generator=g, device=DEV)
    q, k, v = (x[:, i * dim:(i + 1) * dim] for i in range(3))
    n = torch.ones(B, dtype=torch.int64, device=DEV)
    n[::7] = 0
    n[1::7] = 2
    first = torch.cat([torch.zeros(1, dtype=torch.int64, device=DEV), n.cumsum(0)]).to(torch.int32)
    T = int(first[-1])
    assert T <= B
    out = base.prompt(q[:T], k[:T], v[:T], first, first, 1, 1, dim, True, 0.25)
    starts = first[:-1][n > 0].long()
    assert torch.equal(out[starts], v[starts])           # a sequence's first token sees itself alone
    cache = mq.kv_cache(B, 1, dim, DEV)
    table = torch.arange(B, dtype=torch.int32, device=DEV).flip(0).view(B, 1)
    zero = torch.zeros(B, dtype=torch.int32, device=DEV)
    base.append(cache, table, first, zero, None, k[:T], v[:T], 1)
    a = torch.full((B,), 0.0, device=DEV)
    rows = torch.arange(B, device=DEV).repeat_interleave(n)
    a.index_reduce_(0, rows, k[:T].abs().amax(1), "amax")
    there = n > 0
    assert torch.equal(cache.amax.view(B, 2)[:, 0].flip(0)[there], a[there])
    got = base.cached(cache, table, n.to(torch.int32), 2, q.contiguous(), 1, 0.25)
    one = n == 1
    step = cache.amax.view(B, 2)[:, 1].flip(0)[:, None] / 127
    assert ((got - v[first[:-1].long().clamp(max=B - 1)]).abs() <= 0.51 * step + 1e-6 * step.abs() * 127)[one].all()
    assert (got[n == 0] == 0).all()


def forget(s):
    """Everything that a run writes holds something else, and the cache what it had before the first run."""
    for x in (s.qkv, s.qkv1, s.kr, s.qr, s.kr1, s.qr1, s.o, s.o1, s.lp, s.ent, s.alt, s.sa):
        x.fill_(math.nan)
    s.tok.fill_(-1)
    for x in (s.pa, s.wl, s.wp, s.wc, s.ws, s.wq):
        x.fill_(255)
    for x in (s.cache.keys, s.cache.values, s.cache.amax):
        x.zero_()


def test_captured_steps_write_everything_they_should():
    one, eager = base.Step(), base.Step()
    eager.run()
    torch.cuda.synchronize()
    want = eager.results()
    one.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        one.run()
    for _ in range(4):
        forget(one)
        graph.replay()
        forget(eager)
        eager.run()
        torch.cuda.synchronize()
        for s in (one, eager):
            for x, y in zip(s.results(), want):
                assert torch.equal(x, y)


def test_two_streams_write_everything_they_should():
    steps = [base.Step(), base.Step()]
    steps[0].run()
    torch.cuda.synchronize()
    want = steps[0].results()
    for s in steps:
        forget(s)
    torch.cuda.synchronize()
    for s, at in zip(steps, (torch.cuda.Stream(), torch.cuda.Stream())):
        with torch.cuda.stream(at):
            s.run()
    torch.cuda.synchronize()
    for s in steps:
        for x, y in zip(s.results(), want):
            assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_prompt_and_next_token_in_sixteen_bits(dtype):
    # rotated keys and queries of the append go on to the attention of the prompt and, a token later, of the cache; captured as well
    g = base.gen(61)
    heads, hk, dim, n = 8, 2, 128, [200, 1, 64, 333]
    f = [0, 200, 201, 265, 598]
    T, B, D, W = f[-1], 4, 8 * 128, (8 + 4) * 128
    x, y = base.normal(g, T, W).to(dtype), base.normal(g, B, W).to(dtype)
    xd, yd = x.to(DEV), y.to(DEV)
    freq = torch.tensor([10000.0 ** (-2 * i / dim) for i in range(dim // 2)], dtype=F32)
    table = torch.arange(B * 6, dtype=torch.int32).flip(0).view(B, 6)
    fd, held, after, zero, td = base.i32(f), base.i32(n), base.i32([i + 1 for i in n]), base.i32([0] * B), table.to(DEV)
    cache = base.make_cache(B * 6, hk, dim)
    e = lambda rows, cols: torch.empty((rows, cols), dtype=dtype, device=DEV)  # noqa: E731
    kr, qr, o, kr1, qr1, o1 = e(T, hk * dim), e(T, D), e(T, D), e(B, hk * dim), e(B, D), e(B, D)
    t = mq.dtype_code(dtype)
    wp = torch.empty(mq.mq_prompt_attention_ws_bytes(t, B, T, hk, dim), dtype=torch.uint8, device=DEV)
    wc = torch.empty(mq.mq_cached_attention_ws_bytes(B, 384, heads, hk, dim), dtype=torch.uint8, device=DEV)
    fq = freq.to(DEV)

    def run():
        for z, first, at, rows, k_out, q_out in ((xd, fd, zero, T, kr, qr), (yd, None, held, B, kr1, qr1)):
            q, k, v = z[:, :D], z[:, D:D + hk * dim], z[:, D + hk * dim:]
            mq.mq_kv_append(cache, td, 6, first, at, B, rows, k, W, v, W, q, W, heads, t, fq, dim, False, k_out, q_out)
        mq.mq_prompt_attention(qr, D, kr, hk * dim, xd[:, D + hk * dim:], W, t, fd, fd, B, T, T, heads, hk, dim, True, dim ** -0.5, o, D,
                               wp, wp.numel())
        mq.mq_cached_attention(cache, td, 6, after, B, 384, qr1, D, heads, t, dim ** -0.5, o1, D, wc, wc.numel())

    run()
    torch.cuda.synchronize()
    for b in range(B):
        for z, rows, pos, kk, qq in ((x, slice(f[b], f[b + 1]), torch.arange(n[b]), kr, qr), (y, slice(b, b + 1), torch.tensor([n[b]]), kr1, qr1)):
            k = base.rotated(z[rows, D:D + hk * dim].reshape(-1, hk, dim), pos, freq, dim, False).float().to(dtype)
            q = base.rotated(z[rows, :D].reshape(-1, heads, dim), pos, freq, dim, False).float().to(dtype)
            assert torch.equal(kk[rows].cpu().view(-1, hk, dim), k) and torch.equal(qq[rows].cpu().view(-1, heads, dim), q)
    want, tol = base.prompt_reference(qr.cpu(), kr.cpu(), x[:, D + hk * dim:], f, f, heads, hk, dim, True, dim ** -0.5)
    assert ((o.cpu().double() - want).abs() <= tol).all()
    want, tol = base.cached_reference(cache, table, [i + 1 for i in n], 384, qr1.cpu(), heads, dim ** -0.5)
    assert ((o1.cpu().double() - want).abs() <= tol).all()
    eager = [z.clone() for z in (kr, qr, o, kr1, qr1, o1, cache.keys, cache.values, cache.amax)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for _ in range(3):
        for z in (kr, qr, o, kr1, qr1, o1):
            z.fill_(math.nan)
        wp.fill_(255), wc.fill_(255)
        cache.keys.fill_(77), cache.values.fill_(-78), cache.amax.fill_(123.0)
        graph.replay()
        torch.cuda.synchronize()
        for z, w in zip((kr, qr, o, kr1, qr1, o1, cache.keys, cache.values, cache.amax), eager):
            assert torch.equal(z, w)
