"""The sequence operators (include/mq_seq.h) on the GPU against plain implementations in 64 bits.

Tolerances come from the number formats, before any run.  With eps = torch.finfo(type).eps a rounding to the type is off by at
most eps / 2 of the value.  Errors of scores (natural logarithms) enter an attention's output as exp(2 error) - 1 times the
largest value, errors of probabilities in proportion.
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


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def normal(g, *shape):
    return torch.randn(shape, generator=g)


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def place(t):
    return 16 * ((t // 4) % 4) + 4 * (t // 16) + t % 4


PLACES = [place(t) for t in range(BLOCK)]


# ---- append -----------------------------------------------------------------------------------------------------------

class Blocks:
    """The cache's rule, token rows one after the other, in binary32 where the library says binary32."""

    def __init__(self, blocks, heads, dim):
        self.q = [np.zeros((blocks, heads, BLOCK, dim), np.int8) for _ in range(2)]
        self.amax = np.zeros((blocks, heads, 2), np.float32)

    def append(self, table, held, rows):
        """rows: (keys, values) binary32 [n, heads, dim] of one sequence, at positions held .."""
        n = rows[0].shape[0]
        at = held
        while at < held + n:
            end = min((at // BLOCK + 1) * BLOCK, held + n)
            col, lo = at // BLOCK, at % BLOCK
            block = table[col] if 0 <= col < len(table) else -1
            if 0 <= block < len(self.amax):
                for w in range(2):
                    x = rows[w][at - held:end - held].astype(np.float32)
                    for h in range(x.shape[1]):
                        finite = np.where(np.isfinite(x[:, h]), np.abs(x[:, h]), 0)
                        a = np.float32(finite.max())
                        had = self.amax[block, h, w]
                        if lo == 0:
                            self.q[w][block, h] = 0
                        else:
                            a = max(a, had)
                            if a > had:
                                r = np.float32(had) / np.float32(a)
                                self.q[w][block, h] = np.clip(np.rint(self.q[w][block, h].astype(np.float32) * r), -127, 127)
                        with np.errstate(all="ignore"):
                            y = np.rint(x[:, h] * (np.float32(127) / a if a > 0 else np.float32(1)))
                        y = np.where(np.isnan(y), 0, np.clip(y, -127, 127))
                        self.q[w][block, h, lo:lo + end - at] = y.astype(np.int8)
                        self.amax[block, h, w] = a
            at = end


def rotated(x, pos, freq, rot, interleaved):
    """x [n, heads, dim] in 64 bits."""
    x = x.double().clone()
    if rot:
        a = pos.double()[:, None, None] * freq.double()
        one, two = (range(0, rot, 2), range(1, rot, 2)) if interleaved else (range(rot // 2), range(rot // 2, rot))
        u, v = x[..., list(one)], x[..., list(two)]
        x[..., list(one)], x[..., list(two)] = u * a.cos() - v * a.sin(), u * a.sin() + v * a.cos()
    return x


def cache_ints(cache):
    """(keys, values) as [blocks, heads, 64, dim]."""
    d = cache.head_dim
    return [cache.keys[..., :d].cpu().numpy(), cache.values.transpose(2, 3)[:, :, PLACES, :d].cpu().numpy()]


def make_cache(blocks, heads, dim):
    """One whose every byte is set to something, as memory that has been in use."""
    c = mq.kv_cache(blocks, heads, dim, DEV)
    c.keys.fill_(77)
    c.values.fill_(-78)
    c.amax.fill_(123.0)
    return c


def append(cache, table, first, held, q, k, v, heads, freq=None, rot=0, interleaved=False, outs=True, stream=None):
    B, T, t = table.shape[0], k.shape[0], mq.dtype_code(k.dtype)
    k_out = torch.full((T, cache.kv_heads * cache.head_dim), 9.0, dtype=k.dtype, device=DEV) if outs else None
    q_out = torch.full((T, heads * cache.head_dim), 9.0, dtype=k.dtype, device=DEV) if q is not None else None
    mq.mq_kv_append(cache, table, table.shape[1], first, held, B, T, k, k.stride(0), v, v.stride(0), q,
                    q.stride(0) if q is not None else 0, heads, t, freq, rot, interleaved, k_out, q_out, stream)
    return k_out, q_out


CASES = [  # heads, kv heads, dim, rot, interleaved, new tokens, held
    (8, 8, 64, 0, False, [1, 1, 1, 1, 1], [0, 5, 63, 64, 130]),
    (4, 1, 128, 128, False, [3, 0, 70, 1, 200, 64], [0, 7, 60, 127, 33, 64]),
    (6, 2, 96, 64, True, [65, 1, 128, 2], [63, 63, 0, 190]),
    (1, 1, 1, 0, False, [130, 5], [0, 1]),
    (2, 1, 33, 8, True, [17, 90], [40, 3]),
    (2, 2, 256, 256, False, [64, 65, 1], [0, 10, 2]),
    (16, 4, 80, 40, False, [9] * 70, list(range(70))),
    (8, 4, 128, 64, True, [1] * 30 + [40, 1, 0, 3], list(range(25, 59))),       # few tokens to a block, but for one
    (4, 2, 256, 256, False, [1, 1, 7, 1, 20], [63, 64, 60, 127, 50]),
    (2, 2, 48, 16, False, [64, 128, 1], [0, 32, 5]),
    (4, 2, 160, 32, True, [100, 33], [0, 64]),
    (66, 2, 128, 128, True, [1] * 20 + [5, 1], list(range(50, 72))),            # several waves to a token's queries
    (40, 8, 128, 128, False, [90, 3], [5, 60]),
    (4, 4, 64, 64, False, [8, 1, 8, 3, 8, 8, 0, 4], [0, 60, 61, 64, 3, 59, 9, 0]),       # several to a block, but few
]


@pytest.mark.parametrize("extra", [5, 16])           # rows of any alignment, and of whole 16-byte pieces
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("case", CASES)
def test_append_is_the_rule_bit_for_bit(case, dtype, extra):
    heads, hk, dim, rot, inter, new, held = case
    g = gen(sum(new) + dim)
    B, rounds = len(new), 3
    need = [-(-(h + rounds * n) // BLOCK) for n, h in zip(new, held)]
    blocks, width = sum(need) + 2, max(need)
    order = torch.randperm(blocks, generator=g).tolist()
    table = torch.full((B, width), -1, dtype=torch.int32)
    for b in range(B):
        for i in range(need[b]):
            table[b, i] = order.pop()
    cache, model = make_cache(blocks, hk, dim), Blocks(blocks, hk, dim)
    for w, fill in enumerate((77, -78)):
        model.q[w][:] = fill
    model.amax[:] = 123.0
    freq = torch.tensor(10000.0 ** (-np.arange(0, rot, 2) / max(rot, 1)), dtype=F32)
    # front and back rows that belong to nobody, and columns of one wide product
    front, back = 2, 3
    width_all = (heads + 2 * hk) * dim + extra
    at = list(held)
    for step in range(rounds):
        T = sum(new) + front + back
        x = (normal(g, T, width_all) * (1 + 2 * step)).to(dtype)
        first = np.cumsum([front] + new)
        q, k, v = (x[:, a * dim:b * dim] for a, b in ((0, heads), (heads, heads + hk), (heads + hk, heads + 2 * hk)))
        xd = x.to(DEV)
        qd, kd, vd = (xd[:, a * dim:b * dim] for a, b in ((0, heads), (heads, heads + hk), (heads + hk, heads + 2 * hk)))
        k_out, q_out = append(cache, table.to(DEV), i32(first), i32(at), qd, kd, vd, heads, freq.to(DEV) if rot else None, rot, inter)
        torch.cuda.synchronize()
        for b in range(B):
            rows = slice(first[b], first[b + 1])
            pos = torch.arange(at[b], at[b] + new[b])
            kr = rotated(k[rows].reshape(-1, hk, dim), pos, freq, rot, inter).float()
            qr = rotated(q[rows].reshape(-1, heads, dim), pos, freq, rot, inter).float()
            model.append(table[b].tolist(), at[b], (kr.numpy(), v[rows].reshape(-1, hk, dim).float().numpy()))
            assert torch.equal(k_out[rows].cpu().view(-1, hk, dim), kr.to(dtype))
            assert torch.equal(q_out[rows].cpu().view(-1, heads, dim), qr.to(dtype))
            at[b] += new[b]
        for outside in (slice(0, front), slice(T - back, T)):
            assert (k_out[outside] == 9).all() and (q_out[outside] == 9).all()
        ints = cache_ints(cache)
        assert np.array_equal(ints[0], model.q[0]) and np.array_equal(ints[1], model.q[1])
        assert np.array_equal(cache.amax.cpu().numpy(), model.amax)
    # padding of the blocks written is zero, of others untouched
    used = sorted({int(table[b, i]) for b in range(B) for i in range(held[b] // BLOCK, need[b])})
    fresh = [int(table[b, i]) for b in range(B) for i in range(-(-held[b] // BLOCK), need[b])]
    if fresh:
        assert (cache.keys[fresh][..., dim:] == 0).all() and (cache.values[fresh][:, :, dim:] == 0).all()
    rest = [i for i in range(blocks) if i not in used]
    assert (cache.keys[rest] == 77).all() and (cache.values[rest] == -78).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_append_one_token_each_without_a_list(dtype):
    g = gen(5)
    hk, dim, B = 3, 64, 9
    held = [0, 1, 62, 63, 64, 65, 127, 128, 300]
    table = torch.arange(B * 5, dtype=torch.int32).flip(0).view(B, 5)
    one, two = make_cache(B * 5, hk, dim), make_cache(B * 5, hk, dim)
    k, v = normal(g, B, hk * dim).to(dtype).to(DEV), normal(g, B, hk * dim).to(dtype).to(DEV)
    append(one, table.to(DEV), None, i32(held), None, k, v, hk)
    append(two, table.to(DEV), i32(range(B + 1)), i32(held), None, k, v, hk)
    assert torch.equal(one.keys, two.keys) and torch.equal(one.values, two.values) and torch.equal(one.amax, two.amax)
    # blocks that start anew took the new maximum, others keep the larger one they had
    assert all((one.amax[int(table[b, held[b] // BLOCK])] < 10).all() == (held[b] % BLOCK == 0) for b in range(B))


def test_append_special_values():
    hk, dim = 1, 64
    x = torch.zeros(5, dim)
    x[0, :6] = torch.tensor([1.0, -2.0, math.nan, math.inf, -math.inf, 1e-30])
    x[2] = 1e-42                                     # subnormal
    x[3] = -3.4e38
    x[4] = math.nan
    table = torch.arange(5, dtype=torch.int32).view(5, 1)
    cache, model = make_cache(5, hk, dim), Blocks(5, hk, dim)
    xd = x.to(DEV)
    append(cache, table.to(DEV), None, i32([0] * 5), None, xd, xd, hk, outs=False)
    for b in range(5):
        model.append([b], 0, (x[b:b + 1, None].numpy(), x[b:b + 1, None].numpy()))
    ints = cache_ints(cache)
    assert np.array_equal(ints[0], model.q[0]) and np.array_equal(ints[1], model.q[1])
    assert np.array_equal(cache.amax.cpu().numpy(), model.amax)
    assert ints[0][0, 0, 0, :6].tolist() == [64, -127, 0, 127, -127, 0] and (ints[0][3, 0, 0] == -127).all()


def test_append_leaves_out_what_has_no_block():
    g = gen(6)
    hk, dim, blocks = 2, 32, 4
    # past the table, entries that are no block, positions below zero (whose last tokens arrive at 0)
    table = torch.tensor([[0, -1], [4, 1], [2, 1 << 30], [3, -(1 << 31)]], dtype=torch.int32)
    new, held = [70, 60, 40, 10], [60, 10, 120, -4]
    first = np.cumsum([0] + new)
    k, v = normal(g, 180, hk * dim), normal(g, 180, hk * dim)
    cache, model = make_cache(blocks, hk, dim), Blocks(blocks, hk, dim)
    for w, fill in enumerate((77, -78)):
        model.q[w][:] = fill
    model.amax[:] = 123.0
    k_out, _ = append(cache, table.to(DEV), i32(first), i32(held), None, k.to(DEV), v.to(DEV), hk)
    for b in range(4):
        model.append(table[b].tolist(), held[b],
                     tuple(x[first[b]:first[b + 1]].view(-1, hk, dim).numpy() for x in (k, v)))
    ints = cache_ints(cache)
    assert np.array_equal(ints[0], model.q[0]) and np.array_equal(ints[1], model.q[1])
    assert np.array_equal(cache.amax.cpu().numpy(), model.amax)
    assert torch.equal(k_out.cpu(), k)               # rotated (by nothing) all the same


def test_append_angles_of_far_positions():
    g = gen(7)
    dim, held = 128, [0, 1000, 100_003, 1_000_000, 16_000_001]
    B = len(held)
    freq = torch.tensor(np.exp(np.linspace(0, -12, dim // 2)), dtype=F32)
    k = normal(g, B, dim)
    cache = mq.kv_cache(1, 1, dim, DEV)
    table = torch.full((B, 1), -1, dtype=torch.int32)
    k_out, q_out = append(cache, table.to(DEV), None, i32(held), k.to(DEV), k.to(DEV), k.to(DEV), 1, freq.to(DEV), dim, False)
    want = rotated(k.view(B, 1, dim), torch.tensor(held), freq, dim, False).view(B, dim)
    # one rounding to binary32 of a sum of two products that 64 bits give to 1e-9 at these angles (2^24 2^-53)
    for got in (k_out, q_out):
        assert ((got.cpu().double() - want).abs() <= EPS32 / 2 * want.abs() + 1e-8).all()
    assert torch.equal(k_out, q_out)


# ---- attention over the cache -------------------------------------------------------------------------------------------

def filled_cache(g, blocks, hk, dim):
    c = mq.kv_cache(blocks, hk, dim, DEV)
    c.keys[..., :dim] = torch.randint(-127, 128, (blocks, hk, BLOCK, dim), generator=g).to(torch.int8)
    c.values[:, :, :dim] = torch.randint(-127, 128, (blocks, hk, dim, BLOCK), generator=g).to(torch.int8)
    c.amax.copy_(torch.exp(normal(g, blocks, hk, 2)))
    return c


def cache_rows(c, table_row, n):
    """Keys and values [hk, n, dim] in 64 bits of the first n tokens, and which of them lie in a block."""
    d = c.head_dim
    k, v, there = [], [], []
    for i in range(-(-n // BLOCK)):
        block = int(table_row[i])
        ok = 0 <= block < c.blocks
        b = block if ok else 0
        k.append(c.keys[b, :, :, :d].cpu().double() * (c.amax[b, :, 0].cpu().double() / 127)[:, None, None])
        v.append(c.values[b, :, :d][..., PLACES].cpu().double().transpose(1, 2) * (c.amax[b, :, 1].cpu().double() / 127)[:, None, None])
        there += [ok] * BLOCK
    if not k:
        return torch.zeros(c.kv_heads, 0, d).double(), torch.zeros(c.kv_heads, 0, d).double(), torch.zeros(0, dtype=torch.bool)
    return torch.cat(k, 1)[:, :n], torch.cat(v, 1)[:, :n], torch.tensor(there[:n])


def cached_reference(c, table, lens, max_len, q, heads, scale):
    """Output and tolerance."""
    dtype, per, d = q.dtype, heads // c.kv_heads, c.head_dim
    digits = 127 * 65536 if dtype == F32 else 127 * 256
    out, tol = torch.zeros(len(lens), heads, d).double(), torch.zeros(len(lens), heads, d).double()
    for b, n_any in enumerate(lens):
        n = max(0, min(n_any, max_len))
        k, v, there = cache_rows(c, table[b], n)
        if not there.any():
            continue
        k, v = k[:, there], v[:, there]
        x = q[b].double().view(c.kv_heads, per, d)
        s = x @ k.transpose(1, 2) * scale
        out[b] = (torch.softmax(s, -1) @ v).view(heads, d)
        # query digits: half a step of the row's largest; about a dozen binary32 roundings on the way to the exponent
        ds = abs(scale) * x.abs().amax(-1) / (2 * digits) * k.abs().sum(-1).amax(-1, keepdim=True) + 16 * EPS32 * s.abs().amax(-1)
        # probabilities: half a step of a block's largest each, 64 to a block; binary32 sums over the blocks
        dp = BLOCK / (2 * digits) + (n / BLOCK + 32) * EPS32
        vmax = v.abs().amax((1, 2))[:, None]
        t = vmax * (torch.expm1(2 * ds) + dp)
        tol[b] = t.reshape(heads, 1) + torch.finfo(dtype).eps / 2 * out[b].abs() + torch.finfo(dtype).tiny
    return out.view(len(lens), -1), tol.view(len(lens), -1)


def cached(c, table, lens, max_len, q, heads, scale, ldo=None, stream=None, ws=None):
    B, d = q.shape[0], c.head_dim
    ldo = ldo or heads * d
    out = torch.full((B, ldo), 7.0, dtype=q.dtype, device=DEV)
    n = mq.mq_cached_attention_ws_bytes(B, max_len, heads, c.kv_heads, d)
    ws = torch.full((n,), 255, dtype=torch.uint8, device=DEV) if ws is None else ws
    mq.mq_cached_attention(c, table, table.shape[1], lens, B, max_len, q, q.stride(0), heads, mq.dtype_code(q.dtype), scale,
                           out, ldo, ws, n, stream)
    return out


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("heads,hk,dim", [(8, 8, 64), (8, 2, 128), (16, 1, 80), (40, 2, 33), (4, 4, 256), (3, 1, 192), (5, 5, 1), (64, 1, 16)])
@pytest.mark.parametrize("lens", [[0, 1, 2, 63, 64, 65, 129, 700], [1500], [33] * 40, [9000, 0, 64, 4097]])
def test_cached_attention(heads, hk, dim, dtype, lens):
    g = gen(heads * dim + len(lens))
    B = len(lens)
    need = [-(-n // BLOCK) for n in lens]
    c = filled_cache(g, sum(need) + 1, hk, dim)
    order = torch.randperm(sum(need) + 1, generator=g).tolist()
    table = torch.full((B, max(need)), -1, dtype=torch.int32)
    for b in range(B):
        for i in range(need[b]):
            table[b, i] = order.pop()
    q = normal(g, B, heads * dim + 3).to(dtype)[:, :heads * dim]
    scale = dim ** -0.5
    want, tol = cached_reference(c, table, lens, max(lens), q, heads, scale)
    qd = torch.zeros(B, heads * dim + 3, dtype=dtype, device=DEV)[:, :heads * dim]
    qd.copy_(q)
    for max_len in sorted({max(lens), table.shape[1] * BLOCK}):
        got = cached(c, table.to(DEV), i32(lens), max_len, qd, heads, scale, ldo=heads * dim + 7).cpu().double()
        assert (got[:, heads * dim:] == 7).all()
        assert ((got[:, :heads * dim] - want).abs() <= tol).all()


def test_cached_attention_bounds_of_lengths_and_blocks():
    g = gen(11)
    heads, hk, dim = 4, 2, 64
    c = filled_cache(g, 6, hk, dim)
    table = torch.tensor([[0, 1, 2], [3, -1, 4], [-5, 6, 1 << 30], [5, 0, 7], [2, 2, 2]], dtype=torch.int32)
    lens = [1000, 150, 190, -3, 130]
    q = normal(g, 5, heads * dim)
    for max_len in (192, 100):
        want, tol = cached_reference(c, table, lens, max_len, q, heads, 0.2)
        got = cached(c, table.to(DEV), i32(lens), max_len, q.to(DEV), heads, 0.2).cpu().double()
        assert ((got - want).abs() <= tol).all()
        assert (got[2] == 0).all() and (got[3] == 0).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_cached_attention_special_rows(dtype):
    g = gen(12)
    heads, hk, dim, B = 2, 1, 64, 7
    c = filled_cache(g, 8, hk, dim)
    c.amax[4] = 0                                    # a block of zeros
    c.amax[5, :, 0] = 1e30                           # scores of which one is all there is
    table = torch.tensor([[i % 8, (i + 1) % 8] for i in range(B)], dtype=torch.int32)
    q = normal(g, B, heads * dim).to(dtype)
    q[0] = 0
    q[1, 5] = math.nan
    q[2, dim + 9] = math.inf
    q[6] = 1e-30 if dtype != F16 else 6e-8
    lens = [100, 100, 100, 128, 128, 128, 70]
    got = cached(c, table.to(DEV), i32(lens), 128, q.to(DEV), heads, 0.125).cpu().double().view(B, heads, dim)
    assert torch.isnan(got[1, 0]).all() and torch.isnan(got[2, 1]).all()
    clean = torch.nan_to_num(q, nan=0.0, posinf=0.0)
    want, tol = cached_reference(c, table, lens, 128, clean, heads, 0.125)
    want, tol = want.view(B, heads, dim), tol.view(B, heads, dim)
    for b, h in [(0, 0), (0, 1), (1, 1), (2, 0), (3, 0), (3, 1), (6, 0), (6, 1)]:
        assert ((got[b, h] - want[b, h]).abs() <= tol[b, h]).all(), (b, h)
    assert torch.isfinite(got[4]).all() and torch.isfinite(got[5]).all()


def test_cached_attention_small_probabilities_of_a_long_run():
    # one token far above 20 000 others whose probabilities are 1e-6 of its: together they are 2 % of the sum
    hk, dim, n = 1, 64, 20_000
    blocks = -(-n // BLOCK)
    c = mq.kv_cache(blocks, hk, dim, DEV)
    c.amax.fill_(127.0)
    c.keys[0, 0, 0, 0] = 100
    c.values[:, :, 0] = 50
    c.values[0, 0, 0, 0] = 0
    table = torch.arange(blocks, dtype=torch.int32).view(1, -1)
    for dtype in TYPES:
        q = torch.zeros(1, dim, dtype=dtype)
        q[0, 0] = 0.14
        want, tol = cached_reference(c, table, [n], n, q, 1, 1.0)
        got = cached(c, table.to(DEV), i32([n]), n, q.to(DEV), 1, 1.0).cpu().double()
        # (values of a block are alike but in one: the digits' errors do not add up to the worst case)
        assert abs(got[0, 0] - want[0, 0]) <= min(tol[0, 0], 0.02 * want[0, 0])


def test_cache_past_4_gib():
    g = gen(13)
    hk, dim = 8, 128
    blocks = 70_000                                   # 4.6 GB of keys, as much of values
    c = mq.kv_cache(blocks, hk, dim, DEV)
    table = torch.tensor([[blocks - 1, 65_537, 3], [65_535, blocks - 2, 65_536]], dtype=torch.int32)
    x = normal(g, 300, 3 * hk * dim)
    k, v = x[:, :hk * dim], x[:, hk * dim:2 * hk * dim]
    xd = x.to(DEV)
    append(c, table.to(DEV), i32([0, 150, 300]), i32([0, 0]), None, xd[:, :hk * dim], xd[:, hk * dim:2 * hk * dim], hk)
    model = {}
    for b in range(2):
        m = Blocks(3, hk, dim)
        m.append([0, 1, 2], 0, tuple(y[150 * b:150 * b + 150].view(-1, hk, dim).numpy() for y in (k, v)))
        for i in range(3):
            block = int(table[b, i])
            assert np.array_equal(c.keys[block].cpu().numpy(), m.q[0][i])
            assert np.array_equal(c.values[block].transpose(1, 2)[:, PLACES].cpu().numpy(), m.q[1][i])
            model[block] = m.amax[i]
    for block, a in model.items():
        assert np.array_equal(c.amax[block].cpu().numpy(), a)
    q = normal(g, 2, hk * dim)
    want, tol = cached_reference(c, table, [150, 150], 192, q, hk, 0.1)
    got = cached(c, table.to(DEV), i32([150, 150]), 192, q.to(DEV), hk, 0.1).cpu().double()
    assert ((got - want).abs() <= tol).all()


# ---- attention of packed sequences ----------------------------------------------------------------------------------------

def prompt(q, k, v, qf, kf, heads, hk, dim, causal, scale, ldo=None, out=None, stream=None, ws=None):
    ldo = ldo or heads * dim
    out = torch.full((q.shape[0], ldo), 7.0, dtype=q.dtype, device=DEV) if out is None else out
    B, t = len(qf) - 1, mq.dtype_code(q.dtype)
    n = mq.mq_prompt_attention_ws_bytes(t, B, k.shape[0], hk, dim)
    ws = torch.full((n,), 255, dtype=torch.uint8, device=DEV) if ws is None else ws
    qf, kf = (x if isinstance(x, torch.Tensor) else i32(x) for x in (qf, kf))
    mq.mq_prompt_attention(q, q.stride(0), k, k.stride(0), v, v.stride(0), t, qf, kf, B, q.shape[0], k.shape[0], heads, hk, dim,
                           causal, scale, out, ldo, ws, n, stream)
    return out


def prompt_reference(q, k, v, qf, kf, heads, hk, dim, causal, scale):
    """Output and tolerance; rows of no sequence are 7."""
    dtype, per = q.dtype, heads // hk
    eps = torch.finfo(dtype).eps
    out, tol = torch.full((q.shape[0], heads, dim), 7.0).double(), torch.zeros(q.shape[0], heads, dim).double()
    for b in range(len(qf) - 1):
        n, m = qf[b + 1] - qf[b], kf[b + 1] - kf[b]
        if n <= 0:
            continue
        x = q[qf[b]:qf[b + 1]].double().view(n, hk, per, dim).permute(1, 2, 0, 3)
        ks, vs = (y[kf[b]:kf[b + 1]].double().view(max(m, 0), hk, dim).permute(1, 0, 2)[:, None] for y in (k, v))
        s = x @ ks.transpose(-1, -2) * scale
        seen = torch.ones(n, m, dtype=torch.bool)
        if causal:
            seen = torch.arange(m)[None, :] <= torch.arange(n)[:, None] + m - n
        w = torch.nan_to_num(torch.softmax(s.masked_fill(~seen, -math.inf), -1))
        o = w @ vs                                                # [hk, per, n, dim]
        # scores: dim products summed in binary32 (and, binary32, parts left out: 2^-24 a product)
        size = ((x.abs() @ ks.abs().transpose(-1, -2)) * seen).amax(-1) * abs(scale) if m else torch.zeros(hk, per, n).double()
        ds = (dim / 2 + 8) * EPS32 * size
        # probabilities rounded to a 16-bit type, sums in binary32
        dp = (eps / 2 if dtype != F32 else 4 * EPS32) + (m / 2 + 16) * EPS32
        vmax = vs.abs().amax((-1, -2))[..., None] if m else torch.zeros(hk, 1, 1).double()
        t = (vmax * (torch.expm1(2 * ds) + dp))[..., None] + eps / 2 * o.abs() + torch.finfo(dtype).tiny
        out[qf[b]:qf[b + 1]] = o.permute(2, 0, 1, 3).reshape(n, heads, dim)
        tol[qf[b]:qf[b + 1]] = t.permute(2, 0, 1, 3).reshape(n, heads, dim)
    return out.view(len(out), -1), tol.view(len(out), -1)


SEQUENCES = [  # queries, keys
    ([1, 31, 32, 33, 0, 64, 65, 127, 128, 129, 5], None),
    ([200, 300], None),
    ([1, 40, 1, 130], [70, 200, 1, 131]),
    ([50, 33, 3], [20, 0, 1]),                       # more queries than keys: with a causal mask the first see nothing
    ([1, 31, 32, 33, 0, 64, 65, 7], [3, 31, 40, 33, 0, 64, 65, 100]),       # few of each: the one-launch form
    ([700, 257], [700, 300]),
    ([600, 450, 33, 1], [2500, 1, 0, 40]),
    ([1, 31, 32, 33, 0, 64, 65, 127, 128, 129, 5, 1501, 700], None),       # short ones beside long ones
    ([1700, 1500], [1700, 1601]),                    # many of each: two tiles a wave (16-bit types)
    ([1601, 1473], [33, 2000]),
]


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("heads,hk,dim", [(4, 4, 64), (4, 1, 128), (6, 3, 80), (2, 1, 33), (2, 2, 256), (1, 1, 1), (3, 3, 160), (2, 1, 224), (2, 2, 192), (8, 8, 16)])
@pytest.mark.parametrize("which", range(len(SEQUENCES)))
def test_prompt_attention(which, heads, hk, dim, dtype, causal):
    n, m = SEQUENCES[which]
    m = m or n
    g = gen(which * 1000 + heads * dim)
    front, back = 3, 2
    qf, kf = np.cumsum([front] + n).tolist(), np.cumsum([front] + m).tolist()
    q = normal(g, qf[-1] + back, heads * dim).to(dtype)
    kv = normal(g, kf[-1] + back, 2 * hk * dim + 1).to(dtype)
    k, v = kv[:, :hk * dim], kv[:, hk * dim + 1:]
    q[:front] = math.nan                             # rows of no sequence may hold anything
    kv[:front] = math.nan
    kv[kf[-1]:] = math.inf
    kvd = kv.to(DEV)
    want, tol = prompt_reference(q, k, v, qf, kf, heads, hk, dim, causal, dim ** -0.5)
    got = prompt(q.to(DEV), kvd[:, :hk * dim], kvd[:, hk * dim + 1:], qf, kf, heads, hk, dim, causal, dim ** -0.5,
                 ldo=heads * dim + 5).cpu().double()
    assert (got[:, heads * dim:] == 7).all()
    got = got[:, :heads * dim]
    assert (got[:front] == 7).all() and (got[qf[-1]:] == 7).all()
    assert ((got - want).abs() <= tol).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,others,dim", [(150, 0, 64), (150, 7, 64), (300, 0, 64), (1600, 0, 64), (150, 7, 256), (150, 0, 192)])      # (empty sequences: the one-launch form takes the call)
def test_prompt_attention_masked_places_never_count(dtype, n, others, dim):
    g = gen(21)
    heads, hk = 2, 1
    ends = [0] + [n] * (1 + others)
    q, k, v = (normal(g, n, h * dim).to(dtype) for h in (heads, hk, hk))
    want, tol = prompt_reference(q, k, v, ends, ends, heads, hk, dim, True, 0.125)
    clean = prompt(q.to(DEV), k.to(DEV), v.to(DEV), ends, ends, heads, hk, dim, True, 0.125).cpu()
    for at, kind in ((100, "k"), (70, "v"), (149, "kv"), (96, "v")):
        for bad in (math.nan, math.inf, -math.inf, torch.finfo(dtype).max, torch.finfo(dtype).min):
            kb, vb = k.clone(), v.clone()
            if "k" in kind:
                kb[at, 3] = bad
            if "v" in kind:
                vb[at, 5] = bad
            got = prompt(q.to(DEV), kb.to(DEV), vb.to(DEV), ends, ends, heads, hk, dim, True, 0.125).cpu()
            assert torch.equal(got[:at], clean[:at]), (at, kind, bad)
            if not math.isfinite(bad):
                assert torch.isnan(got[at:]).all(), (at, kind, bad)
    assert ((clean.double() - want).abs() <= tol).all()
    qb = q.clone()
    qb[7, dim + 2] = math.nan                        # a query's own NaN stays with its head
    got = prompt(qb.to(DEV), k.to(DEV), v.to(DEV), ends, ends, heads, hk, dim, True, 0.125).cpu()
    assert torch.isnan(got[7, dim:]).all() and torch.equal(got[7, :dim], clean[7, :dim])
    assert torch.equal(got[:7], clean[:7]) and torch.equal(got[8:], clean[8:])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("scale", [-0.125, 0.0])
@pytest.mark.parametrize("n", [70, 300, 1600])
def test_prompt_attention_scales_that_are_not_positive(n, scale, dtype):
    g = gen(25)
    heads, hk, dim = 2, 1, 64
    q, k, v = (normal(g, n, h * dim).to(dtype) for h in (heads, hk, hk))
    want, tol = prompt_reference(q, k, v, [0, n], [0, n], heads, hk, dim, True, scale)
    got = prompt(q.to(DEV), k.to(DEV), v.to(DEV), [0, n], [0, n], heads, hk, dim, True, scale).cpu().double()
    assert ((got - want).abs() <= tol).all()


@pytest.mark.parametrize("others", [0, 3])
def test_prompt_attention_values_of_any_magnitude(others):
    g = gen(22)
    heads, hk, dim, n = 1, 1, 32, 90
    q, k, v = (normal(g, n, dim) for _ in range(3))
    for row, size in ((3, 1e30), (40, 1e-30), (80, 1e15)):
        v[row] *= size
    q *= 1e-12
    k *= 1e12
    want, tol = prompt_reference(q, k, v, [0, n], [0, n], heads, hk, dim, True, 0.125)
    ends = [0] + [n] * (1 + others)
    got = prompt(q.to(DEV), k.to(DEV), v.to(DEV), ends, ends, heads, hk, dim, True, 0.125).cpu().double()
    assert ((got - want).abs() <= tol).all()
    # rows in front of the large ones are as exact as without them
    w2, t2 = prompt_reference(q[:3], k[:3], v[:3], [0, 3], [0, 3], heads, hk, dim, True, 0.125)
    assert ((got[:3] - w2).abs() <= t2).all()


@pytest.mark.parametrize("qf,kf", [([0, 5, 1000], [0, 9, 1 << 30]), ([-7, 20, 40], [-1, 3, 40]), ([0, 30, 10], [0, 35, 20]),
                                   ([50, 60, 70], [0, 1, 2]), ([40, 40, 40], [40, 40, 40])])
def test_prompt_attention_lists_that_do_not_fit(qf, kf):
    # bounds are taken as the nearest of [0, rows], a sequence that ends before it starts is empty; no row outside is written
    g = gen(23)
    heads, hk, dim, n = 2, 2, 48, 40
    x = normal(g, n, 3 * heads * dim)
    q, k, v = (x[:, i * heads * dim:(i + 1) * heads * dim] for i in range(3))
    room = torch.full((n + 20, heads * dim), 7.0, device=DEV)
    xd = x.to(DEV)
    dq, dk, dv = (xd[:, i * heads * dim:(i + 1) * heads * dim] for i in range(3))
    prompt(dq, dk, dv, qf, kf, heads, hk, dim, False, 0.2, out=room[10:10 + n])
    torch.cuda.synchronize()
    got = room.cpu().double()
    assert (got[:10] == 7).all() and (got[10 + n:] == 7).all()
    cq, ck = ([min(max(f, 0), n) for f in x] for x in (qf, kf))
    if cq == sorted(cq) and ck == sorted(ck):
        want, tol = prompt_reference(q, k, v, cq, ck, heads, hk, dim, False, 0.2)
        assert ((got[10:10 + n] - want).abs() <= tol).all()


def test_prompt_attention_in_place_and_many_sequences():
    g = gen(24)
    heads, hk, dim = 2, 1, 64
    n = torch.randint(0, 60, (700,), generator=g).tolist()
    f = np.cumsum([0] + n).tolist()
    q, k, v = (normal(g, f[-1], h * dim) for h in (heads, hk, hk))
    want, tol = prompt_reference(q, k, v, f, f, heads, hk, dim, True, 0.125)
    qd = q.to(DEV)
    prompt(qd, k.to(DEV), v.to(DEV), f, f, heads, hk, dim, True, 0.125, out=qd)
    assert ((qd.cpu().double() - want).abs() <= tol).all()


# ---- log probabilities ----------------------------------------------------------------------------------------------------

def packed(q):
    rows, cols = q.shape
    one = torch.ones(1, device=DEV)
    out = torch.empty(mq.mq_packed_bytes(8, rows, cols), dtype=torch.uint8, device=DEV)
    mq.mq_quantize_pack_f32(q.float().to(DEV).contiguous(), rows, cols, 8, one, out)
    return out


def score(pA, pW, M, N, K, sA, sW, target, k, entropy=True, stream=None, ws=None):
    logprob, ent = torch.full((M,), 7.0, device=DEV), torch.full((M,), 7.0, device=DEV) if entropy else None
    tok = torch.full((M, k), -7, dtype=torch.int32, device=DEV) if k else None
    alt = torch.full((M, k), 7.0, device=DEV) if k else None
    n = mq.mq_token_logprob_ws_bytes(M, N, k)
    ws = torch.full((n,), 255, dtype=torch.uint8, device=DEV) if ws is None else ws
    mq.mq_gemm_token_logprob_packed(pA, pW, M, N, K, sA, sW, target, k, logprob, ent, tok, alt, ws, n, stream)
    return logprob, ent, tok, alt


def check_score(qA, qW, sA, sW, target, k):
    (M, K), N = qA.shape, qW.shape[0]
    a, w = torch.tensor([sA], device=DEV), torch.tensor([sW], device=DEV)
    logprob, ent, tok, alt = score(packed(qA), packed(qW), M, N, K, a, w, target.to(DEV), k)
    acc = (qA.double().to(DEV) @ qW.double().to(DEV).T)           # exact
    y = acc / (float(a) * float(w))
    p = torch.log_softmax(y, -1)
    # u: three roundings; a word's exponent: that of its logit, of the reference and of the sum; binary32 sums over at most
    # 16 words of each 32, one lane after another; log2 and the last products
    tol = (4 * EPS32 * y.abs().amax(-1) + (N / 4 + 64) * EPS32 / 2 + 4 * EPS32 * p.abs().amax(-1))
    t = target.long().to(DEV)
    there = (t >= 0) & (t < N)
    want = torch.where(there, p.gather(1, t.clamp(0, N - 1)[:, None])[:, 0], torch.zeros_like(tol))
    assert ((logprob.double() - want).abs() <= tol).all()
    # the sum of p log p: each log p off by tol at most, and p by tol in proportion
    h = -(p.exp() * torch.where(p.exp() > 0, p, torch.zeros_like(p))).sum(-1)
    assert ((ent.double() - h).abs() <= tol * (2 + h)).all()
    if k:
        key = acc.to(torch.int64) * N + (N - 1 - torch.arange(N, device=DEV))
        best = N - 1 - torch.topk(key, k, -1).values % N
        assert torch.equal(tok.long(), best)
        assert ((alt.double() - p.gather(1, best)).abs() <= tol[:, None]).all()


def ints(g, rows, cols, most=127):
    return torch.randint(-most, most + 1, (rows, cols), generator=g)


@pytest.mark.parametrize("M,N,K,k", [
    (1, 1, 1, 1), (1, 36000, 512, 4), (7, 36000, 512, 4), (7, 1000, 1024, 8), (32, 33, 64, 8), (33, 31, 100, 5), (65, 5000, 512, 0),
    (100, 2049, 777, 3), (300, 4000, 512, 4), (384, 4000, 513, 4), (600, 3001, 512, 8), (600, 3001, 1000, 1), (2100, 1500, 512, 4),
    (2100, 1500, 1024, 0), (31, 255, 32, 2), (129, 8, 48, 8), (520, 36000, 960, 4), (2100, 1500, 512, 0), (900, 33000, 300, 0),
    (897, 31, 40, 0), (2500, 4000, 512, 8)])
def test_token_logprob(M, N, K, k):
    g = gen(M + N + K)
    target = torch.randint(-2, N + 2, (M,), generator=g, dtype=torch.int32)
    qA, qW = ints(g, M, K, 60), ints(g, N, K, 60)
    check_score(qA, qW, 30.0, 30.0 * math.sqrt(K) / 3, target, k)


@pytest.mark.parametrize("M", [5, 300])
@pytest.mark.parametrize("K", [512, 1024])
def test_token_logprob_extreme_sums(M, K):
    g = gen(K)
    N = 700
    qA = torch.full((M, K), 127)
    qA[1::2] = -127
    qW = torch.where(torch.rand(N, 1, generator=g) < 0.5, 127, -127).expand(N, K).clone()
    qW[5] = 0
    target = torch.arange(M, dtype=torch.int32) % N
    check_score(qA, qW, 127.0, 127.0, target, 8)           # logits of +-K: one side of the words is all there is
    check_score(qA, qW, 4000.0, 4000.0, target, 8)         # within a unit of each other
    check_score(qA, torch.full((N, K), 3), 10.0, 10.0, target, 8)      # all equal: the lowest words
    check_score(torch.zeros(M, K, dtype=torch.long), qW, 1.0, 1.0, target, 4)


@pytest.mark.parametrize("M", [3, 70, 520])
def test_token_logprob_ties_go_to_the_lowest_word(M):
    g = gen(31)
    N, K = 3100, 64
    qA, qW = ints(g, M, K, 1), ints(g, N, K, 1)            # few different sums, hundreds of words with each
    check_score(qA, qW, 1.0, 2.0, torch.zeros(M, dtype=torch.int32), 8)


def test_token_logprob_agrees_with_the_beam_output_layer():
    g = gen(32)
    M, N, K, k = 90, 7000, 512, 4
    qA, qW = ints(g, M, K), ints(g, N, K)
    pA, pW = packed(qA), packed(qW)
    a, w = torch.tensor([300.0], device=DEV), torch.tensor([200.0], device=DEV)
    tok, lp = torch.empty((M, k), dtype=torch.int32, device=DEV), torch.empty((M, k), device=DEV)
    n = mq.mq_topk_ws_bytes(M, N, k)
    mq.mq_gemm_topk_packed(pA, pW, None, 0, M, N, K, a, w, k, tok, lp, torch.empty(n, dtype=torch.uint8, device=DEV), n)
    logprob, ent, tok2, alt = score(pA, pW, M, N, K, a, w, tok[:, 1].contiguous(), k)
    assert torch.equal(tok, tok2)
    assert (logprob - lp[:, 1]).abs().max() <= 2e-4 and (alt - lp).abs().max() <= 2e-4     # the beam layer's own 1e-4, twice
    none, ent2, _, _ = score(pA, pW, M, N, K, a, w, tok[:, 1].contiguous(), 0, entropy=False)
    assert ent2 is None and (none - logprob).abs().max() <= 1e-5


# ---- together -----------------------------------------------------------------------------------------------------------

class Step:
    """A prompt taken in, scored, and continued by one token: every operator on what the one before it gave."""

    def __init__(self, dtype=F32):
        g = gen(41)
        self.heads, self.hk, self.dim, self.N, self.K = 4, 2, 64, 1000, 256
        self.n = [70, 1, 128, 33]
        self.f = np.cumsum([0] + self.n).tolist()
        B, T, width = 4, self.f[-1], (self.heads + 2 * self.hk) * self.dim
        self.x = normal(g, T, self.K).to(DEV)
        self.y = normal(g, B, self.K).to(DEV)
        self.pw = mq.prepare_weight((normal(g, width, self.K) * 0.06).to(DEV), 8)
        self.pe = mq.prepare_weight((normal(g, self.N, self.K) * 0.2).to(DEV), 8)
        self.target = torch.randint(0, self.N, (T,), generator=g, dtype=torch.int32).to(DEV)
        self.freq = torch.tensor(10000.0 ** (-np.arange(0, 64, 2) / 64), dtype=F32, device=DEV)
        self.table = torch.tensor([[3, 7, 0], [5, 2, 1], [6, 4, 8], [9, 11, 10]], dtype=torch.int32, device=DEV)
        self.first, self.zero, self.held = i32(self.f), i32([0] * B), i32(self.n)
        self.after = i32([n + 1 for n in self.n])
        self.cache = mq.kv_cache(12, self.hk, self.dim, DEV)
        D = self.heads * self.dim
        assert D == self.K
        e = lambda *s, **kw: torch.empty(s, device=DEV, **kw)  # noqa: E731
        self.qkv, self.qkv1 = e(T, width), e(B, width)
        self.kr, self.qr, self.kr1, self.qr1 = e(T, self.hk * self.dim), e(T, D), e(B, self.hk * self.dim), e(B, D)
        self.o, self.o1 = e(T, D), e(B, D)
        self.lp, self.ent, self.tok, self.alt = e(T), e(T), e(T, 3, dtype=torch.int32), e(T, 3)
        self.pa, self.sa = e(mq.mq_packed_bytes(8, T, D), dtype=torch.uint8), e(1)
        u8 = lambda n: e(n, dtype=torch.uint8)  # noqa: E731
        self.wl = u8(mq.mq_linear_ws_bytes(8, T, self.K))
        self.wp = u8(mq.mq_prompt_attention_ws_bytes(0, B, T, self.hk, self.dim))
        self.wc = u8(mq.mq_cached_attention_ws_bytes(B, 192, self.heads, self.hk, self.dim))
        self.ws = u8(mq.mq_token_logprob_ws_bytes(T, self.N, 3))
        self.wq = u8(mq.mq_quantize_absmax_ws_bytes())

    def run(self):
        h, hk, d, K, D = self.heads, self.hk, self.dim, self.K, self.heads * self.dim
        T, B, width = self.x.shape[0], 4, self.qkv.shape[1]

        def take(x, rows, qkv, first, held, kr, qr):
            mq.mq_linear_f32(x, rows, K, None, self.pw.packed, self.pw.scale, 8, width, None, False, qkv, None, self.wl,
                             self.wl.numel())
            q, k, v = qkv[:, :D], qkv[:, D:D + hk * d], qkv[:, D + hk * d:]
            mq.mq_kv_append(self.cache, self.table, 3, first, held, B, rows, k, width, v, width, q, width, h, 0, self.freq, d, False, kr, qr)
            return v

        v = take(self.x, T, self.qkv, self.first, self.zero, self.kr, self.qr)
        mq.mq_prompt_attention(self.qr, D, self.kr, hk * d, v, width, 0, self.first, self.first, B, T, T, h, hk, d, True, d ** -0.5,
                               self.o, D, self.wp, self.wp.numel())
        mq.mq_quantize_absmax_pack_f32(self.o, T, D, 8, self.pa, self.sa, self.wq, self.wq.numel())
        mq.mq_gemm_token_logprob_packed(self.pa, self.pe.packed, T, self.N, D, self.sa, self.pe.scale, self.target, 3, self.lp,
                                        self.ent, self.tok, self.alt, self.ws, self.ws.numel())
        take(self.y, B, self.qkv1, None, self.held, self.kr1, self.qr1)
        mq.mq_cached_attention(self.cache, self.table, 3, self.after, B, 192, self.qr1, D, h, 0, d ** -0.5, self.o1, D, self.wc,
                               self.wc.numel())

    def results(self):
        return [x.clone() for x in (self.o, self.lp, self.ent, self.tok, self.alt, self.o1, self.cache.keys, self.cache.values,
                                    self.cache.amax)]


def test_a_prompt_its_scores_and_the_next_token():
    s = Step()
    s.run()
    torch.cuda.synchronize()
    D, hk, d, h = 256, 2, 64, 4
    # rotation and cache
    model = Blocks(12, hk, d)
    for b in range(4):
        rows = slice(s.f[b], s.f[b + 1])
        qkv = s.qkv[rows].cpu()
        pos = torch.arange(s.n[b])
        k = rotated(qkv[:, D:D + hk * d].reshape(-1, hk, d), pos, s.freq.cpu(), d, False).float()
        q = rotated(qkv[:, :D].reshape(-1, h, d), pos, s.freq.cpu(), d, False).float()
        assert torch.equal(s.kr[rows].cpu().view(-1, hk, d), k) and torch.equal(s.qr[rows].cpu().view(-1, h, d), q)
        model.append(s.table[b].tolist(), 0, (k.numpy(), qkv[:, D + hk * d:].reshape(-1, hk, d).numpy()))
        one = s.qkv1[b:b + 1].cpu()
        k1 = rotated(one[:, D:D + hk * d].reshape(-1, hk, d), torch.tensor([s.n[b]]), s.freq.cpu(), d, False).float()
        model.append(s.table[b].tolist(), s.n[b], (k1.numpy(), one[:, D + hk * d:].reshape(-1, hk, d).numpy()))
    used = [int(s.table[b, i]) for b in range(4) for i in range(-(-(s.n[b] + 1) // BLOCK))]
    got = cache_ints(s.cache)
    assert np.array_equal(got[0][used], model.q[0][used]) and np.array_equal(got[1][used], model.q[1][used])
    # attention over the prompt, over the cache
    want, tol = prompt_reference(s.qr.cpu(), s.kr.cpu(), s.qkv[:, D + hk * d:].cpu(), s.f, s.f, h, hk, d, True, d ** -0.5)
    assert ((s.o.cpu().double() - want).abs() <= tol).all()
    want, tol = cached_reference(s.cache, s.table.cpu(), [n + 1 for n in s.n], 192, s.qr1.cpu(), h, d ** -0.5)
    assert ((s.o1.cpu().double() - want).abs() <= tol).all()
    # scores of what the quantizer made of the attention's output
    q = torch.empty((s.f[-1], D), dtype=torch.int8, device=DEV)
    mq.mq_unpack_weight(s.pa, 8, s.f[-1], D, q)
    e = torch.empty((s.N, D), dtype=torch.int8, device=DEV)
    mq.mq_unpack_weight(s.pe.packed, 8, s.N, D, e)
    y = q.double() @ e.double().T / (float(s.sa) * float(s.pe.scale))
    p = torch.log_softmax(y, -1)
    assert (s.lp.double() - p.gather(1, s.target.long()[:, None])[:, 0]).abs().max() <= 1e-4
    assert torch.equal(s.tok[:, 0].long(), p.argmax(-1))


def test_captured_steps_replay_beside_eager_ones():
    one, two, eager = Step(), Step(), Step()
    eager.run()
    torch.cuda.synchronize()
    want = eager.results()
    graphs = []
    for s in (one, two):
        s.run()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            s.run()
        graphs.append(g)
    for turn in range(4):
        for s, g in zip((one, two), graphs):
            for x in (s.wl, s.wp, s.wc, s.ws, s.wq):
                x.fill_(255 if turn % 2 else 0)
            for x in (s.o, s.lp, s.ent, s.alt, s.o1):
                x.fill_(math.nan)
            g.replay()
        eager.run()
        torch.cuda.synchronize()
        for s in (one, two, eager):
            for x, y in zip(s.results(), want):
                assert torch.equal(x, y)


def test_two_streams_at_once():
    # buffers and workspaces of their own: neither call sees the other
    steps = [Step(), Step()]
    for s in steps:
        s.run()
    torch.cuda.synchronize()
    want = steps[0].results()
    for s in steps:
        for x in (s.o, s.lp, s.ent, s.alt, s.o1, s.kr, s.qr, s.kr1, s.qr1):
            x.fill_(math.nan)
        for x in (s.wp, s.wc, s.ws):
            x.fill_(255)
        s.cache.keys.zero_(), s.cache.values.zero_(), s.cache.amax.zero_()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(4):
        for s, at in zip(steps, streams):
            D, hk, d, h, T, B, width = 256, s.hk, s.dim, s.heads, s.x.shape[0], 4, s.qkv.shape[1]
            for x, first, held, kr, qr in ((s.qkv, s.first, s.zero, s.kr, s.qr), (s.qkv1, None, s.held, s.kr1, s.qr1)):
                q, k, v = x[:, :D], x[:, D:D + hk * d], x[:, D + hk * d:]
                mq.mq_kv_append(s.cache, s.table, 3, first, held, B, len(x), k, width, v, width, q, width, h, 0, s.freq, d, False,
                                kr, qr, stream=at)
                if first is None:
                    mq.mq_cached_attention(s.cache, s.table, 3, s.after, B, 192, qr, D, h, 0, d ** -0.5, s.o1, D, s.wc, s.wc.numel(),
                                           stream=at)
                else:
                    mq.mq_prompt_attention(qr, D, kr, hk * d, v, width, 0, first, first, B, T, T, h, hk, d, True, d ** -0.5, s.o, D,
                                           s.wp, s.wp.numel(), stream=at)
                    mq.mq_gemm_token_logprob_packed(s.pa, s.pe.packed, T, s.N, D, s.sa, s.pe.scale, s.target, 3, s.lp, s.ent, s.tok,
                                                    s.alt, s.ws, s.ws.numel(), stream=at)
    torch.cuda.synchronize()
    for s in steps:
        for x, y in zip(s.results(), want):
            assert torch.equal(x, y)


def test_another_stream():
    s, want = Step(), Step()
    want.run()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        s.run()
    side.synchronize()
    for x, y in zip(s.results(), want.results()):
        assert torch.equal(x, y)
