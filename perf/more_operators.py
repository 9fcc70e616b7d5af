"""What is measured of the serving operators (include/mq_serve.h): cases over their range, their inputs and their plain forms.

The operators: attention of several new tokens per sequence over the paged 8-bit cache (chunk), tables of continued sequences
with shared blocks, copies on write and new blocks (fork), a cache's used blocks moved to its front (compact), residual addition
with root-mean-square norm, its result in the type or as 8-bit rows with a multiplier each (norm), and products with 4-bit weights in
groups with scale and zero (product4).  Where `own` is false `run` computes them with elementary torch operations, where it is
true with the library's calls.

Layout of the cache: blocks of 64 tokens; keys int8 [blocks][kv heads][64][dk], dk = head width up to a multiple of 64;
values int8 [blocks][kv heads][dv][64], dv = head width up to a multiple of 16, token t of the block at place
16 ((t / 4) % 4) + 4 (t / 16) + t % 4; amax float [blocks][kv heads][2].  A value is q * amax / 127.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
BLOCK = 64
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
UNUSED = 1 << 30                                   # state of a block that nobody uses


# ---- cases ------------------------------------------------------------------------------------------------------------

def listed():
    return [
        # ends of 64 translations tried on what the decoder holds already, width 512 in 8 heads: latency
        dict(name="chunk_sentences", op="chunk", dtype="f32", batch=64, new_lo=1, new_hi=12, held_lo=1, held_hi=90, heads=8,
             kv_heads=8, dim=64, causal=True, twist=0.2),
        # serving: a few proposed tokens of every sequence checked in one step
        dict(name="chunk_verify", op="chunk", dtype="bf16", batch=32, new_lo=3, new_hi=6, held_lo=1000, held_hi=9000, heads=32,
             kv_heads=8, dim=128, causal=True, twist=0.5),
        # long prompts taken in by pieces, each piece behind what came before
        dict(name="chunk_pieces", op="chunk", dtype="bf16", batch=4, new_lo=300, new_hi=1100, held_lo=2000, held_hi=16000, heads=32,
             kv_heads=8, dim=128, causal=True, twist=0.1),
        # a step of beam search: 75 sentences, 4 hypotheses each, one more token
        dict(name="fork_beams", op="fork", groups=75, rows=4, ways=4, len_lo=1, len_hi=90, grow=1, kept=0.0, spare=400, heads=8, dim=64,
             twist=0.3),
        # 32 answers begun to each of 8 long prompts, room for 20 tokens of each
        dict(name="fork_answers", op="fork", groups=8, rows=1, ways=32, len_lo=2000, len_hi=16000, grow=20, kept=0.1, spare=700,
             heads=8, dim=128, twist=0.6),
        # what is left of a batch of sentences
        dict(name="compact_sentences", op="compact", batch=90, len_lo=1, len_hi=90, kept=0.0, blocks=300, heads=8, dim=64, twist=0.1),
        # long sequences in a cache of which half is free again
        dict(name="compact_long", op="compact", batch=24, len_lo=1000, len_hi=12000, kept=0.02, blocks=3500, heads=8, dim=128,
             twist=0.4),
        # in front of a product in a serving step of 64 sequences
        dict(name="norm_step", op="norm", form="rows8", dtype="bf16", rows=64, dim=4096, residual=True),
        # the same for prompts, result in the type
        dict(name="norm_prompt", op="norm", form="y", dtype="bf16", rows=8192, dim=4096, residual=True),
        # one token of one sequence
        dict(name="product4_one", op="product4", dtype="bf16", rows=1, words=4096, dim=4096, group=128, bias=False),
        # a step of a few sequences, 8-bit rows as the norm leaves them, odd width
        dict(name="product4_step", op="product4", dtype="rows8", rows=24, words=11000, dim=4096, group=64, bias=False),
        # many rows in binary32, fine groups
        dict(name="product4_batch", op="product4", dtype="f32", rows=150, words=2048, dim=8000, group=32, bias=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["chunk", "chunk", "fork", "compact", "norm", "product4", "product4"])
    twist = round(rng.random(), 3)
    if op == "norm":
        dim = rng.choice([64, 100, 512, 777, 1024, 2048, 4096, 5000, 8192])
        return dict(op=op, form=rng.choice(["rows8", "y"]), dtype=rng.choice(list(TYPES)), dim=dim,
                    rows=_log_int(rng, 1, max(1, 16000000 // dim)), residual=rng.random() < 0.7)
    if op == "product4":
        words, dim = _log_int(rng, 100, 12000), _log_int(rng, 64, 12000)
        return dict(op=op, dtype=rng.choice(["rows8", "f32", "f16", "bf16"]), words=words, dim=dim,
                    rows=_log_int(rng, 1, max(1, min(200, int(2e9 / (words * dim))))), group=rng.choice([32, 64, 128]),
                    bias=rng.random() < 0.5)
    dim = rng.choice([32, 64, 64, 80, 96, 128, 128, 256])
    kv = rng.choice([1, 2, 4, 5, 8, 16])
    if op == "chunk":
        heads = kv * rng.choice([1, 1, 2, 4, 8])
        new = _log_int(rng, 1, 1200)
        held = rng.choice([0, _log_int(rng, 1, 16000), _log_int(rng, 1, 16000)])
        room = min(int(1.2e8 / ((held + new) * kv * dim)), int(2e11 / (4 * dim * heads * new * (held + new))))
        return dict(op=op, dtype=rng.choice(list(TYPES)), batch=max(1, min(200, rng.randint(1, max(1, room)))),
                    new_lo=rng.choice([0, 1, max(1, new // 4), new]), new_hi=new, held_lo=held // rng.choice([1, 8]), held_hi=held,
                    heads=heads, kv_heads=kv, dim=dim, causal=rng.random() < 0.8, twist=twist)
    size = 2 * BLOCK * kv * dim                       # bytes of a block
    if op == "fork":
        hi = _log_int(rng, 1, 16000)
        per = -(-hi // BLOCK)
        groups = _log_int(rng, 1, max(1, min(80, int(3e8 / (size * per)))))
        ways = rng.randint(1, max(1, min(32, int(3e7 / (size * groups)))))
        return dict(op=op, groups=groups, rows=rng.choice([1, ways]), ways=ways, len_lo=rng.choice([0, hi // 8, hi]), len_hi=hi,
                    grow=rng.choice([0, 1, 1, 5, 100]), kept=rng.choice([0.0, 0.1]), spare=rng.choice([3 * groups * ways + 5, groups]),
                    heads=kv, dim=dim, twist=twist)
    hi = _log_int(rng, 1, 12000)
    blocks = _log_int(rng, 10, max(11, min(4000, int(4e8 / size))))
    return dict(op=op, batch=max(1, min(300, int(0.5 * blocks / -(-hi // BLOCK)))), len_lo=rng.choice([0, hi // 8, hi]), len_hi=hi,
                kept=rng.choice([0.0, 0.02, 0.2]), blocks=blocks, heads=kv, dim=dim, twist=twist)


# ---- inputs -----------------------------------------------------------------------------------------------------------

def _spread(lo, hi, n, twist):
    """n whole numbers from lo to hi, spread evenly over the logarithm."""
    u = (twist + 0.6180339887498949 * np.arange(1, n + 1)) % 1.0
    x = np.exp(np.log(lo + 1.0) + u * (np.log(hi + 1.0) - np.log(lo + 1.0))) - 1.0
    return np.clip(np.rint(x), lo, hi).astype(np.int64)


def _lengths(c):
    """New tokens of each sequence and all that the cache holds of it then."""
    new = _spread(c["new_lo"], c["new_hi"], c["batch"], c["twist"])
    new[0] = max(new[0], 1)
    return new, new + _spread(c["held_lo"], c["held_hi"], c["batch"], c["twist"] + 0.37)


def _i32(x):
    return torch.tensor(np.asarray(x).astype(np.int32), device=DEV)


def _cache(blocks, heads, dim, g):
    dk, dv = -(-dim // 64) * 64, -(-dim // 16) * 16

    def ints(shape):          # as unit normal values with their largest at 127 come out, about
        return torch.randint(-90, 91, shape, generator=g, device=DEV, dtype=torch.int8)

    keys, values = ints((blocks, heads, BLOCK, dk)), ints((blocks, heads, dv, BLOCK))
    keys[..., dim:] = 0
    values[:, :, dim:] = 0
    return dict(keys=keys, values=values, amax=2.5 + 2.0 * torch.rand((blocks, heads, 2), generator=g, device=DEV), blocks=blocks)


def _table(need, width, order):
    """Rows of that many blocks each, handed out of `order` one after the other."""
    table = torch.full((len(need), width), -1, dtype=torch.int32, device=DEV)
    at = torch.arange(width, device=DEV)[None, :] < torch.tensor(need, device=DEV)[:, None]
    table[at] = order[:int(need.sum())].to(torch.int32)
    return table


def _kept(c, blocks, g):
    return (torch.rand(blocks, generator=g, device=DEV) < c["kept"]).to(torch.int32)


def _fork_sizes(c):
    """Lengths by group, blocks of the cache, columns of the table."""
    n = _spread(c["len_lo"], c["len_hi"], c["groups"], c["twist"])
    full, open_ = n // BLOCK, (n % BLOCK > 0).astype(np.int64)
    used = int((full + open_ * c["rows"]).sum())
    return n, full, open_, used, used + c["spare"], max(1, int(-(-(n.max() + c["grow"]) // BLOCK)))


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=DEV)

    s = dict(case=c)
    if c["op"] == "norm":
        t = TYPES[c["dtype"]]
        s["x"] = normal(c["rows"], c["dim"]).to(t)
        s["r"] = (normal(c["rows"], c["dim"]) * 3).to(t) if c["residual"] else None
        s["gamma"] = 0.5 + torch.rand(c["dim"], generator=g, device=DEV)
        return s
    if c["op"] == "product4":
        M, N, K, G = c["rows"], c["words"], c["dim"], c["group"]
        groups = -(-K // G)
        s["codes"] = (8 + normal(N, K) * 2.7).round_().clamp_(0, 15).to(torch.uint8)
        s["zeros"] = (8 + normal(N, groups)).round_().clamp_(0, 15).to(torch.uint8)
        s["scales"] = ((0.5 + torch.rand((N, groups), generator=g, device=DEV)) * 0.4 / math.sqrt(K)).bfloat16().float()
        s["bias"] = normal(N) if c["bias"] else None
        if c["dtype"] == "rows8":
            s["x"] = (normal(M, K) * 30).round_().clamp_(-127, 127).to(torch.int8)
            s["rowscale"] = 25 + 10 * torch.rand(M, generator=g, device=DEV)
            s["out"] = torch.bfloat16
        else:
            s["out"] = TYPES[c["dtype"]]
            s["x"], s["rowscale"] = normal(M, K).to(s["out"]), None
        if own:
            import paper_1805_12096_amd as mq
            s["packed"] = mq.w4_pack(s["codes"], s["scales"], s["zeros"], G)
            s["ws"] = torch.empty(mq.mq_w4_product_ws_bytes(M, N, K), dtype=torch.uint8, device=DEV)
        return s
    if c["op"] == "chunk":
        t, hk, dim = TYPES[c["dtype"]], c["kv_heads"], c["dim"]
        new, n = _lengths(c)
        need = -(-n // BLOCK)
        s.update(_cache(int(need.sum()) + 1, hk, dim, g))
        s["table"] = _table(need, int(need.max()), torch.randperm(int(need.sum()), generator=g, device=DEV))
        s["first"], s["lens"] = _i32(np.concatenate([[0], np.cumsum(new)])), _i32(n)
        s["longest"], s["most_new"] = int(n.max()), int(new.max())
        s["q"] = normal(int(new.sum()), c["heads"] * dim).to(t)
        if own:
            import paper_1805_12096_amd as mq
            s["cache"] = mq.KvCache(s["keys"], s["values"], s["amax"], s["blocks"], hk, dim)
            s["ws"] = torch.empty(mq.mq_chunk_attention_ws_bytes(c["batch"], len(s["q"]), s["longest"], c["heads"], hk, dim),
                                  dtype=torch.uint8, device=DEV)
        return s
    if c["op"] == "fork":
        n, full, open_, used, blocks, width = _fork_sizes(c)
        rows = c["rows"]
        s.update(_cache(blocks, c["heads"], c["dim"], g))
        order = torch.randperm(blocks, generator=g, device=DEV)
        # the rows of a group share its whole blocks, the last one is each row's own
        table = _table(full, width, order).repeat_interleave(rows, dim=0)
        last = np.repeat(full, rows)
        has = torch.tensor(np.repeat(open_, rows) > 0, device=DEV)
        fresh = order[int(full.sum()) + torch.cumsum(has.long(), 0) - 1].to(torch.int32)
        at = torch.tensor(last, device=DEV)[:, None].clamp(max=width - 1)
        table.scatter_(1, at, torch.where(has, fresh, table.gather(1, at)[:, 0])[:, None])
        s["table"], s["lens"] = table, _i32(np.repeat(n, rows))
        ways = c["ways"]
        pick = torch.randint(0, rows, (c["groups"], ways), generator=g, device=DEV)
        parent = pick + rows * torch.arange(c["groups"], device=DEV)[:, None]
        parent[torch.rand(parent.shape, generator=g, device=DEV) < 0.05] = -1               # ended
        s["parent"] = parent.reshape(-1).to(torch.int32)
        s["grow"] = torch.full((c["groups"] * ways,), c["grow"], dtype=torch.int32, device=DEV)
        s["keep"] = _kept(c, blocks, g)
    else:
        n = _spread(c["len_lo"], c["len_hi"], c["batch"], c["twist"])
        need = -(-n // BLOCK)
        blocks = max(c["blocks"], int(need.sum()))
        s.update(_cache(blocks, c["heads"], c["dim"], g))
        s["table"] = _table(need, max(1, int(need.max())), torch.randperm(blocks, generator=g, device=DEV))
        s["lens"], s["keep"] = _i32(n), _kept(c, blocks, g)
    if own:
        import paper_1805_12096_amd as mq
        s["cache"] = mq.KvCache(s["keys"], s["values"], s["amax"], s["blocks"], c["heads"], c["dim"])
        if c["op"] == "fork":
            size = mq.mq_kv_fork_ws_bytes(s["blocks"], len(s["parent"]), s["table"].shape[1])
        else:
            size = mq.mq_kv_compact_ws_bytes(s["blocks"])
        s["ws"] = torch.empty(size, dtype=torch.uint8, device=DEV)
    return s


# ---- the operators ----------------------------------------------------------------------------------------------------

def run(state):
    op = state["case"]["op"]
    if own:
        return {"chunk": _own_chunk, "fork": _own_fork, "compact": _own_compact, "norm": _own_norm, "product4": _own_product4}[op](state)
    return {"chunk": _chunk, "fork": _fork, "compact": _compact, "norm": _norm, "product4": _product4}[op](state)


def _own_chunk(s):
    import paper_1805_12096_amd as mq
    c, dim = s["case"], s["case"]["dim"]
    out = torch.empty_like(s["q"])
    mq.mq_chunk_attention(s["cache"], s["table"], s["table"].shape[1], s["first"], s["lens"], c["batch"], len(out), s["longest"],
                          c["causal"], s["q"], s["q"].stride(0), c["heads"], mq.dtype_code(out.dtype), dim ** -0.5, out,
                          out.stride(0), s["ws"], s["ws"].numel())
    return out


def _own_fork(s):
    import paper_1805_12096_amd as mq
    B, width = len(s["parent"]), s["table"].shape[1]
    table = torch.empty((B, width), dtype=torch.int32, device=DEV)
    lens, missing = torch.empty(B, dtype=torch.int32, device=DEV), torch.empty(1, dtype=torch.int32, device=DEV)
    mq.mq_kv_fork(s["cache"], s["keep"], s["table"], width, s["lens"], len(s["lens"]), s["parent"], s["grow"], B, table, lens, missing,
                  s["ws"], s["ws"].numel())
    return [table, lens, missing, s["keys"], s["values"], s["amax"]]


def _own_compact(s):
    import paper_1805_12096_amd as mq
    table = torch.empty_like(s["table"])
    moved, used = torch.empty(s["blocks"], dtype=torch.int32, device=DEV), torch.empty(1, dtype=torch.int32, device=DEV)
    mq.mq_kv_compact(s["cache"], s["keep"], s["table"], table.shape[1], s["lens"], len(table), table, moved, used, s["ws"],
                     s["ws"].numel())
    return [table, moved, used, s["keys"], s["values"], s["amax"]]


def _own_norm(s):
    import paper_1805_12096_amd as mq
    M, d = s["x"].shape
    t = mq.dtype_code(s["x"].dtype)
    h = torch.empty_like(s["x"]) if s["r"] is not None else None
    if s["case"]["form"] == "y":
        y = torch.empty_like(s["x"])
        mq.mq_add_rms_norm(s["x"], d, s["r"], d, t, s["gamma"], M, d, 1e-6, h, d, y, d)
        return [y] if h is None else [y, h]
    q, scale = torch.empty((M, d), dtype=torch.int8, device=DEV), torch.empty(M, device=DEV)
    mq.mq_add_rms_norm_rows8(s["x"], d, s["r"], d, t, s["gamma"], M, d, 1e-6, h, d, q, d, scale)
    return _values8(q, scale) + ([] if h is None else [h])


def _own_product4(s):
    import paper_1805_12096_amd as mq
    M, K = s["x"].shape
    c, N = s["case"], s["case"]["words"]
    y = torch.empty((M, N), dtype=s["out"], device=DEV)
    code = mq.MQ_ROWS8 if s["rowscale"] is not None else mq.dtype_code(s["out"])
    mq.mq_w4_product(s["x"], K, code, s["rowscale"], s["packed"], M, N, K, c["group"], s["bias"], y, N, mq.dtype_code(s["out"]), s["ws"],
                     s["ws"].numel())
    return y


def _values8(q, scale):
    """8-bit rows as the values they stand for (bfloat16 holds all of an 8-bit value's bits), and their multipliers."""
    return [(q.float() / scale[:, None]).bfloat16(), scale]


# ---- plain forms ------------------------------------------------------------------------------------------------------

def _place(t):
    """Where token t of a block lies in a row of the values."""
    return 16 * ((t // 4) % 4) + 4 * (t // 16) + t % 4


def _chunk(s):
    c = s["case"]
    B, hk, dim, L = c["batch"], c["kv_heads"], c["dim"], s["most_new"]
    per, T = c["heads"] // hk, len(s["q"])
    width = -(-s["longest"] // BLOCK)
    at = s["table"][:, :width].long().clamp(min=0)
    step = s["amax"][at] / 127.0                                               # [B, width, hk, 2]
    k = s["keys"][at][..., :dim].float() * step[..., 0, None, None]            # [B, width, hk, 64, dim]
    k = k.permute(0, 2, 1, 3, 4).reshape(B, hk, width * BLOCK, dim)
    v = s["values"][at][:, :, :, :dim].float() * step[..., 1, None, None]      # [B, width, hk, dim, 64]
    v = v.permute(0, 2, 1, 4, 3)[:, :, :, _place(torch.arange(BLOCK, device=DEV))].reshape(B, hk, width * BLOCK, dim)
    f, n = s["first"].long(), s["lens"].long()
    i, j = torch.arange(L, device=DEV), torch.arange(width * BLOCK, device=DEV)
    q = s["q"].float().view(T, hk, per, dim)[(f[:-1, None] + i).clamp(max=T - 1)]
    q = q.permute(0, 2, 3, 1, 4).reshape(B, hk, per * L, dim)
    sc = (torch.matmul(q, k.transpose(-1, -2).contiguous()) * dim ** -0.5).view(B, hk, per, L, width * BLOCK)
    seen = (j < n[:, None])[:, None, :].expand(B, L, width * BLOCK)
    if c["causal"]:
        seen = seen & (j[None, None, :] <= i[None, :, None] + (n - (f[1:] - f[:-1]))[:, None, None])
    sc.masked_fill_(~seen[:, None, None], -math.inf)
    m = sc.amax(-1, keepdim=True).clamp_(min=-3e38)
    p = sc.sub_(m).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(B, hk, per * L, -1), v).view(B, hk, per, L, dim) / torch.where(total > 0, total, torch.ones_like(total))
    t = torch.arange(T, device=DEV)
    b = torch.searchsorted(f[1:].contiguous(), t, right=True)
    return o.permute(0, 3, 1, 2, 4)[b, t - f[b]].reshape(T, -1).to(s["q"].dtype)


def _copied(s, source, target):
    s["keys"][target] = s["keys"][source]
    s["values"][target] = s["values"][source]
    s["amax"][target] = s["amax"][source]


def _fork(s):
    table, parent, grow, blocks = s["table"], s["parent"].long(), s["grow"].long().clamp(min=0), s["blocks"]
    B, width = table.shape
    known = (parent >= 0) & (parent < B)
    p = parent.clamp(0, B - 1)
    n = torch.where(known, s["lens"].long()[p].clamp(0, width * BLOCK), torch.zeros_like(p))
    held, end = -(-n // BLOCK), torch.clamp(-(-(n + grow) // BLOCK), max=width)
    j, e = torch.arange(width, device=DEV), table[p].long()
    there = (j < held[:, None]) & (e >= 0) & (e < blocks)
    written = there & (j == held[:, None] - 1) & (n % BLOCK > 0)[:, None] & (grow > 0)[:, None]
    row = torch.arange(len(p), device=DEV)[:, None].expand_as(e)
    # the lowest row that writes to a block, plus one; 0 where somebody only reads it
    state = torch.full((blocks + 1,), UNUSED, dtype=torch.int64, device=DEV)
    use = torch.where(written, row + 1, torch.zeros_like(row))
    state.scatter_reduce_(0, torch.where(there, e, torch.full_like(e, blocks)).view(-1), use.reshape(-1), "amin")
    state = torch.where(s["keep"] != 0, torch.zeros_like(state[:-1]), state[:-1])
    stays = written & (state[e.clamp(0, blocks - 1)] == row + 1)
    moves = written & ~stays
    wanted = moves | ((j >= held[:, None]) & (j < end[:, None]))
    rank = (torch.cumsum(wanted.view(-1).long(), 0) - 1).view_as(e)
    free = state == UNUSED
    order, room = torch.argsort((~free).to(torch.int32), stable=True), free.sum()
    got = wanted & (rank < room)
    new = torch.where(got, order[rank.clamp(0, blocks - 1)], torch.full_like(e, -1))
    out = torch.where(wanted, new, torch.where(there, e, torch.full_like(e, -1))).to(torch.int32)
    _copied(s, e[moves & got], new[moves & got])
    return [out, n.to(torch.int32), (wanted & ~got).sum().to(torch.int32).view(1), s["keys"], s["values"], s["amax"]]


def _compact(s):
    table, blocks = s["table"].long(), s["blocks"]
    B, width = table.shape
    held = -(-s["lens"].long().clamp(0, width * BLOCK) // BLOCK)
    there = (torch.arange(width, device=DEV) < held[:, None]) & (table >= 0) & (table < blocks)
    used = torch.zeros(blocks + 1, dtype=torch.bool, device=DEV)
    used[torch.where(there, table, torch.full_like(table, blocks)).view(-1)] = True
    used = used[:-1] | (s["keep"] != 0)
    count, i = used.sum(), torch.arange(blocks, device=DEV)
    source, target = i[used & (i >= count)], i[~used & (i < count)]
    moved = torch.where(used, i, torch.full_like(i, -1))
    moved[source] = target
    _copied(s, source, target)
    out = torch.where(there, moved[table.clamp(0, blocks - 1)], torch.full_like(table, -1))
    return [out.to(torch.int32), moved.to(torch.int32), count.to(torch.int32).view(1), s["keys"], s["values"], s["amax"]]


def _norm(s):
    x, gamma = s["x"], s["gamma"]
    h = x if s["r"] is None else (x.float() + s["r"].float()).to(x.dtype)
    if s["case"]["form"] == "y":
        z = h.float()
        y = [(z * torch.rsqrt((z * z).mean(-1, keepdim=True) + 1e-6) * gamma).to(x.dtype)]
    else:                                            # in 64 bits: values next to a half
        z = h.double()
        z = z / torch.sqrt((z * z).mean(-1, keepdim=True) + 1e-6) * gamma.double()
        amax = z.abs().amax(-1)
        scale = torch.where(amax > 0, 127.0 / amax, torch.ones_like(amax))
        y = _values8((z * scale[:, None]).round().clamp(-127, 127), scale.float())
    return y if s["r"] is None else y + [h]


def _product4(s):
    c = s["case"]
    N, K, G = c["words"], c["dim"], c["group"]
    groups = -(-K // G)
    codes = torch.zeros((N, groups * G), device=DEV)
    codes[:, :K] = s["codes"]
    w = ((codes.view(N, groups, G) - s["zeros"].float()[..., None]) * s["scales"][..., None]).view(N, -1)[:, :K]
    x = s["x"].float()
    if s["rowscale"] is not None:
        x = x / s["rowscale"][:, None]
    y = torch.matmul(x, w.t())
    return (y if s["bias"] is None else y + s["bias"]).to(s["out"])


# ---- what a pass cannot do without --------------------------------------------------------------------------------------

def _fork_moves(c):
    """Copies, and blocks, columns and rows of the tables."""
    n, full, open_, used, blocks, width = _fork_sizes(c)
    alive = 0.95 * c["ways"]                         # and so many different rows are picked, about
    lost = int(open_.sum() * (alive - c["rows"] * (1 - (1 - 1 / c["rows"]) ** alive))) if c["grow"] else 0
    return min(lost, c["spare"]), blocks, width, c["groups"] * c["rows"], c["groups"] * c["ways"]


def work(case):
    c = case
    if c["op"] == "norm":
        es = 4 if c["dtype"] == "f32" else 2
        n = c["rows"] * c["dim"]
        rows = n * es * (3 if c["residual"] else 1) + (n + 4 * c["rows"] if c["form"] == "rows8" else n * es)
        return {"bytes": rows + 4 * c["dim"], "flops": 6 * n}
    if c["op"] == "product4":
        M, N, K = c["rows"], c["words"], c["dim"]
        xs, ys = {"rows8": (1, 2), "f32": (4, 4)}.get(c["dtype"], (2, 2))
        return {"bytes": N * K // 2 + 4 * N * -(-K // c["group"]) + xs * M * K + ys * M * N, "flops": 2 * M * N * K}
    if c["op"] == "chunk":
        new, n = _lengths(c)
        es = 4 if c["dtype"] == "f32" else 2
        pairs = np.sum(new * n) - (np.sum(new * (new - 1) // 2) if c["causal"] else 0)
        return {"bytes": int(2 * n.sum() * c["kv_heads"] * c["dim"] + 2 * new.sum() * c["heads"] * c["dim"] * es),
                "flops": int(4 * pairs * c["heads"] * c["dim"])}
    size = BLOCK * c["heads"] * (-(-c["dim"] // 64) * 64 + -(-c["dim"] // 16) * 16) + 8 * c["heads"]
    if c["op"] == "fork":
        copies, blocks, width, rows, new = _fork_moves(c)
        return {"bytes": 2 * size * copies + 4 * (width * (rows + new) + 3 * new + rows + blocks), "flops": new * width}
    need = -(-_spread(c["len_lo"], c["len_hi"], c["batch"], c["twist"]) // BLOCK)
    used, blocks = int(need.sum()), max(c["blocks"], int(need.sum()))
    copies = int((blocks - used) * (used / blocks))                             # of blocks in no order
    return {"bytes": 2 * size * copies + 4 * (2 * blocks + 2 * c["batch"] * max(1, int(need.max()))), "flops": blocks}


# ---- the definitions, in 64 bits ----------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    c = case
    if c["op"] == "norm":
        h = s["x"] if s["r"] is None else (s["x"].double() + s["r"].double()).to(s["x"].dtype)
        y = h.double() * s["gamma"].double() / (h.double().pow(2).sum(-1, keepdim=True) / c["dim"] + 1e-6).sqrt()
        if c["form"] == "rows8":
            top = y.abs().max(dim=-1).values
            step = torch.where(top > 0, top / 127, torch.ones_like(top))
            y = [torch.clamp(torch.round(y / step[:, None]), -127, 127) * step[:, None], 1 / step]
        else:
            y = [y]
        return y if s["r"] is None else y + [h.double()]
    if c["op"] == "product4":
        at = torch.arange(c["dim"], device=DEV) // c["group"]
        w = s["codes"].double().sub_(s["zeros"].double()[:, at]).mul_(s["scales"].double()[:, at])
        x = s["x"].double() if s["rowscale"] is None else s["x"].double() / s["rowscale"].double()[:, None]
        y = x @ w.T.contiguous()
        return y if s["bias"] is None else y + s["bias"].double()
    if c["op"] == "chunk":
        return _exact_chunk(s)
    return _exact_tables(s)


def _exact_chunk(s):
    c = s["case"]
    dim, hk = c["dim"], c["kv_heads"]
    per = c["heads"] // hk
    f, lens, table = s["first"].tolist(), s["lens"].tolist(), s["table"].tolist()
    out = torch.zeros((len(s["q"]), hk * per, dim), dtype=torch.float64, device=DEV)
    order = [_place(t) for t in range(BLOCK)]
    for b, n in enumerate(lens):
        new = f[b + 1] - f[b]
        if n == 0 or new == 0:
            continue
        at = table[b][:-(-n // BLOCK)]
        k = s["keys"][at, :, :, :dim].double() * (s["amax"][at, :, 0].double() / 127)[..., None, None]
        v = s["values"][at, :, :dim][..., order].double() * (s["amax"][at, :, 1].double() / 127)[..., None, None]
        k = k.transpose(0, 1).reshape(hk, -1, dim)[:, :n]
        v = v.permute(1, 0, 3, 2).reshape(hk, -1, dim)[:, :n]
        hidden = torch.arange(n, device=DEV)[None, :] > torch.arange(new, device=DEV)[:, None] + (n - new)
        for h in range(hk * per):
            w = s["q"][f[b]:f[b + 1], h * dim:(h + 1) * dim].double() @ k[h // per].T / math.sqrt(dim)
            if c["causal"]:
                w = w.masked_fill(hidden, -math.inf)
            out[f[b]:f[b + 1], h] = torch.softmax(w, dim=-1) @ v[h // per]
    return out.view(len(out), -1)


def _exact_tables(s):
    """The rules of fork and compact, one entry after the other; of what they give only the scales are no whole numbers."""
    amax, table, blocks = s["amax"].double(), s["table"].tolist(), s["blocks"]
    taken = [x != 0 for x in s["keep"].tolist()]
    lens, width = s["lens"].tolist(), len(table[0])
    if s["case"]["op"] == "compact":
        for b, n in enumerate(lens):
            for e in table[b][:-(-n // BLOCK)]:
                taken[e] = True
        holes = [i for i in range(sum(taken)) if not taken[i]]
        for to, at in zip(holes, [i for i in range(sum(taken), blocks) if taken[i]]):
            amax[to] = amax[at]
        return [None, None, None, None, None, amax]
    rows, writers = [], {}
    for b, (p, more) in enumerate(zip(s["parent"].tolist(), s["grow"].tolist())):
        n = lens[p] if p >= 0 else 0
        e = table[p][:-(-n // BLOCK)] if p >= 0 else []
        opened = n % BLOCK > 0 and more > 0
        rows.append((n, e, opened, more))
        for x in e[:-1] if opened else e:
            taken[x] = True
        if opened:
            writers.setdefault(e[-1], []).append(b)
    first = {x: w[0] for x, w in writers.items() if not taken[x]}
    free = [i for i in range(blocks) if not taken[i] and i not in writers]
    for b, (n, e, opened, more) in enumerate(rows):
        if opened and first.get(e[-1]) != b and free:
            amax[free.pop(0)] = amax[e[-1]]
        for _ in range(min(-(-(n + more) // BLOCK), width) - len(e)):
            if free:
                free.pop(0)
    return [None, None, None, None, None, amax]
