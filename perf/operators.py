"""What is measured of the sequence operators (include/mq_seq.h): cases over their range, their inputs and their plain forms.

The operators: new keys and values into a paged 8-bit cache with the position rotation on the way (append), attention of one
query per sequence over that cache (cached), attention of packed sequences of different lengths (prompt), and the log
probabilities of given words with entropy and the best alternatives (score).  Where `own` is false `run` computes them with
elementary torch operations, where it is true with the library's calls.

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


# ---- cases ------------------------------------------------------------------------------------------------------------

def listed():
    return [
        # one decode step of 300 sentences, width 512 in 8 heads, no rotation: the decoder of the benchmark, latency
        dict(name="append_step", op="append", dtype="f32", batch=300, new_lo=1, new_hi=1, held_lo=0, held_hi=50, heads=8,
             kv_heads=8, dim=64, rot=0, interleaved=False, twist=0.1),
        # a serving step: grouped heads, rotated positions in the thousands
        dict(name="append_step_rotated", op="append", dtype="bf16", batch=64, new_lo=1, new_hi=1, held_lo=500, held_hi=4000,
             heads=32, kv_heads=8, dim=128, rot=128, interleaved=False, twist=0.3),
        # prompts taken in at once: whole blocks and ragged ends, part of the head rotated, pairs interleaved
        dict(name="append_prompts", op="append", dtype="bf16", batch=12, new_lo=300, new_hi=4000, held_lo=0, held_hi=0,
             heads=32, kv_heads=8, dim=128, rot=64, interleaved=True, twist=0.5),
        # one sequence, the least a call can be asked for in earnest
        dict(name="cached_one", op="cached", dtype="f32", batch=1, len_lo=777, len_hi=777, heads=8, kv_heads=8, dim=64,
             twist=0.0),
        # target side of a decode step of 300 sentences: many short, ragged sequences
        dict(name="cached_sentences", op="cached", dtype="f32", batch=300, len_lo=1, len_hi=90, heads=8, kv_heads=8, dim=64,
             twist=0.2),
        # serving with long contexts: the cache streams through once
        dict(name="cached_long", op="cached", dtype="bf16", batch=32, len_lo=4000, len_hi=32000, heads=32, kv_heads=8,
             dim=128, twist=0.7),
        # encoder side of 300 short sentences: no causal mask, all lengths below a tile
        dict(name="prompt_sentences", op="prompt", dtype="f32", batch=300, new_lo=2, new_hi=60, ahead_lo=0, ahead_hi=0,
             heads=8, kv_heads=8, dim=64, causal=False, twist=0.4),
        # forced decoding of about 8192 words in binary32, width 1024 in 16 heads
        dict(name="prompt_documents", op="prompt", dtype="f32", batch=10, new_lo=333, new_hi=1900, ahead_lo=0, ahead_hi=0,
             heads=16, kv_heads=16, dim=64, causal=True, twist=0.6),
        # long prompts, grouped heads
        dict(name="prompt_long", op="prompt", dtype="bf16", batch=3, new_lo=4500, new_hi=8190, ahead_lo=0, ahead_hi=0,
             heads=32, kv_heads=8, dim=128, causal=True, twist=0.1),
        # a handful of words against the 36 000-word vocabulary
        dict(name="score_few", op="score", rows=7, words=36000, dim=512, best=4),
        # the words of one decode batch
        dict(name="score_batch", op="score", rows=384, words=36000, dim=512, best=4),
        # words of a corpus batch through the larger model, log probability and entropy only
        dict(name="score_corpus", op="score", rows=8192, words=36000, dim=1024, best=0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "cached", "prompt", "score"])
    if op == "score":
        dim = rng.choice([64, 192, 500, 512, 512, 777, 1024, 1024])
        words = _log_int(rng, 1000, 50000)
        rows = _log_int(rng, 1, max(1, min(8192, int(2.8e11 / (dim * words)))))
        return dict(op=op, rows=rows, words=words, dim=dim, best=rng.choice([0, 1, 2, 4, 5, 8]))
    dtype = rng.choice(["f32", "f16", "bf16"])
    dim = rng.choice([32, 64, 64, 80, 96, 128, 128, 256])
    kv_heads = rng.choice([1, 2, 4, 5, 8, 16])
    heads = kv_heads * rng.choice([1, 1, 2, 4, 8])
    c = dict(op=op, dtype=dtype, heads=heads, kv_heads=kv_heads, dim=dim, twist=round(rng.random(), 3))
    width = (heads + 2 * kv_heads) * dim
    if op == "append":
        rot = rng.choice([0, dim, dim, dim // 2])
        tokens = min(15000, int(7e7 / width))
        if rng.random() < 0.5:
            held = _log_int(rng, 1, 4000)
            batch = _log_int(rng, 1, max(1, min(512, tokens, int(4e8 / (held * kv_heads * dim)))))
            return dict(c, batch=batch, new_lo=1, new_hi=1, held_lo=held // 4, held_hi=held, rot=rot,
                        interleaved=rng.random() < 0.5)
        hi = _log_int(rng, 3, max(4, min(4000, tokens // 2)))
        held = rng.choice([0, 0, 100, 1000])
        return dict(c, batch=max(1, min(300, tokens // hi, int(4e8 / ((held + hi) * kv_heads * dim)))),
                    new_lo=max(1, hi // 10), new_hi=hi, held_lo=held // 3, held_hi=held, rot=rot,
                    interleaved=rng.random() < 0.5)
    if op == "cached":
        hi = _log_int(rng, 1, 32000)
        room = int(4e8 / (hi * kv_heads * dim))
        return dict(c, batch=_log_int(rng, 1, max(1, min(512, room))), len_lo=rng.choice([0, hi // 8, hi]), len_hi=hi)
    hi = _log_int(rng, 1, 6000)
    ahead = rng.choice([0, 0, hi // 2])
    room = min(int(8e7 / (hi * width)), int(7e11 / (4 * dim * heads * hi * (hi + ahead))))
    return dict(c, batch=max(1, min(300, room)), new_lo=max(1, hi // 8), new_hi=hi, ahead_lo=0, ahead_hi=ahead,
                causal=rng.random() < 0.7)


# ---- inputs -----------------------------------------------------------------------------------------------------------

def _spread(lo, hi, n, twist):
    """n whole numbers from lo to hi, spread evenly over the logarithm."""
    u = (twist + 0.6180339887498949 * np.arange(1, n + 1)) % 1.0
    x = np.exp(np.log(lo + 1.0) + u * (np.log(hi + 1.0) - np.log(lo + 1.0))) - 1.0
    return np.clip(np.rint(x), lo, hi).astype(np.int64)


def _lengths(c):
    if c["op"] == "append":
        return _spread(c["new_lo"], c["new_hi"], c["batch"], c["twist"]), _spread(c["held_lo"], c["held_hi"], c["batch"], c["twist"] + 0.37)
    if c["op"] == "cached":
        return _spread(c["len_lo"], c["len_hi"], c["batch"], c["twist"])
    new = _spread(c["new_lo"], c["new_hi"], c["batch"], c["twist"])
    return new, new + _spread(c["ahead_lo"], c["ahead_hi"], c["batch"], c["twist"] + 0.37)


def _firsts(n):
    return torch.tensor(np.concatenate([[0], np.cumsum(n)]).astype(np.int32), device=DEV)


def _cache(c, tokens, g):
    """A cache whose sequences hold `tokens` tokens, in blocks of no order, and its table."""
    need = -(-tokens // BLOCK)
    blocks, width = int(need.sum()), max(1, int(need.max()))
    order = torch.randperm(blocks, generator=g, device=DEV).to(torch.int32)
    table = torch.full((len(tokens), width), -1, dtype=torch.int32, device=DEV)
    at = torch.arange(width, device=DEV)[None, :] < torch.tensor(need, device=DEV)[:, None]
    table[at] = order
    dk, dv = -(-c["dim"] // 64) * 64, -(-c["dim"] // 16) * 16
    hk = c["kv_heads"]
    blocks += 1          # and one that no sequence has

    def ints(shape):          # as unit normal values with their largest at 127 come out, about
        return torch.randint(-90, 91, shape, generator=g, device=DEV, dtype=torch.int8)

    keys, values = ints((blocks, hk, BLOCK, dk)), ints((blocks, hk, dv, BLOCK))
    keys[..., c["dim"]:] = 0
    values[:, :, c["dim"]:] = 0
    amax = 2.5 + 2.0 * torch.rand((blocks, hk, 2), generator=g, device=DEV)
    return dict(keys=keys, values=values, amax=amax, table=table, blocks=blocks)


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=DEV)

    s = dict(case=c)
    if c["op"] == "score":
        M, N, K = c["rows"], c["words"], c["dim"]
        # 8-bit hidden states and embedding with the multipliers that go with them; peaked rows as a trained model has
        s["qA"] = (normal(M, K) * 30).round_().clamp_(-127, 127).to(torch.int8)
        s["qW"] = (normal(N, K) * 30).round_().clamp_(-127, 127).to(torch.int8)
        s["sA"] = torch.full((1,), 30.0, device=DEV)
        s["sW"] = torch.full((1,), 30.0 * math.sqrt(K) / 3.0, device=DEV)
        target = torch.randint(0, N, (M,), generator=g, device=DEV, dtype=torch.int32)
        target[torch.rand(M, generator=g, device=DEV) < 0.05] = -1          # padded places
        s["target"] = target
        s["A"], s["W"] = s["qA"].float(), s["qW"].float()
        if own:
            import paper_1805_12096_amd as mq
            one = torch.ones(1, device=DEV)
            s["pW"] = mq.prepare_weight(s["W"], 8, scale=one).packed
            s["pA"] = torch.empty(mq.mq_packed_bytes(8, M, K), dtype=torch.uint8, device=DEV)
            mq.mq_quantize_pack_f32(s["A"], M, K, 8, one, s["pA"])
            s["ws"] = torch.empty(mq.mq_token_logprob_ws_bytes(M, N, c["best"]), dtype=torch.uint8, device=DEV)
        return s
    t, hk, dim = TYPES[c["dtype"]], c["kv_heads"], c["dim"]
    width = (c["heads"] + 2 * hk) * dim
    if c["op"] == "cached":
        n = _lengths(c)
        s.update(_cache(c, n, g))
        s["lens"] = torch.tensor(n.astype(np.int32), device=DEV)
        s["longest"] = max(1, int(n.max()))
        s["q"] = normal(c["batch"], c["heads"] * dim).to(t)
        if own:
            import paper_1805_12096_amd as mq
            s["cache"] = mq.KvCache(s["keys"], s["values"], s["amax"], s["blocks"], hk, dim)
            s["ws"] = torch.empty(mq.mq_cached_attention_ws_bytes(c["batch"], s["longest"], c["heads"], hk, dim),
                                  dtype=torch.uint8, device=DEV)
        return s
    if c["op"] == "append":
        n, held = _lengths(c)
        s.update(_cache(c, n + held, g))
        s["first"], s["held"] = _firsts(n), torch.tensor(held.astype(np.int32), device=DEV)
        s["longest"] = int(n.max())
        T = int(n.sum())
        if c["rot"]:
            s["freq"] = torch.tensor(10000.0 ** (-np.arange(0, c["rot"], 2) / c["rot"]), dtype=torch.float32, device=DEV)
        if own:
            import paper_1805_12096_amd as mq
            s["cache"] = mq.KvCache(s["keys"], s["values"], s["amax"], s["blocks"], hk, dim)
    else:
        n, nk = _lengths(c)
        T, Tk = int(n.sum()), int(nk.sum())
        s["first"], s["k_first"] = _firsts(n), _firsts(nk)
        s["longest"], s["k_longest"] = int(n.max()), int(nk.max())
        if own:
            import paper_1805_12096_amd as mq
            s["ws"] = torch.empty(mq.mq_prompt_attention_ws_bytes(mq.dtype_code(t), c["batch"], Tk, hk, dim), dtype=torch.uint8,
                                  device=DEV)
        if Tk != T:
            s["q"] = normal(T, c["heads"] * dim).to(t)
            kv = normal(Tk, 2 * hk * dim).to(t)
            s["k"], s["v"] = kv[:, :hk * dim], kv[:, hk * dim:]
            return s
    # one product gives queries, keys and values next to each other, as the layers have them
    x = normal(T, width).to(t)
    s["q"], s["k"], s["v"] = x[:, :c["heads"] * dim], x[:, c["heads"] * dim:(c["heads"] + hk) * dim], x[:, (c["heads"] + hk) * dim:]
    return s


# ---- the operators ----------------------------------------------------------------------------------------------------

def run(state):
    op = state["case"]["op"]
    if own:
        return {"append": _own_append, "cached": _own_cached, "prompt": _own_prompt, "score": _own_score}[op](state)
    return {"append": _append, "cached": _cached, "prompt": _prompt, "score": _score}[op](state)


def _own_append(s):
    import paper_1805_12096_amd as mq
    c, dim, T = s["case"], s["case"]["dim"], s["q"].shape[0]
    rotated = bool(c["rot"])
    q_out = torch.empty((T, c["heads"] * dim), dtype=s["q"].dtype, device=DEV) if rotated else None
    k_out = torch.empty((T, c["kv_heads"] * dim), dtype=s["q"].dtype, device=DEV) if rotated else None
    mq.mq_kv_append(s["cache"], s["table"], s["table"].shape[1], s["first"], s["held"], c["batch"], T,
                    s["k"], s["k"].stride(0), s["v"], s["v"].stride(0), s["q"] if rotated else None, s["q"].stride(0),
                    c["heads"], mq.dtype_code(s["q"].dtype), s["freq"] if rotated else None, c["rot"], c["interleaved"],
                    k_out, q_out)
    return [s["keys"], s["values"], s["amax"]] + ([q_out, k_out] if rotated else [])


def _own_cached(s):
    import paper_1805_12096_amd as mq
    c, dim = s["case"], s["case"]["dim"]
    out = torch.empty((c["batch"], c["heads"] * dim), dtype=s["q"].dtype, device=DEV)
    mq.mq_cached_attention(s["cache"], s["table"], s["table"].shape[1], s["lens"], c["batch"], s["longest"], s["q"],
                           s["q"].stride(0), c["heads"], mq.dtype_code(s["q"].dtype), dim ** -0.5, out, out.stride(0), s["ws"],
                           s["ws"].numel())
    return out


def _own_prompt(s):
    import paper_1805_12096_amd as mq
    c, dim = s["case"], s["case"]["dim"]
    out = torch.empty((s["q"].shape[0], c["heads"] * dim), dtype=s["q"].dtype, device=DEV)
    mq.mq_prompt_attention(s["q"], s["q"].stride(0), s["k"], s["k"].stride(0), s["v"], s["v"].stride(0),
                           mq.dtype_code(s["q"].dtype), s["first"], s["k_first"], c["batch"], s["q"].shape[0], s["k"].shape[0],
                           c["heads"], c["kv_heads"], dim, c["causal"], dim ** -0.5, out, out.stride(0), s["ws"],
                           s["ws"].numel())
    return out


def _own_score(s):
    import paper_1805_12096_amd as mq
    c = s["case"]
    M, N, K, best = c["rows"], c["words"], c["dim"], c["best"]
    logprob, entropy = torch.empty(M, device=DEV), torch.empty(M, device=DEV)
    tok = torch.empty((M, best), dtype=torch.int32, device=DEV) if best else None
    alt = torch.empty((M, best), device=DEV) if best else None
    mq.mq_gemm_token_logprob_packed(s["pA"], s["pW"], M, N, K, s["sA"], s["sW"], s["target"], best, logprob, entropy, tok, alt,
                                    s["ws"], s["ws"].numel())
    return [logprob, entropy] + ([tok, alt] if best else [])


# ---- plain forms ------------------------------------------------------------------------------------------------------

def _place(t):
    """Where token t of a block lies in a row of the values."""
    return 16 * ((t // 4) % 4) + 4 * (t // 16) + t % 4


def _rotated(x, pos, freq, rot, interleaved):
    """x [T, heads, dim] rotated by position, in 64 bits, rounded to binary32."""
    if not rot:
        return x.float()
    a = pos.double()[:, None, None] * freq.double()
    cos, sin = a.cos(), a.sin()
    d = x.double()
    if interleaved:
        u, v = d[..., 0:rot:2], d[..., 1:rot:2]
        y = torch.stack([u * cos - v * sin, v * cos + u * sin], dim=-1).flatten(-2)
    else:
        u, v = d[..., :rot // 2], d[..., rot // 2:rot]
        y = torch.cat([u * cos - v * sin, v * cos + u * sin], dim=-1)
    return torch.cat([y, d[..., rot:]], dim=-1).float()


def _append(s):
    c = s["case"]
    hk, dim, T, B = c["kv_heads"], c["dim"], s["q"].shape[0], c["batch"]
    first, held, table, keys, values, amax = (s[k] for k in ("first", "held", "table", "keys", "values", "amax"))
    t = torch.arange(T, device=DEV)
    b = torch.searchsorted(first[1:].long(), t, right=True)
    pos = held[b].long() + t - first[b].long()
    k = _rotated(s["k"].view(T, hk, dim), pos, s.get("freq"), c["rot"], c["interleaved"])
    v = s["v"].view(T, hk, dim).float()
    out = []
    if c["rot"]:
        q = _rotated(s["q"].view(T, c["heads"], dim), pos, s["freq"], c["rot"], c["interleaved"])
        out = [q.reshape(T, -1).to(s["q"].dtype), k.reshape(T, -1).to(s["q"].dtype)]
    block, place = table[b, pos // BLOCK].long(), pos % BLOCK
    # the blocks a call touches: of each sequence, the one with its first new token and those after it; places past a
    # sequence's end stand for the spare block, which gets what it has
    spare = len(amax) - 1
    span = (s["longest"] + 2 * BLOCK - 2) // BLOCK
    col = (held.long() // BLOCK)[:, None] + torch.arange(span, device=DEV)
    end = held.long() + (first[1:] - first[:-1]).long()
    live = col * BLOCK < end[:, None]
    at = torch.where(live, table.gather(1, col.clamp(max=table.shape[1] - 1)).long(), torch.full_like(col, spare)).view(-1)
    fresh = (live & (col * BLOCK >= held.long()[:, None])).view(-1)
    new = torch.zeros_like(amax)
    new.index_reduce_(0, block, torch.stack([k.abs().amax(-1), v.abs().amax(-1)], dim=-1), "amax")
    old = torch.where(fresh[:, None, None], torch.zeros_like(new[at]), amax[at])
    a = torch.maximum(old, new[at])
    one = torch.ones_like(a)
    ratio = torch.where(a > 0, old / a, one)
    scale = torch.ones_like(amax)
    scale[at] = torch.where(a > 0, 127.0 * one / a, one)
    keys[at] = (keys[at].float() * ratio[:, :, 0, None, None]).round().clamp(-127, 127).to(torch.int8)
    values[at] = (values[at].float() * ratio[:, :, 1, None, None]).round().clamp(-127, 127).to(torch.int8)
    amax[at] = a
    sk, sv = scale[block, :, 0, None], scale[block, :, 1, None]
    keys[block, :, place, :dim] = (k * sk).round().clamp(-127, 127).to(torch.int8)
    values.transpose(2, 3)[block, :, _place(place), :dim] = (v * sv).round().clamp(-127, 127).to(torch.int8)
    return [keys, values, amax] + out


def _softmax_product(sc, seen, v):
    """softmax over the places seen of sc [.., q, k], times v [.., k, d]; rows that see nothing give 0."""
    sc.masked_fill_(~seen, -math.inf)
    m = sc.amax(-1, keepdim=True).clamp_(min=-3e38)
    p = sc.sub_(m).exp_()
    total = p.sum(-1, keepdim=True)
    return torch.matmul(p, v) / torch.where(total > 0, total, torch.ones_like(total))


def _cached(s):
    c = s["case"]
    B, hk, dim = c["batch"], c["kv_heads"], c["dim"]
    per = c["heads"] // hk
    width = -(-s["longest"] // BLOCK)
    at = s["table"][:, :width].long().clamp(min=0)
    step = s["amax"][at] / 127.0                                               # [B, width, hk, 2]
    k = s["keys"][at][..., :dim].float() * step[..., 0, None, None]            # [B, width, hk, 64, dim]
    k = k.permute(0, 2, 1, 3, 4).reshape(B, hk, width * BLOCK, dim)
    place = _place(torch.arange(BLOCK, device=DEV))
    v = s["values"][at][:, :, :, :dim].float() * step[..., 1, None, None]      # [B, width, hk, dim, 64]
    v = v.permute(0, 2, 1, 4, 3)[:, :, :, place].reshape(B, hk, width * BLOCK, dim)
    q = s["q"].float().view(B, hk, per, dim)
    sc = torch.matmul(q, k.transpose(-1, -2)) * dim ** -0.5
    seen = torch.arange(width * BLOCK, device=DEV)[None, :] < s["lens"][:, None]
    o = _softmax_product(sc, seen[:, None, None, :].expand_as(sc), v)
    return o.reshape(B, -1).to(s["q"].dtype)


def _prompt(s):
    c = s["case"]
    hk, dim, B = c["kv_heads"], c["dim"], c["batch"]
    per, L, Lk = c["heads"] // hk, s["longest"], s["k_longest"]
    f, fk = s["first"].long(), s["k_first"].long()
    n, nk = f[1:] - f[:-1], fk[1:] - fk[:-1]
    i, j = torch.arange(L, device=DEV), torch.arange(Lk, device=DEV)
    T, Tk = s["q"].shape[0], s["k"].shape[0]
    qi, kj = (f[:-1, None] + i).clamp(max=T - 1), (fk[:-1, None] + j).clamp(max=Tk - 1)
    q = s["q"].float().view(T, hk, per, dim)[qi].permute(0, 2, 3, 1, 4).reshape(B, hk, per * L, dim)
    k = s["k"].float().reshape(Tk, hk, dim)[kj].permute(0, 2, 1, 3)
    v = s["v"].float().reshape(Tk, hk, dim)[kj].permute(0, 2, 1, 3)
    sc = (torch.matmul(q, k.transpose(-1, -2)) * dim ** -0.5).view(B, hk, per, L, Lk)
    seen = (j < nk[:, None])[:, None, :].expand(B, L, Lk)
    if c["causal"]:
        seen = seen & (j[None, None, :] <= i[None, :, None] + (nk - n)[:, None, None])
    o = _softmax_product(sc, seen[:, None, None].expand_as(sc), v[:, :, None])      # [B, hk, per, L, dim]
    t = torch.arange(T, device=DEV)
    b = torch.searchsorted(f[1:], t, right=True)
    return o.permute(0, 3, 1, 2, 4)[b, t - f[b]].reshape(T, -1).to(s["q"].dtype)


def _score(s):
    c = s["case"]
    N, best = c["words"], c["best"]
    acc = torch.matmul(s["A"], s["W"].t())                       # whole numbers below 2^24: exact
    u = 1.0 / (s["sA"] * s["sW"])
    y = acc * u
    m = y.amax(-1, keepdim=True)
    z = y - m
    e = z.exp()
    total = e.sum(-1)
    norm = total.log()
    target = s["target"].long()
    there = target >= 0
    logprob = torch.where(there, z.gather(1, target.clamp(min=0)[:, None])[:, 0] - norm, torch.zeros_like(norm))
    out = [logprob, norm - (e * z).sum(-1) / total]
    if best:                                                      # largest sum first, lowest index first among equals
        key = acc.to(torch.int64) * N + (N - 1 - torch.arange(N, device=DEV))
        tok = N - 1 - torch.topk(key, best, dim=-1).values % N
        out += [tok.to(torch.int32), z.gather(1, tok) - norm[:, None]]
    return out


# ---- what a pass cannot do without --------------------------------------------------------------------------------------

def work(case):
    c = case
    if c["op"] == "score":
        M, N, K = c["rows"], c["words"], c["dim"]
        return {"bytes": M * K + N * K + 12 * M + 8 * M * c["best"], "flops": 2 * M * N * K}
    es = 4 if c["dtype"] == "f32" else 2
    h, hk, d = c["heads"], c["kv_heads"], c["dim"]
    if c["op"] == "append":
        T = int(_lengths(c)[0].sum())
        moved = T * d * es * 2 * hk + 2 * T * hk * d + T * hk * 8 // BLOCK
        return {"bytes": moved + (T * d * es * (2 * h + hk) if c["rot"] else 0), "flops": 4 * T * hk * d}
    if c["op"] == "cached":
        n = int(_lengths(c).sum())
        return {"bytes": 2 * n * hk * d + 2 * c["batch"] * h * d * es, "flops": 4 * n * h * d}
    n, nk = _lengths(c)
    pairs = np.sum(n * nk)
    if c["causal"]:
        pairs -= np.sum(n * (n - 1) // 2)
    return {"bytes": int(n.sum()) * 2 * h * d * es + int(nk.sum()) * 2 * hk * d * es, "flops": int(4 * pairs * h * d)}


# ---- the definitions, in 64 bits ----------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    c = case
    if c["op"] == "score":
        return _exact_score(s)
    if c["op"] == "append":
        return _exact_append(s)
    dim, hk = c["dim"], c["kv_heads"]
    per = c["heads"] // hk
    if c["op"] == "cached":
        lens, table = s["lens"].tolist(), s["table"].tolist()
        out = torch.zeros((c["batch"], hk, per, dim), dtype=torch.float64, device=DEV)
        order = [_place(t) for t in range(BLOCK)]
        for b, n in enumerate(lens):
            if n == 0:
                continue
            at = table[b][:-(-n // BLOCK)]
            k = s["keys"][at, :, :, :dim].double() * (s["amax"][at, :, 0].double() / 127)[..., None, None]
            v = s["values"][at, :, :dim][..., order].double() * (s["amax"][at, :, 1].double() / 127)[..., None, None]
            k = k.transpose(0, 1).reshape(hk, -1, dim)[:, :n]
            v = v.permute(1, 0, 3, 2).reshape(hk, -1, dim)[:, :n]
            for h in range(hk):
                w = torch.softmax(s["q"][b].double().view(hk, per, dim)[h] @ k[h].T / math.sqrt(dim), dim=-1)
                out[b, h] = w @ v[h]
        return out.view(c["batch"], -1)
    f, fk = s["first"].tolist(), s["k_first"].tolist()
    out = torch.zeros((s["q"].shape[0], hk * per, dim), dtype=torch.float64, device=DEV)
    for b in range(c["batch"]):
        n, nk = f[b + 1] - f[b], fk[b + 1] - fk[b]
        hidden = torch.arange(nk, device=DEV)[None, :] > torch.arange(n, device=DEV)[:, None] + (nk - n)
        for h in range(hk * per):
            kv = slice((h // per) * dim, (h // per + 1) * dim)
            k, v = s["k"][fk[b]:fk[b + 1], kv].double(), s["v"][fk[b]:fk[b + 1], kv].double()
            w = s["q"][f[b]:f[b + 1], h * dim:(h + 1) * dim].double() @ k.T / math.sqrt(dim)
            if c["causal"]:
                w = w.masked_fill(hidden, -math.inf)
            out[f[b]:f[b + 1], h] = torch.softmax(w, dim=-1) @ v
    return out.view(len(out), -1)


def _exact_score(s):
    c, N = s["case"], s["case"]["words"]
    u = 1.0 / (float(s["sA"]) * float(s["sW"]))
    found = []
    for at in range(0, c["rows"], 512):
        rows = slice(at, at + 512)
        y = s["qA"][rows].double() @ s["qW"].double().T * u
        p = torch.log_softmax(y, dim=-1)
        t = s["target"][rows].long()
        one = [torch.where(t >= 0, p[torch.arange(len(t), device=DEV), t.clamp(min=0)], torch.zeros_like(p[:, 0])),
               -(p.exp() * p).sum(-1)]
        if c["best"]:
            one += [p.sort(dim=-1, descending=True).values[:, :c["best"]]]
        found.append(one)
    got = [torch.cat(x) for x in zip(*found)]
    return got[:2] + ([None, got[2]] if c["best"] else [])


def _exact_append(s):
    c = s["case"]
    hk, dim, half = c["kv_heads"], c["dim"], c["rot"] // 2
    f, held, table = s["first"].tolist(), s["held"].tolist(), s["table"].tolist()
    T = f[-1]
    pos = torch.cat([torch.arange(held[b], held[b] + f[b + 1] - f[b], device=DEV) for b in range(c["batch"])])

    def turn(x, heads):
        x = x.double().reshape(T, heads, dim).clone()
        if half:
            angle = pos.double()[:, None] * s["freq"].double()[None]
            w = torch.polar(torch.ones_like(angle), angle)[:, None]
            one = list(range(0, 2 * half, 2)) if c["interleaved"] else list(range(half))
            two = list(range(1, 2 * half, 2)) if c["interleaved"] else list(range(half, 2 * half))
            z = torch.complex(x[..., one], x[..., two]) * w
            x[..., one], x[..., two] = z.real.contiguous(), z.imag.contiguous()
        return x

    k, v = turn(s["k"], hk), s["v"].double().reshape(T, hk, dim)
    amax = s["amax"].double().clone()
    for b in range(c["batch"]):
        at = held[b]
        while at < held[b] + f[b + 1] - f[b]:
            end = min((at // BLOCK + 1) * BLOCK, held[b] + f[b + 1] - f[b])
            rows = slice(f[b] + at - held[b], f[b] + end - held[b])
            block = table[b][at // BLOCK]
            had = amax[block] if at % BLOCK else torch.zeros_like(amax[block])
            amax[block] = torch.maximum(had, torch.stack([k[rows].abs().amax((0, 2)), v[rows].abs().amax((0, 2))], dim=-1))
            at = end
    out = [None, None, amax]
    if half:
        out += [turn(s["q"], c["heads"]).view(T, -1), k.view(T, -1)]
    return out
