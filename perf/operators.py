"""What serving a chunk of new tokens over a paged key/value cache is measured by: rotary positions, the append of a chunk's
keys and values to their pages, the attention of the chunk over those pages, and copies of pages (forks of a sequence,
compaction).

A page ("block") of one layer holds [K|V][key/value head][position in the block][feature]; a sequence lists its blocks in a
row of the block table.  The new tokens of a batch lie packed, sequence after sequence (cu_seqlens); len counts a
sequence's positions with the new ones, so the last of its new tokens has position len - 1.

A case's lengths and where its blocks lie are drawn from the case alone, so that a case is the same work for every seed;
the values are drawn from the seed.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
TORCH_TYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
CODE = {"f32": 0, "bf16": 1}


def _attention(dtype, heads, kv_heads, dim, block, singles, chunks, new_lo, new_hi, ctx_lo, ctx_hi, window=0):
    """`singles` sequences bring one new token, `chunks` bring new_lo to new_hi; ctx: positions with the new ones."""
    return {"op": "attention", "dtype": dtype, "heads": heads, "kv_heads": kv_heads, "dim": dim, "block": block, "singles": singles,
            "chunks": chunks, "new_lo": new_lo, "new_hi": new_hi, "ctx_lo": ctx_lo, "ctx_hi": ctx_hi, "window": window}


def _append(dtype, heads, kv_heads, dim, rot, interleaved, block, singles, chunks, new_lo, new_hi, ctx_lo, ctx_hi):
    c = _attention(dtype, heads, kv_heads, dim, block, singles, chunks, new_lo, new_hi, ctx_lo, ctx_hi)
    del c["window"]
    c.update(op="append", rot=rot, interleaved=interleaved)
    return c


def _rotary(dtype, tokens, heads, dim, rot, interleaved, far):
    return {"op": "rotary", "dtype": dtype, "tokens": tokens, "heads": heads, "dim": dim, "rot": rot, "interleaved": interleaved,
            "far": far}


def _copy(dtype, layers, blocks, block, kv_heads, dim, copies, rows_lo, rows_hi, one_source):
    return {"op": "copy", "dtype": dtype, "layers": layers, "blocks": blocks, "block": block, "kv_heads": kv_heads, "dim": dim,
            "copies": copies, "rows_lo": rows_lo, "rows_hi": rows_hi, "one_source": one_source}


def listed():
    named = {
        # One interactive request at the OPT-13B shape, one new token: the smallest call, where latency counts.
        "attn_one_token": _attention("bf16", 40, 40, 128, 64, 1, 0, 1, 1, 576, 576),
        # A decode batch of long ragged contexts, four query heads to a key/value head, small pages: streams 1 GB of cache.
        "attn_decode_64_grouped": _attention("bf16", 32, 8, 128, 16, 64, 0, 1, 1, 500, 8100),
        # Chunks of prompts whose first part is cached, OPT-13B heads.
        "attn_chunks_opt13b": _attention("bf16", 40, 40, 128, 64, 0, 8, 97, 256, 400, 1280),
        # One long document fed in chunks: 2048 tokens behind 30720 cached ones.
        "attn_long_chunk_grouped": _attention("bf16", 32, 8, 128, 64, 0, 1, 2048, 2048, 32768, 32768),
        # Decode rows and two prompt chunks in one call, sliding window, 64-wide heads.
        "attn_mixed_window": _attention("bf16", 32, 4, 64, 32, 24, 2, 350, 512, 900, 6000, window=1024),
        # The float path, in which a model is checked before it is served in bf16.
        "attn_chunks_f32": _attention("f32", 12, 4, 64, 8, 1, 4, 33, 120, 150, 900),
        # Queries and keys of one token, far into a long context.
        "rotary_one_token": _rotary("bf16", 1, 40, 128, 128, 0, 1000000),
        # Queries and keys of a long prompt, half of every head turned, neighbours paired, in float.
        "rotary_prompt_f32": _rotary("f32", 4099, 40, 128, 64, 1, 4200),
        # A decode batch appends a token each.
        "append_decode_64": _append("bf16", 32, 8, 128, 128, 0, 16, 64, 0, 1, 1, 500, 8100),
        # Prompt chunks at the OPT-13B widths, neighbours paired.
        "append_chunks_opt13b": _append("bf16", 40, 40, 128, 128, 1, 64, 0, 8, 300, 700, 700, 1280),
        # A prompt forked into eight candidates: the last page, partly filled, of all 40 layers, once for each.
        "copy_fork_8": _copy("bf16", 40, 12, 64, 40, 128, 8, 37, 37, 1),
        # Compaction: whole pages out of the upper part of a pool into holes of the lower one.
        "copy_compact": _copy("bf16", 8, 200, 64, 40, 128, 90, 64, 64, 0),
    }
    return [dict(c, name=n) for n, c in named.items()]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw_heads(rng, most):
    kv = rng.choice([1, 2, 3, 4, 5, 8, 8, 16])
    return kv * rng.choice([g for g in (1, 1, 2, 3, 4, 6, 8) if kv * g <= most]), kv


def draw(rng):
    """One more case of the same ranges, sizes over their logarithm, none of more work than the largest listed one."""
    kind = rng.choice(["decode", "decode", "chunks", "chunks", "long", "mixed", "f32", "rotary", "append", "append", "copy"])
    block = rng.choice([8, 16, 32, 64, 128])
    dim = rng.choice([64, 128, 128])
    if kind == "decode":
        h, kv = _draw_heads(rng, 40)
        n, hi = _log_int(rng, 1, 96), _log_int(rng, 40, 9000)
        hi = min(hi, 500000 // n)
        return _attention("bf16", h, kv, dim, block, n, 0, 1, 1, max(1, hi // rng.choice([1, 2, 9])), hi, rng.choice([0, 0, 0, 700]))
    if kind == "chunks":
        h, kv = _draw_heads(rng, 40)
        n, m = _log_int(rng, 1, 12), _log_int(rng, 2, 700)
        return _attention("bf16", h, kv, dim, block, 0, n, max(1, m // 2), m, m, m + _log_int(rng, 1, 1500), rng.choice([0, 0, 0, 300]))
    if kind == "long":
        h, kv = _draw_heads(rng, 32)
        m = _log_int(rng, 3, 1900)
        ctx = m + _log_int(rng, 2000, 30000)
        return _attention("bf16", h, kv, dim, block, 0, 1, m, m, ctx, ctx, rng.choice([0, 0, 4097]))
    if kind == "mixed":
        h, kv = _draw_heads(rng, 32)
        m = _log_int(rng, 16, 500)
        return _attention("bf16", h, kv, dim, block, _log_int(rng, 1, 30), rng.randint(1, 3), max(1, m // 3), m, m, m + _log_int(rng, 30, 4000),
                          rng.choice([0, 0, 1000]))
    if kind == "f32":
        h, kv = _draw_heads(rng, 16)
        m = _log_int(rng, 1, 150)
        return _attention("f32", h, kv, dim, block, rng.randint(1, 8), rng.randint(0, 4), 1, m, m, m + _log_int(rng, 1, 900),
                          rng.choice([0, 0, 100]))
    if kind == "rotary":
        rot = rng.choice([dim, dim // 2, 2 * rng.randint(1, dim // 2)])
        return _rotary(rng.choice(["f32", "bf16"]), _log_int(rng, 1, 6000), rng.randint(1, 48), dim, rot, rng.randint(0, 1),
                       _log_int(rng, 100, 1000000))
    if kind == "append":
        h, kv = _draw_heads(rng, 40)
        rot = rng.choice([dim, dim, dim // 2, 2 * rng.randint(0, dim // 2)])
        m = _log_int(rng, 1, 700)
        return _append(rng.choice(["f32", "bf16", "bf16"]), h, kv, dim, rot, rng.randint(0, 1), block, _log_int(rng, 1, 64), rng.randint(0, 5),
                       max(1, m // 3), m, m, m + _log_int(rng, 1, 3500))
    kv = rng.choice([1, 4, 8, 40])
    layers, one = rng.randint(1, 40), rng.randint(0, 1)
    copies = _log_int(rng, 1, 96)
    # the pool: at most 2 GiB
    blocks = min(2 * copies + rng.randint(2, 60), max(4, (2 << 30) // (layers * 2 * kv * block * dim * 2)))
    lo = rng.randint(1, block)
    return _copy("bf16", layers, blocks, block, kv, dim, max(1, min(copies, blocks // 2 - 1)), lo, rng.choice([lo, block]), one)


class _State:
    pass


def _lengths(case):
    """(new tokens, positions with them) of every sequence, from the case alone; single tokens and chunks shuffled."""
    rng = np.random.default_rng([case[k] for k in ("singles", "chunks", "new_hi", "ctx_lo", "ctx_hi", "block")])
    new = np.concatenate([np.ones(case["singles"], dtype=np.int64),
                          rng.integers(case["new_lo"], case["new_hi"] + 1, size=case["chunks"])])
    rng.shuffle(new)
    ctx = rng.integers(case["ctx_lo"], case["ctx_hi"] + 1, size=len(new))
    return new, np.maximum(new, ctx)


def _frequencies(rot, far):
    """Radians per position of every pair; for contexts beyond 8192 the slow ones stretched by 8, the fast ones left,
    a ramp between (by turns over 8192 positions), and the amplitude that goes with it."""
    f = 10000.0 ** (-np.arange(0, rot, 2, dtype=np.float64) / max(rot, 1))
    if far <= 8192:
        return f, 1.0
    keep = np.clip((8192 * f / (2 * math.pi) - 1.0) / (32.0 - 1.0), 0.0, 1.0)
    return f * keep + f / 8 * (1.0 - keep), 0.1 * math.log(8.0) + 1.0


def _rand(gen, shape, dtype, scale=1.0):
    t = torch.randn(shape, generator=gen, device=DEV, dtype=TORCH_TYPE[dtype])
    return t.mul_(scale) if scale != 1.0 else t


def _ints(a):
    return torch.as_tensor(np.ascontiguousarray(a), dtype=torch.int32, device=DEV)


def prepare(case, seed):
    s = _State()
    s.case = case
    gen = torch.Generator(device=DEV).manual_seed(int(seed))
    rng = np.random.default_rng(seed)
    t, d = case["dtype"], case["dim"]
    if case["op"] == "rotary":
        n, h = case["tokens"], case["heads"]
        s.x = _rand(gen, (n, h * d), t)
        s.pos = _ints(rng.integers(0, case["far"], size=n))
        f, s.amplitude = _frequencies(case["rot"], case["far"])
        s.inv_freq = torch.as_tensor(f, device=DEV)
        s.out = torch.empty_like(s.x)
        return s
    if case["op"] == "copy":
        L, B, k = case["layers"], case["blocks"], case["copies"]
        s.pool = _rand(gen, (L, B, 2, case["kv_heads"], case["block"], d), t)
        order = rng.permutation(B)
        src = np.repeat(order[:1], k) if case["one_source"] else order[:k]
        dst = order[1:k + 1] if case["one_source"] else order[k:2 * k]
        rows = np.random.default_rng(k).integers(case["rows_lo"], case["rows_hi"] + 1, size=k)
        s.copies = np.stack([src, dst, rows], axis=1).astype(np.int32)
        return s
    # attention and append: a batch over a paged cache
    new, ctx = _lengths(case)
    H, Hkv, bs = case["heads"], case["kv_heads"], case["block"]
    T = int(new.sum())
    need = -(-ctx // bs)
    s.n_blocks, s.max_blocks = int(need.sum()) + 1, int(need.max())
    table = np.zeros((len(new), s.max_blocks), dtype=np.int32)
    table[np.arange(s.max_blocks)[None] < need[:, None]] = rng.permutation(s.n_blocks)[:int(need.sum())]
    s.table, s.len = _ints(table), _ints(ctx)
    s.cu = _ints(np.concatenate([[0], np.cumsum(new)]))
    s.tokens, s.max_new, s.max_len = T, int(new.max()), int(ctx.max())
    s.pool = _rand(gen, (s.n_blocks, 2, Hkv, bs, d), t)
    if case["op"] == "append":
        s.qkv = _rand(gen, (T, (H + 2 * Hkv) * d), t)
        f, s.amplitude = _frequencies(case["rot"], case["ctx_hi"])
        s.inv_freq = torch.as_tensor(f, device=DEV)
        s.q_out = torch.empty((T, H * d), dtype=s.qkv.dtype, device=DEV)
    else:
        s.q = _rand(gen, (T, H * d), t, 1.5)
        s.scale = 1.0 / math.sqrt(d)
        s.out = torch.empty((T, H * d), dtype=s.q.dtype, device=DEV)
        s.workspace = None
    return s


# ---------------------------------------------------------------- plain forms

def _where(s):
    """Sequence and position of every new token."""
    new = (s.cu[1:] - s.cu[:-1]).long()
    seq = torch.repeat_interleave(torch.arange(len(new), device=DEV), new, output_size=s.tokens)
    return seq, (s.len.long() - new - s.cu[:-1].long())[seq] + torch.arange(s.tokens, device=DEV)


def _plain_turn(x, pos, inv_freq, amplitude, rot, interleaved):
    """x [tokens, heads, dim] in float; the angles in 64 bits."""
    angle = pos.double()[:, None] * inv_freq[None, :]
    c, s = (angle.cos() * amplitude).float()[:, None, :], (angle.sin() * amplitude).float()[:, None, :]
    t = x[..., :rot]
    if interleaved:
        a, b = t[..., 0::2], t[..., 1::2]
        y = torch.stack([a * c - b * s, b * c + a * s], dim=-1).flatten(-2)
    else:
        a, b = t[..., :rot // 2], t[..., rot // 2:]
        y = torch.cat([a * c - b * s, b * c + a * s], dim=-1)
    return torch.cat([y, x[..., rot:]], dim=-1)


def _plain_rotary(s):
    c = s.case
    x = s.x.float().view(c["tokens"], c["heads"], c["dim"])
    s.out.copy_(_plain_turn(x, s.pos, s.inv_freq, s.amplitude, c["rot"], c["interleaved"]).flatten(1))
    return s.out


def _plain_append(s):
    c = s.case
    H, Hkv, d, bs = c["heads"], c["kv_heads"], c["dim"], c["block"]
    seq, pos = _where(s)
    x = s.qkv.view(s.tokens, H + 2 * Hkv, d)
    qk = _plain_turn(x[:, :H + Hkv].float(), pos, s.inv_freq, s.amplitude, c["rot"], c["interleaved"]).to(x.dtype)
    s.q_out.copy_(qk[:, :H].flatten(1))
    blk = s.table[seq, pos // bs].long()
    row = pos % bs
    s.pool[blk, 0, :, row] = qk[:, H:]
    s.pool[blk, 1, :, row] = x[:, H + Hkv:]
    return s.q_out, s.pool


def _plain_attention(s):
    c = s.case
    H, Hkv, d, bs = c["heads"], c["kv_heads"], c["dim"], c["block"]
    G, B = H // Hkv, c["singles"] + c["chunks"]
    seq, pos = _where(s)
    at = torch.arange(s.tokens, device=DEV) - s.cu.long()[seq]                # place among the sequence's new tokens
    q = torch.zeros((B, s.max_new, H, d), device=DEV)
    q[seq, at] = s.q.float().view(s.tokens, H, d)
    q = q.view(B, s.max_new, Hkv, G, d).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * s.max_new, d)
    pages = s.pool[s.table.long()].float()                                    # [B, blocks, 2, Hkv, bs, d]
    kv = pages.permute(2, 0, 3, 1, 4, 5).reshape(2, B, Hkv, s.max_blocks * bs, d)[:, :, :, :s.max_len]
    scores = torch.matmul(q, kv[0].transpose(-1, -2).contiguous()).mul_(s.scale).view(B, Hkv, G, s.max_new, s.max_len)
    key = torch.arange(s.max_len, device=DEV)
    first = (s.len - (s.cu[1:] - s.cu[:-1])).long()
    qpos = first[:, None] + torch.arange(s.max_new, device=DEV)[None]
    hidden = key[None, None] > qpos[:, :, None]
    if c["window"]:
        hidden |= key[None, None] <= qpos[:, :, None] - c["window"]
    scores.masked_fill_(hidden[:, None, None], -math.inf)
    scores.sub_(scores.amax(-1, keepdim=True)).exp_()
    total = scores.sum(-1, keepdim=True)
    o = torch.matmul(scores.view(B, Hkv, G * s.max_new, s.max_len), kv[1].contiguous()).view(B, Hkv, G, s.max_new, d) / total
    s.out.copy_(o.permute(0, 3, 1, 2, 4)[seq, at].reshape(s.tokens, H * d))
    return s.out


def _plain_copy(s):
    src, dst, rows = torch.as_tensor(s.copies.astype(np.int64), device=DEV).unbind(1)
    moved = torch.arange(s.case["block"], device=DEV)[None] < rows[:, None]
    s.pool[:, dst] = torch.where(moved[None, :, None, None, :, None], s.pool[:, src], s.pool[:, dst])
    return s.pool


# ---------------------------------------------------------------- the framework's calls

def _own_rotary(s):
    import paper_2404_07947_amd as exe
    c = s.case
    exe.exe_op_rotary(CODE[c["dtype"]], c["tokens"], s.x, c["heads"] * c["dim"], c["heads"], c["dim"], c["rot"], c["interleaved"], s.pos,
                      s.inv_freq, s.amplitude, s.out, c["heads"] * c["dim"])
    return s.out


def _own_append(s):
    import paper_2404_07947_amd as exe
    c = s.case
    H, Hkv, d = c["heads"], c["kv_heads"], c["dim"]
    exe.exe_op_rotary_append_paged(CODE[c["dtype"]], c["singles"] + c["chunks"], s.cu, s.tokens, s.qkv, (H + 2 * Hkv) * d, H, Hkv, d, c["rot"],
                                   c["interleaved"], None, s.inv_freq, s.amplitude, s.pool, s.n_blocks, s.table, s.max_blocks, c["block"],
                                   s.len, s.q_out, H * d)
    return s.q_out, s.pool


def _own_attention(s):
    import paper_2404_07947_amd as exe
    c = s.case
    B, H, Hkv, d = c["singles"] + c["chunks"], c["heads"], c["kv_heads"], c["dim"]
    if s.workspace is None:
        need = exe.exe_op_chunk_attention_paged_workspace(CODE[c["dtype"]], B, s.tokens, s.max_new, s.max_len, H, Hkv, d, c["window"])
        s.workspace = torch.empty(max(need, 16), dtype=torch.uint8, device=DEV)
    exe.exe_op_chunk_attention_paged(CODE[c["dtype"]], B, s.cu, s.tokens, s.max_new, s.q, H * d, s.pool, s.n_blocks, s.table, s.max_blocks,
                                     c["block"], s.len, s.max_len, H, Hkv, d, s.scale, c["window"], s.out, H * d, s.workspace)
    return s.out


def _own_copy(s):
    import paper_2404_07947_amd as exe
    c = s.case
    exe.exe_op_kv_copy_blocks(CODE[c["dtype"]], s.pool, c["layers"], c["blocks"], c["block"], c["kv_heads"], c["dim"], s.copies)
    return s.pool


def run(state):
    op = state.case["op"]
    if own:
        return {"rotary": _own_rotary, "append": _own_append, "attention": _own_attention, "copy": _own_copy}[op](state)
    return {"rotary": _plain_rotary, "append": _plain_append, "attention": _plain_attention, "copy": _plain_copy}[op](state)


def _pairs(case):
    """(query token, key) pairs that the masks leave, and the cached positions that any token of a sequence sees."""
    new, ctx = _lengths(case)
    window = case["window"] or 1 << 40
    pairs = sum(int(np.minimum(np.arange(c - n, c) + 1, window).sum()) for n, c in zip(new, ctx))
    seen = sum(int(min(c, window + n - 1)) for n, c in zip(new, ctx))
    return pairs, seen


def work(case):
    """Attention: queries and the positions that a mask leaves read once, outputs written once; a multiply-add per feature for
    every (query, key) pair and again for its value.  Rotary and append: every element read once and written once (the pass-through
    part of a head too).  Copies: the copied rows read (a source of several copies once) and written."""
    e = 4 if case["dtype"] == "f32" else 2
    d = case["dim"]
    if case["op"] == "rotary":
        n = case["tokens"] * case["heads"] * d
        return {"bytes": 2.0 * n * e, "flops": 3.0 * case["tokens"] * case["heads"] * case["rot"]}
    if case["op"] == "copy":
        rows = np.random.default_rng(case["copies"]).integers(case["rows_lo"], case["rows_hi"] + 1, size=case["copies"])
        read = int(rows.max()) if case["one_source"] else int(rows.sum())
        return {"bytes": float(read + int(rows.sum())) * case["layers"] * 2 * case["kv_heads"] * d * e, "flops": 0.0}
    T = int(_lengths(case)[0].sum())
    if case["op"] == "append":
        return {"bytes": 2.0 * T * (case["heads"] + 2 * case["kv_heads"]) * d * e,
                "flops": 3.0 * T * (case["heads"] + case["kv_heads"]) * case["rot"]}
    pairs, seen = _pairs(case)
    return {"bytes": (2.0 * T * case["heads"] + 2.0 * seen * case["kv_heads"]) * d * e, "flops": 4.0 * pairs * case["heads"] * d}


# ---------------------------------------------------------------- the definitions, in 64 bits

def _exact_turn(x, pos, inv_freq, amplitude, rot, interleaved):
    """Pairs as complex numbers times amplitude * exp(i * pos * frequency)."""
    if rot == 0:
        return x
    w = torch.polar(torch.full((len(pos), rot // 2), float(amplitude), dtype=torch.float64, device=DEV), pos.double()[:, None] * inv_freq)
    lanes = torch.arange(rot, device=DEV).view(rot // 2, 2) if interleaved else torch.arange(rot, device=DEV).view(2, rot // 2).t()
    z = torch.complex(x[..., lanes[:, 0]], x[..., lanes[:, 1]]) * w[:, None]
    y = x.clone()
    y[..., lanes[:, 0]], y[..., lanes[:, 1]] = z.real, z.imag
    return y


def exact(case, seed):
    s = prepare(case, seed)
    d = case["dim"]
    if case["op"] == "rotary":
        x = s.x.double().view(case["tokens"], case["heads"], d)
        return _exact_turn(x, s.pos, s.inv_freq, s.amplitude, case["rot"], case["interleaved"]).flatten(1)
    if case["op"] == "copy":
        p = s.pool.double()
        for a, b, n in s.copies.tolist():
            p[:, b, :, :, :n] = s.pool[:, a, :, :, :n].double()
        return p
    new, ctx = _lengths(case)
    cu = np.concatenate([[0], np.cumsum(new)])
    H, Hkv, bs = case["heads"], case["kv_heads"], case["block"]
    table = s.table.cpu().numpy()
    if case["op"] == "append":
        x = s.qkv.double().view(-1, H + 2 * Hkv, d)
        q, pool = torch.empty((s.tokens, H, d), dtype=torch.float64, device=DEV), s.pool.double()
        for b in range(len(new)):
            pos = torch.arange(int(ctx[b] - new[b]), int(ctx[b]), device=DEV)
            y = _exact_turn(x[cu[b]:cu[b + 1], :H + Hkv], pos, s.inv_freq, s.amplitude, case["rot"], case["interleaved"])
            q[cu[b]:cu[b + 1]] = y[:, :H]
            page = torch.as_tensor(table[b].astype(np.int64), device=DEV)[pos // bs]
            pool[page, 0, :, pos % bs] = y[:, H:]
            pool[page, 1, :, pos % bs] = x[cu[b]:cu[b + 1], H + Hkv:]
        return q.flatten(1), pool
    out = torch.empty((s.tokens, H, d), dtype=torch.float64, device=DEV)
    for b in range(len(new)):
        L, n = int(ctx[b]), int(new[b])
        kv = s.pool[torch.as_tensor(table[b, :-(-L // bs)].astype(np.int64), device=DEV)]     # [blocks, 2, Hkv, bs, d]
        qpos = torch.arange(L - n, L, device=DEV)[:, None]
        key = torch.arange(L, device=DEV)[None]
        seen = (key <= qpos) & (key > qpos - (case["window"] or L + 1))
        for h in range(H):
            k, v = (kv[:, i, h // (H // Hkv)].reshape(-1, d)[:L].double() for i in (0, 1))
            x = s.q[cu[b]:cu[b + 1], h * d:(h + 1) * d].double()
            p = torch.softmax((x @ k.t().contiguous() * s.scale).masked_fill(~seen, -math.inf), dim=-1)
            out[cu[b]:cu[b + 1], h] = p @ v
    return out.flatten(1)
