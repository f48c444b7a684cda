"""What serving several continuations of one prompt over a paged key/value cache is measured by: norms of the heads of queries and
keys with their rotary positions (alone, and with the append of a chunk's keys and values), the attention of a batch whose
sequences share prefixes in groups, and log probabilities with entropy and top alternatives of rows of logits.

A page ("block") of one layer holds [K|V][key/value head][position in the block][feature]; a sequence lists its blocks in a
row of the block table.  The new tokens of a batch lie packed, sequence after sequence (cu_seqlens); len counts a
sequence's positions with the new ones, so the last of its new tokens has position len - 1.  Group g of a batch with shared prefixes
holds the sequences cu_groups[g] .. cu_groups[g + 1] - 1, whose first prefix[g] positions are the same; full blocks of them are in
all their tables, and a block that the prefix ends in was copied, as a fork of a sequence leaves it.

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
EPS = 1e-6


def _norm(dtype, tokens, heads, dim, rms, per_head, rot, interleaved, far):
    return {"op": "norm", "dtype": dtype, "tokens": tokens, "heads": heads, "dim": dim, "rms": rms, "per_head": per_head, "rot": rot,
            "interleaved": interleaved, "far": far}


def _append(dtype, heads, kv_heads, dim, rms, per_head, rot, interleaved, block, singles, chunks, new_lo, new_hi, ctx_lo, ctx_hi):
    """`singles` sequences bring one new token, `chunks` bring new_lo to new_hi; ctx: positions with the new ones."""
    return {"op": "append", "dtype": dtype, "heads": heads, "kv_heads": kv_heads, "dim": dim, "rms": rms, "per_head": per_head, "rot": rot,
            "interleaved": interleaved, "block": block, "singles": singles, "chunks": chunks, "new_lo": new_lo, "new_hi": new_hi,
            "ctx_lo": ctx_lo, "ctx_hi": ctx_hi}


def _prefix(dtype, heads, kv_heads, dim, block, groups, seqs_lo, seqs_hi, new_lo, new_hi, prefix_lo, prefix_hi, own_lo, own_hi):
    """groups of seqs_lo to seqs_hi sequences; own: positions of a sequence behind its prefix, with its new ones."""
    return {"op": "prefix", "dtype": dtype, "heads": heads, "kv_heads": kv_heads, "dim": dim, "block": block, "groups": groups, "seqs_lo": seqs_lo,
            "seqs_hi": seqs_hi, "new_lo": new_lo, "new_hi": new_hi, "prefix_lo": prefix_lo, "prefix_hi": prefix_hi, "own_lo": own_lo,
            "own_hi": own_hi}


def _logprobs(dtype, rows, vocab, stride, tokens, top, masked):
    """`tokens` given ones a row; masked: half of the vocabulary is ruled out (minus infinity)."""
    return {"op": "logprobs", "dtype": dtype, "rows": rows, "vocab": vocab, "stride": stride, "tokens": tokens, "top": top, "masked": masked}


def listed():
    named = {
        # Queries and keys of one token, far into a context: the smallest call, where latency counts.
        "norm_one_token": _norm("bf16", 1, 40, 128, 1, 1, 128, 0, 100000),
        # Queries and keys of a long prompt in float, norms with a mean, half of every head turned, neighbours paired.
        "norm_prompt_f32": _norm("f32", 4099, 20, 64, 0, 1, 32, 1, 4200),
        # A decode batch appends a token each, grouped heads, small pages.
        "append_decode_64": _append("bf16", 32, 8, 128, 1, 0, 128, 0, 16, 64, 0, 1, 1, 500, 8100),
        # Chunks of prompts at the OPT-13B widths.
        "append_chunks_opt13b": _append("bf16", 40, 40, 128, 1, 0, 128, 1, 64, 0, 8, 300, 700, 700, 1280),
        # Two candidates of a short prompt: the smallest call.
        "prefix_pair_small": _prefix("bf16", 12, 12, 64, 16, 1, 2, 2, 1, 1, 200, 200, 20, 60),
        # Eight candidates of one prompt (best of n) at the OPT-13B heads.
        "prefix_8_opt13b": _prefix("bf16", 40, 40, 128, 64, 1, 8, 8, 1, 1, 1500, 1500, 40, 300),
        # A serving batch: a dozen prompts with one to sixteen candidates each, grouped heads.
        "prefix_groups_ragged": _prefix("bf16", 32, 8, 128, 16, 12, 1, 16, 1, 1, 400, 3000, 20, 500),
        # Many questions on one long document, some with a drafted token: streams the document, computes most of all.
        "prefix_long_document": _prefix("bf16", 32, 8, 128, 64, 1, 64, 64, 1, 2, 30001, 30001, 20, 600),
        # The float path, in which a model is checked before it is served in bf16.
        "prefix_groups_f32": _prefix("f32", 12, 4, 64, 8, 3, 2, 9, 1, 3, 150, 900, 5, 200),
        # The next token of one request, with five alternatives.
        "logprobs_one_row": _logprobs("f32", 1, 50272, 50272, 1, 5, 0),
        # A decode batch at the OPT vocabulary, twenty alternatives.
        "logprobs_decode_256": _logprobs("f32", 256, 50272, 50272, 1, 20, 0),
        # Scoring prompts: every position's next token, rows padded, bf16 logits.
        "logprobs_prompts_bf16": _logprobs("bf16", 2048, 50272, 50304, 1, 1, 0),
    }
    return [dict(c, name=n) for n, c in named.items()]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw_heads(rng, most):
    kv = rng.choice([1, 2, 3, 4, 5, 8, 8, 16])
    return kv * rng.choice([g for g in (1, 1, 2, 3, 4, 6, 8) if kv * g <= most]), kv


def draw(rng):
    """One more case of the same ranges, sizes over their logarithm, none of more work than the largest listed one."""
    kind = rng.choice(["norm", "append", "append", "candidates", "candidates", "serving", "serving", "document", "f32", "logprobs", "logprobs", "logprobs"])
    block = rng.choice([8, 16, 32, 64, 128])
    dim = rng.choice([64, 128, 128])
    rot = rng.choice([dim, dim, dim // 2, 2 * rng.randint(0, dim // 2)])
    if kind == "norm":
        return _norm(rng.choice(["f32", "bf16"]), _log_int(rng, 1, 6000), rng.randint(1, 48), dim, rng.randint(0, 1), rng.randint(0, 1), rot,
                     rng.randint(0, 1), _log_int(rng, 100, 1000000))
    if kind == "append":
        h, kv = _draw_heads(rng, 40)
        m = _log_int(rng, 1, 700)
        return _append(rng.choice(["f32", "bf16", "bf16"]), h, kv, dim, rng.randint(0, 1), rng.randint(0, 1), rot, rng.randint(0, 1), block,
                       _log_int(rng, 1, 64), rng.randint(0, 5), max(1, m // 3), m, m, m + _log_int(rng, 1, 3500))
    if kind == "candidates":
        h, kv = _draw_heads(rng, 40)
        n, p, m = _log_int(rng, 1, 40), _log_int(rng, 10, 6000), rng.choice([1, 1, 1, 4])
        return _prefix("bf16", h, kv, dim, block, 1, n, n, 1, m, p, p, m, m + _log_int(rng, 1, 600))
    if kind == "serving":
        h, kv = _draw_heads(rng, 32)
        n, p = _log_int(rng, 1, 20), _log_int(rng, 30, 3000)
        return _prefix("bf16", h, kv, dim, block, _log_int(rng, 1, 16), rng.randint(1, n), n, 1, rng.choice([1, 1, 3]), rng.randint(0, p), p, 3,
                       3 + _log_int(rng, 1, 600))
    if kind == "document":
        h, kv = _draw_heads(rng, 32)
        n, p = _log_int(rng, 4, 64), _log_int(rng, 2000, min(30000, 200000 // kv))
        return _prefix("bf16", h, kv, dim, block, 1, n, n, 1, rng.choice([1, 2]), p, p, 2, 2 + _log_int(rng, 1, 600))
    if kind == "f32":
        h, kv = _draw_heads(rng, 16)
        p, m = _log_int(rng, 1, 900), rng.choice([1, 2, 5])
        return _prefix("f32", h, kv, dim, block, rng.randint(1, 4), 1, rng.randint(1, 9), 1, m, rng.randint(0, p), p, m, m + _log_int(rng, 1, 200))
    vocab = _log_int(rng, 300, 200000)
    rows = _log_int(rng, 1, max(2, min(2000, 45000000 // vocab)))
    return _logprobs(rng.choice(["f32", "f32", "bf16"]), rows, vocab, vocab + rng.choice([0, 0, 1, 40]), rng.choice([1, 1, 5]),
                     rng.choice([1, 5, 20, 64]), rng.choice([0, 0, 1]))


class _State:
    pass


def _lengths(case):
    """(new tokens, positions with them) of every sequence of an append, from the case alone; single tokens and chunks shuffled."""
    rng = np.random.default_rng([case[k] for k in ("singles", "chunks", "new_hi", "ctx_lo", "ctx_hi", "block")])
    new = np.concatenate([np.ones(case["singles"], dtype=np.int64),
                          rng.integers(case["new_lo"], case["new_hi"] + 1, size=case["chunks"])])
    rng.shuffle(new)
    ctx = rng.integers(case["ctx_lo"], case["ctx_hi"] + 1, size=len(new))
    return new, np.maximum(new, ctx)


def _groups(case):
    """Of a batch with shared prefixes, from the case alone: sequences and prefix of every group, new tokens and own positions of every
    sequence."""
    rng = np.random.default_rng([case[k] for k in ("groups", "seqs_hi", "new_hi", "prefix_hi", "own_hi", "block")])
    size = rng.integers(case["seqs_lo"], case["seqs_hi"] + 1, size=case["groups"])
    prefix = rng.integers(case["prefix_lo"], case["prefix_hi"] + 1, size=case["groups"])
    new = rng.integers(case["new_lo"], case["new_hi"] + 1, size=int(size.sum()))
    return size, prefix, new, np.maximum(new, rng.integers(case["own_lo"], case["own_hi"] + 1, size=len(new)))


def _frequencies(rot):
    return 10000.0 ** (-np.arange(0, rot, 2, dtype=np.float64) / max(rot, 1))


def _rand(gen, shape, dtype, scale=1.0):
    t = torch.randn(shape, generator=gen, device=DEV, dtype=TORCH_TYPE[dtype])
    return t.mul_(scale) if scale != 1.0 else t


def _ints(a):
    return torch.as_tensor(np.ascontiguousarray(a), dtype=torch.int32, device=DEV)


def _gain(gen, case, heads):
    """[dim] for all heads, or [heads, dim]"""
    return _rand(gen, (heads if case["per_head"] else 1, case["dim"]), case["dtype"], 0.3).add_(1.0)


def prepare(case, seed):
    s = _State()
    s.case = case
    gen = torch.Generator(device=DEV).manual_seed(int(seed))
    rng = np.random.default_rng(seed)
    t = case["dtype"]
    if case["op"] == "logprobs":
        n, v = case["rows"], case["vocab"]
        s.logits = _rand(gen, (n, case["stride"]), t, 2.5)
        if case["masked"]:
            s.logits[:, :v].masked_fill_(torch.rand((1, v), generator=gen, device=DEV) < 0.5, -math.inf)
            s.logits[:, v // 2] = 1.0                                   # something is left
        s.scale = 1.0 if case["top"] != 5 else 1.25
        s.tokens = _ints(rng.integers(0, v, size=(n, case["tokens"])))
        s.logp = torch.empty((n, case["tokens"]), device=DEV)
        s.entropy = torch.empty(n, device=DEV)
        s.top_ids = torch.empty((n, case["top"]), dtype=torch.int32, device=DEV)
        s.top_logp = torch.empty((n, case["top"]), device=DEV)
        s.workspace = None
        return s
    d = case["dim"]
    if case["op"] == "norm":
        n, h = case["tokens"], case["heads"]
        s.x = _rand(gen, (n, h * d), t, 3.0)
        s.gain = _gain(gen, case, h)
        s.pos = _ints(rng.integers(0, case["far"], size=n))
        s.inv_freq = torch.as_tensor(_frequencies(case["rot"]), device=DEV)
        s.out = torch.empty_like(s.x)
        return s
    H, Hkv, bs = case["heads"], case["kv_heads"], case["block"]
    if case["op"] == "append":
        new, ctx = _lengths(case)
        need = -(-ctx // bs)
        s.n_blocks, s.max_blocks = int(need.sum()) + 1, int(need.max())
        table = np.zeros((len(new), s.max_blocks), dtype=np.int32)
        table[np.arange(s.max_blocks)[None] < need[:, None]] = rng.permutation(s.n_blocks)[:int(need.sum())]
    else:
        size, prefix, new, own_len = _groups(case)
        group = np.repeat(np.arange(len(size)), size)
        ctx = prefix[group] + own_len
        # blocks: the group's full ones first, then a sequence's own
        full, need = prefix // bs, -(-ctx // bs)
        s.n_blocks, s.max_blocks = int(full.sum() + (need - full[group]).sum()) + 1, int(need.max())
        order, at = rng.permutation(s.n_blocks), 0
        table = np.zeros((len(new), s.max_blocks), dtype=np.int32)
        first = np.concatenate([[0], np.cumsum(size)])
        for g in range(len(size)):
            table[first[g]:first[g + 1], :full[g]] = order[at:at + full[g]]
            at += int(full[g])
        for b in range(len(new)):
            k = int(need[b] - full[group[b]])
            table[b, full[group[b]]:need[b]] = order[at:at + k]
            at += k
    T = int(new.sum())
    s.table, s.len = _ints(table), _ints(ctx)
    s.cu = _ints(np.concatenate([[0], np.cumsum(new)]))
    s.n_seqs, s.tokens, s.max_new = len(new), T, int(new.max())
    s.pool = _rand(gen, (s.n_blocks, 2, Hkv, bs, d), t)
    if case["op"] == "append":
        s.qkv = _rand(gen, (T, (H + 2 * Hkv) * d), t, 3.0)
        s.q_gain, s.k_gain = _gain(gen, case, H), _gain(gen, case, Hkv)
        s.inv_freq = torch.as_tensor(_frequencies(case["rot"]), device=DEV)
        s.q_out = torch.empty((T, H * d), dtype=s.qkv.dtype, device=DEV)
        return s
    # the blocks that prefixes end in
    for g in range(len(size)):
        if prefix[g] % bs and size[g] > 1:
            page = torch.as_tensor(table[first[g]:first[g + 1], full[g]].astype(np.int64), device=DEV)
            s.pool[page[1:], :, :, :int(prefix[g] % bs)] = s.pool[page[:1], :, :, :int(prefix[g] % bs)]
    s.q = _rand(gen, (T, H * d), t, 1.5)
    s.scale = 1.0 / math.sqrt(d)
    s.out = torch.empty((T, H * d), dtype=s.q.dtype, device=DEV)
    s.cu_groups, s.prefix = _ints(first), _ints(prefix)
    # what a serving program knows on the host
    s.n_groups, s.sizes, s.prefixes, s.news, s.owns = len(size), size.tolist(), prefix.tolist(), new.tolist(), own_len.tolist()
    s.max_group = int(np.add.reduceat(new, first[:-1]).max())
    s.max_prefix, s.max_own = int(prefix.max()), int(own_len.max())
    s.workspace = None
    return s


# ---------------------------------------------------------------- plain forms

def _plain_norm_turn(x, gain, pos, inv_freq, rms, rot, interleaved):
    """x [tokens, heads, dim] in float; the angles in 64 bits."""
    if not rms:
        x = x - x.mean(-1, keepdim=True)
    x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * gain.float()
    angle = pos.double()[:, None] * inv_freq[None, :]
    c, s = angle.cos().float()[:, None, :], angle.sin().float()[:, None, :]
    t = x[..., :rot]
    if interleaved:
        a, b = t[..., 0::2], t[..., 1::2]
        y = torch.stack([a * c - b * s, b * c + a * s], dim=-1).flatten(-2)
    else:
        a, b = t[..., :rot // 2], t[..., rot // 2:]
        y = torch.cat([a * c - b * s, b * c + a * s], dim=-1)
    return torch.cat([y, x[..., rot:]], dim=-1)


def _plain_norm(s):
    c = s.case
    x = s.x.float().view(c["tokens"], c["heads"], c["dim"])
    s.out.copy_(_plain_norm_turn(x, s.gain, s.pos, s.inv_freq, c["rms"], c["rot"], c["interleaved"]).flatten(1))
    return s.out


def _plain_append(s):
    c = s.case
    H, Hkv, d, bs = c["heads"], c["kv_heads"], c["dim"], c["block"]
    new = (s.cu[1:] - s.cu[:-1]).long()
    seq = torch.repeat_interleave(torch.arange(len(new), device=DEV), new, output_size=s.tokens)
    pos = (s.len.long() - new - s.cu[:-1].long())[seq] + torch.arange(s.tokens, device=DEV)
    x = s.qkv.view(s.tokens, H + 2 * Hkv, d)
    gain = torch.cat([s.q_gain.expand(H, d), s.k_gain.expand(Hkv, d)])
    qk = _plain_norm_turn(x[:, :H + Hkv].float(), gain, pos, s.inv_freq, c["rms"], c["rot"], c["interleaved"]).to(x.dtype)
    s.q_out.copy_(qk[:, :H].flatten(1))
    blk = s.table[seq, pos // bs].long()
    row = pos % bs
    s.pool[blk, 0, :, row] = qk[:, H:]
    s.pool[blk, 1, :, row] = x[:, H + Hkv:]
    return s.q_out, s.pool


def _plain_prefix(s):
    """Group by group: the scores of all its rows with the prefix, of every sequence's with its own positions, one softmax over both."""
    c = s.case
    H, Hkv, d, bs = c["heads"], c["kv_heads"], c["dim"], c["block"]
    G, b0, t0 = H // Hkv, 0, 0
    for size, P in zip(s.sizes, s.prefixes):
        new = s.news[b0:b0 + size]
        n = sum(new)
        q = s.q[t0:t0 + n].float().view(n, Hkv, G, d).permute(1, 0, 2, 3).reshape(Hkv, n * G, d) * s.scale
        pages = s.pool[s.table[b0, :-(-P // bs)].long()].float()                   # [blocks, 2, Hkv, bs, d]
        kv = pages.permute(1, 2, 0, 3, 4).reshape(2, Hkv, -1, d)[:, :, :P]
        shared = torch.matmul(q, kv[0].transpose(-1, -2).contiguous())             # [Hkv, n * G, P]
        outs, r0 = [], 0
        for b, m in zip(range(b0, b0 + size), new):
            L = P + s.owns[b]
            pages = s.pool[s.table[b, P // bs:-(-L // bs)].long()].float()
            mine = pages.permute(1, 2, 0, 3, 4).reshape(2, Hkv, -1, d)[:, :, P % bs:L - P // bs * bs]
            rows = slice(r0 * G, (r0 + m) * G)
            last = torch.matmul(q[:, rows], mine[0].transpose(-1, -2).contiguous()).view(Hkv, m, G, L - P)
            key = torch.arange(P, L, device=DEV)
            last.masked_fill_((key[None] > torch.arange(L - m, L, device=DEV)[:, None])[None, :, None], -math.inf)
            x = torch.cat([shared[:, rows], last.view(Hkv, m * G, L - P)], -1)
            x.sub_(x.amax(-1, keepdim=True)).exp_()
            total = x.sum(-1, keepdim=True)
            o = (torch.matmul(x[..., :P], kv[1]) + torch.matmul(x[..., P:], mine[1])) / total
            outs.append(o.view(Hkv, m, G, d).transpose(0, 1).reshape(m, H * d))
            r0 += m
        s.out[t0:t0 + n] = torch.cat(outs).to(s.out.dtype)
        b0, t0 = b0 + size, t0 + n
    return s.out


def _plain_logprobs(s):
    c = s.case
    x = s.logits[:, :c["vocab"]].float()
    y = (x - x.amax(-1, keepdim=True)) * s.scale
    e = y.exp()
    total = e.sum(-1, keepdim=True)
    entropy = total.log()[:, 0] - torch.where(e > 0, e * y, 0.0).sum(-1) / total[:, 0]
    y -= total.log()
    ids = torch.sort(x, dim=-1, descending=True, stable=True)[1][:, :c["top"]]
    return y.gather(1, s.tokens.long()), entropy, ids.int(), y.gather(1, ids)


# ---------------------------------------------------------------- the framework's calls

def _own_norm(s):
    import paper_2404_07947_amd as exe
    c = s.case
    w = c["heads"] * c["dim"]
    exe.exe_op_head_norm_rotary(CODE[c["dtype"]], c["tokens"], s.x, w, c["heads"], c["dim"], c["rms"], s.gain, c["per_head"], EPS, c["rot"],
                                c["interleaved"], s.pos, s.inv_freq, 1.0, s.out, w)
    return s.out


def _own_append(s):
    import paper_2404_07947_amd as exe
    c = s.case
    H, Hkv, d = c["heads"], c["kv_heads"], c["dim"]
    exe.exe_op_head_norm_rotary_append_paged(CODE[c["dtype"]], s.n_seqs, s.cu, s.tokens, s.qkv, (H + 2 * Hkv) * d, H, Hkv, d, c["rms"], s.q_gain,
                                             s.k_gain, c["per_head"], EPS, c["rot"], c["interleaved"], None, s.inv_freq, 1.0, s.pool, s.n_blocks,
                                             s.table, s.max_blocks, c["block"], s.len, s.q_out, H * d)
    return s.q_out, s.pool


def _own_prefix(s):
    import paper_2404_07947_amd as exe
    c = s.case
    H, Hkv, d = c["heads"], c["kv_heads"], c["dim"]
    if s.workspace is None:
        need = exe.exe_op_prefix_attention_paged_workspace(CODE[c["dtype"]], s.n_seqs, s.tokens, s.max_new, s.n_groups, s.max_group, s.max_prefix,
                                                           s.max_own, H, Hkv, d)
        s.workspace = torch.empty(max(need, 16), dtype=torch.uint8, device=DEV)
    exe.exe_op_prefix_attention_paged(CODE[c["dtype"]], s.n_seqs, s.cu, s.tokens, s.max_new, s.n_groups, s.cu_groups, s.prefix, s.max_group,
                                      s.max_prefix, s.q, H * d, s.pool, s.n_blocks, s.table, s.max_blocks, c["block"], s.len, s.max_own, H, Hkv, d,
                                      s.scale, s.out, H * d, s.workspace)
    return s.out


def _own_logprobs(s):
    import paper_2404_07947_amd as exe
    c = s.case
    if s.workspace is None:
        need = exe.exe_op_logprobs_workspace(CODE[c["dtype"]], c["rows"], c["vocab"], c["top"])
        s.workspace = torch.empty(max(need, 16), dtype=torch.uint8, device=DEV)
    exe.exe_op_logprobs(CODE[c["dtype"]], s.logits, c["stride"], c["rows"], c["vocab"], s.scale, s.tokens, c["tokens"], s.logp, s.entropy, c["top"],
                        s.top_ids, s.top_logp, s.workspace)
    return s.logp, s.entropy, s.top_ids, s.top_logp


def run(state):
    op = state.case["op"]
    if own:
        return {"norm": _own_norm, "append": _own_append, "prefix": _own_prefix, "logprobs": _own_logprobs}[op](state)
    return {"norm": _plain_norm, "append": _plain_append, "prefix": _plain_prefix, "logprobs": _plain_logprobs}[op](state)


def work(case):
    """Norms and appends: every element read once and written once.  Attention: queries, prefixes (once a group) and own positions read
    once, outputs written once; a multiply-add per feature for every (query, key) pair and again for its value.  Log probabilities:
    logits read once; a subtraction, a product, an exponential and two sums an element."""
    e = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "logprobs":
        n = case["rows"] * case["vocab"]
        return {"bytes": float(n) * e + case["rows"] * (8.0 * case["tokens"] + 4.0 + 8.0 * case["top"]), "flops": 5.0 * n}
    d = case["dim"]
    if case["op"] == "norm":
        n = case["tokens"] * case["heads"]
        return {"bytes": 2.0 * n * d * e, "flops": n * (4.0 * d + 3.0 * case["rot"])}
    H, Hkv = case["heads"], case["kv_heads"]
    if case["op"] == "append":
        T = int(_lengths(case)[0].sum())
        return {"bytes": 2.0 * T * (H + 2 * Hkv) * d * e, "flops": T * (H + Hkv) * (4.0 * d + 3.0 * case["rot"])}
    size, prefix, new, own_len = _groups(case)
    group = np.repeat(np.arange(len(size)), size)
    pairs = int((new * (prefix[group] + own_len) - new * (new - 1) // 2).sum())
    seen = int(prefix.sum() + own_len.sum())
    return {"bytes": (2.0 * int(new.sum()) * H + 2.0 * seen * Hkv) * d * e, "flops": 4.0 * pairs * H * d}


# ---------------------------------------------------------------- the definitions, in 64 bits

def _exact_norm_turn(x, gain, pos, inv_freq, rms, rot, interleaved):
    """Norms as vectors of length sqrt(dim); pairs as complex numbers times exp(i * pos * frequency)."""
    d = x.shape[-1]
    if not rms:
        x = x - x.sum(-1, keepdim=True) / d
    x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / d + EPS) * gain.double()
    if rot == 0:
        return x
    w = torch.polar(torch.ones((len(pos), rot // 2), dtype=torch.float64, device=DEV), pos.double()[:, None] * inv_freq)
    lanes = torch.arange(rot, device=DEV).view(rot // 2, 2) if interleaved else torch.arange(rot, device=DEV).view(2, rot // 2).t()
    z = torch.complex(x[..., lanes[:, 0]], x[..., lanes[:, 1]]) * w[:, None]
    y = x.clone()
    y[..., lanes[:, 0]], y[..., lanes[:, 1]] = z.real, z.imag
    return y


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "logprobs":
        x = s.logits[:, :case["vocab"]].contiguous()
        y = torch.log_softmax(x.double() * s.scale, dim=-1)
        p = y.exp()
        entropy = -torch.where(p > 0, p * y, 0.0).sum(-1)
        # the order of (logit, lowest index) as one whole number; no logit is NaN, and -0 is 0
        bits = (x.float() + 0.0).view(torch.int32).long()
        place = torch.where(bits >= 0, bits, -(bits & 0x7FFFFFFF))
        key = place * (1 << 31) + ((1 << 31) - 1 - torch.arange(case["vocab"], device=DEV))
        ids = torch.topk(key, case["top"], dim=-1)[1] if case["top"] else torch.zeros((case["rows"], 0), dtype=torch.int64, device=DEV)
        return y.gather(1, s.tokens.long()), entropy, ids.int(), y.gather(1, ids)
    d = case["dim"]
    if case["op"] == "norm":
        x = s.x.double().view(case["tokens"], case["heads"], d)
        return _exact_norm_turn(x, s.gain, s.pos, s.inv_freq, case["rms"], case["rot"], case["interleaved"]).flatten(1)
    H, Hkv, bs = case["heads"], case["kv_heads"], case["block"]
    table, cu, ctx = s.table.cpu().numpy(), s.cu.cpu().numpy(), s.len.cpu().numpy()
    if case["op"] == "append":
        x = s.qkv.double().view(-1, H + 2 * Hkv, d)
        q, pool = torch.empty((s.tokens, H, d), dtype=torch.float64, device=DEV), s.pool.double()
        gain = torch.cat([s.q_gain.expand(H, d), s.k_gain.expand(Hkv, d)])
        for b in range(s.n_seqs):
            pos = torch.arange(int(ctx[b] - (cu[b + 1] - cu[b])), int(ctx[b]), device=DEV)
            y = _exact_norm_turn(x[cu[b]:cu[b + 1], :H + Hkv], gain, pos, s.inv_freq, case["rms"], case["rot"], case["interleaved"])
            q[cu[b]:cu[b + 1]] = y[:, :H]
            page = torch.as_tensor(table[b].astype(np.int64), device=DEV)[pos // bs]
            pool[page, 0, :, pos % bs] = y[:, H:]
            pool[page, 1, :, pos % bs] = x[cu[b]:cu[b + 1], H + Hkv:]
        return q.flatten(1), pool
    # every sequence by itself, over all of its positions
    out = torch.empty((s.tokens, H, d), dtype=torch.float64, device=DEV)
    G = H // Hkv
    for b in range(s.n_seqs):
        L, n = int(ctx[b]), int(cu[b + 1] - cu[b])
        kv = s.pool[torch.as_tensor(table[b, :-(-L // bs)].astype(np.int64), device=DEV)]
        hidden = torch.arange(L, device=DEV)[None] > torch.arange(L - n, L, device=DEV)[:, None]
        x = s.q[cu[b]:cu[b + 1]].double().view(n, H, d)
        for h in range(Hkv):
            k, v = (kv[:, i, h].reshape(-1, d)[:L].double() for i in (0, 1))
            a = x[:, h * G:(h + 1) * G].reshape(n * G, d) @ k.t().contiguous() * s.scale
            p = torch.softmax(a.view(n, G, L).masked_fill(hidden[:, None], -math.inf), dim=-1)
            out[cu[b]:cu[b + 1], h * G:(h + 1) * G] = (p.view(n * G, L) @ v).view(n, G, d)
    return out.flatten(1)
