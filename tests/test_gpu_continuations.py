"""Several continuations of one prompt through one layer, as a serving loop makes the calls: the prompt in chunks (norms of heads, positions,
append, attention of the chunk), forks that share its pages and copy the one it ends in, then steps in which every continuation brings a
token (append, attention over the shared prefix), is scored, and the best ones go on, some of them twice.  Against the same in 64 bits: a logit is a sum of 128
products of 2 x 0.1 x 1 in float, 128 half steps of the 17 that their magnitudes add up to, 1.3e-4 at most, and what the layer in front of it is off by is
smaller; an entropy adds up the log probabilities (up to 10) by their probabilities."""
import numpy as np
import pytest
import torch

import paper_2404_07947_amd as exe
from chunk_util import DEV

pytestmark = pytest.mark.gpu

H, HKV, DH, D, V, BLOCK, EPS = 4, 2, 64, 128, 1000, 16, 1e-6
WQ = (H + 2 * HKV) * DH


class Layer:
    """Embedding, one attention layer and LM head; float on the device, the same numbers in 64 bits on the host."""

    def __init__(self, seed):
        g = torch.Generator().manual_seed(seed)
        r = lambda *s: torch.randn(s, generator=g)
        self.emb, self.wqkv, self.wo, self.lm = r(V, D), r(WQ, D) * D ** -0.5, r(D, H * DH) * (H * DH) ** -0.5, r(V, D) * D ** -0.5 * 2
        self.gq, self.gk = 1 + 0.3 * r(DH), 1 + 0.3 * r(DH)
        self.freq = torch.as_tensor(exe.exe_rotary_frequencies(DH)[0])
        self.d = {k: getattr(self, k).to(DEV) for k in ("emb", "wqkv", "wo", "lm", "gq", "gk", "freq")}

    def host_qkv(self, tok, pos):
        x = self.emb[tok].double()
        y = (self.wqkv.double() @ x).view(-1, DH)
        n = y / torch.sqrt((y * y).mean(-1, keepdim=True) + float(np.float32(EPS)))
        n = torch.cat([n[:H] * self.gq.double(), n[H:H + HKV] * self.gk.double()])
        w = torch.polar(torch.ones(DH // 2, dtype=torch.float64), pos * self.freq)
        z = torch.complex(n[:, :DH // 2], n[:, DH // 2:]) * w
        return x, torch.cat([z.real, z.imag], -1), y[H + HKV:]

    def host_logits(self, toks):
        """Log probabilities behind the last token of a sequence."""
        rows = [self.host_qkv(t, p) for p, t in enumerate(toks)]
        k, v = torch.stack([r[1][H:] for r in rows], 1), torch.stack([r[2] for r in rows], 1)
        x, q = rows[-1][0], rows[-1][1][:H]
        a = torch.softmax((q[:, None] * k.repeat_interleave(H // HKV, 0)).sum(-1) * DH ** -0.5, -1)
        o = (a[..., None] * v.repeat_interleave(H // HKV, 0)).sum(1).flatten()
        return torch.log_softmax((self.lm.double() @ (x + self.wo.double() @ o)) * 0.8, -1)


def i32(a):
    return torch.as_tensor(np.ascontiguousarray(a), dtype=torch.int32).to(DEV)


class Server:
    def __init__(self, layer, seqs, blocks):
        self.l, self.n = layer, seqs
        self.pool = torch.full((blocks, 2, HKV, BLOCK, DH), float("nan"), device=DEV)
        self.table = np.full((seqs, 8), -1, dtype=np.int32)
        self.free = list(range(blocks))
        self.bufs = {}

    def product(self, w, x, out, mode=2):
        M, (N, K) = x.shape[0], w.shape
        need = exe.exe_op_gemm_workspace(0, M, N, K)
        ws = self.bufs.setdefault((M, N, K), torch.empty(max(need, 16), dtype=torch.uint8, device=DEV))
        exe.exe_op_gemm(0, M, N, K, x, w, None, -1, 1.0, mode, out, ws)

    def grow(self, b, upto):
        for i in range(-(-upto // BLOCK)):
            if self.table[b, i] < 0:
                self.table[b, i] = self.free.pop()

    def qkv_append(self, toks, cu, d_table, length, n):
        d = self.l.d
        x = d["emb"][toks.long()]
        qkv = torch.empty((len(toks), WQ), device=DEV)
        self.product(d["wqkv"], x, qkv)
        q = torch.empty((len(toks), H * DH), device=DEV)
        exe.exe_op_head_norm_rotary_append_paged(0, n, cu, len(toks), qkv, WQ, H, HKV, DH, 1, d["gq"], d["gk"], 0, EPS, DH, 0, None, d["freq"], 1.0, self.pool,
                                                 self.pool.shape[0], d_table, 8, BLOCK, length, q, H * DH)
        return x, q

    def step(self, toks, cu, d_table, length, groups, prefix, sizes, k):
        """One token for every sequence: (ids, log probabilities) of the k best next ones, and of the given ones."""
        n = len(toks)
        x, q = self.qkv_append(toks, cu, d_table, length, n)
        o = torch.empty_like(q)
        ng = len(prefix)
        need = exe.exe_op_prefix_attention_paged_workspace(0, n, n, 1, ng, sizes[0], sizes[1], sizes[2], H, HKV, DH)
        ws = self.bufs.setdefault(("prefix", need), torch.empty(max(need, 16), dtype=torch.uint8, device=DEV))
        exe.exe_op_prefix_attention_paged(0, n, cu, n, 1, ng, groups, prefix, sizes[0], sizes[1], q, H * DH, self.pool, self.pool.shape[0], d_table, 8, BLOCK, length, sizes[2],
                                          H, HKV, DH, DH ** -0.5, o, H * DH, ws)
        self.product(self.l.d["wo"], o, x, 1)                       # the residual
        logits = torch.empty((n, V), device=DEV)
        self.product(self.l.d["lm"], x, logits)
        ids, lp = torch.empty((n, k), dtype=torch.int32, device=DEV), torch.empty((n, k), device=DEV)
        given, entropy = torch.empty((n, 1), device=DEV), torch.empty(n, device=DEV)
        exe.exe_op_logprobs(0, logits, V, n, V, 0.8, toks.view(n, 1), 1, given, entropy, k, ids, lp)
        return ids, lp, given, entropy


@pytest.mark.parametrize("prompt", [1, 15, 16, 17, 53, 64])
@pytest.mark.parametrize("bound", [1, 600])
def test_beams(prompt, bound):
    """4 beams of 2 prompts each, 12 steps; the shared prefix is the prompt.  bound: of the own positions, one kernel or parts."""
    l = Layer(prompt)
    s = Server(l, 8, 80)
    g = torch.Generator().manual_seed(prompt)
    prompts = [torch.randint(0, V, (prompt,), generator=g).tolist() for _ in range(2)]
    # the prompts in chunks of 20, both together; all but the last token, which the first step brings
    done = 0
    while done < prompt - 1:
        m = min(20, prompt - 1 - done)
        for b in (0, 4):
            s.grow(b, done + m)
        toks = i32(sum((p[done:done + m] for p in prompts), []))
        tab = i32(s.table[[0, 4]])
        s.qkv_append(toks, i32([0, m, 2 * m]), tab, i32([done + m] * 2), 2)
        done += m
    shared = prompt - 1
    # forks: full pages in every table, the last one copied
    copies = []
    for b in (0, 4):
        for f in range(b + 1, b + 4):
            s.table[f, :shared // BLOCK] = s.table[b, :shared // BLOCK]
            if shared % BLOCK:
                s.table[f, shared // BLOCK] = s.free.pop()
                copies.append((int(s.table[b, shared // BLOCK]), int(s.table[f, shared // BLOCK]), shared % BLOCK))
    if copies:
        exe.exe_op_kv_copy_blocks(0, s.pool, 1, s.pool.shape[0], BLOCK, HKV, DH, copies)
    seqs = [list(prompts[b // 4][:-1]) for b in range(8)]
    nxt = [prompts[b // 4][-1] for b in range(8)]
    groups, prefix = i32([0, 4, 8]), i32([shared] * 2)
    cu = i32(range(9))
    for t in range(12):
        L = shared + t + 1
        for b in range(8):
            s.grow(b, L)
            seqs[b].append(nxt[b])
        ids, lp, given, entropy = s.step(i32(nxt), cu, i32(s.table), i32([L] * 8), groups, prefix, (4, max(shared, 1), max(12, bound)), 6)
        for b in range(8):
            want = l.host_logits(seqs[b])
            assert float((lp[b].cpu().double() - want[ids[b].long().cpu()]).abs().max()) <= 2e-4, (t, b)
            assert abs(float(given[b, 0]) - float(want[nxt[b]])) <= 2e-4
            assert abs(float(entropy[b]) + float((want.exp() * want).sum())) <= 2e-3
            # the best ones are the best but for those as good
            assert float(want.topk(6)[0].min()) <= float(want[ids[b].long().cpu()].min()) + 4e-4
        nxt = []
        for gr in (0, 4):
            # the first two beams go on twice each: their own pages are copied into the others'
            copies = []
            for to, frm in ((gr + 2, gr), (gr + 3, gr + 1)):
                for i in range(shared // BLOCK, -(-L // BLOCK)):
                    copies.append((int(s.table[frm, i]), int(s.table[to, i]), min(BLOCK, L - i * BLOCK)))
                seqs[to] = list(seqs[frm])
            exe.exe_op_kv_copy_blocks(0, s.pool, 1, s.pool.shape[0], BLOCK, HKV, DH, copies)
            row = ids.cpu()
            nxt += [int(row[gr, 0]), int(row[gr + 1, 0]), int(row[gr, 1]), int(row[gr + 1, 1])]


def test_one_graph_of_a_step():
    """The calls of a step captured once and replayed with other tokens, lengths, tables and groups, eager calls between the replays."""
    l = Layer(7)
    s = Server(l, 6, 60)
    s.pool.normal_(generator=torch.Generator(device=DEV).manual_seed(1))
    for b in range(6):
        s.grow(b, 128)
    for b in range(1, 4):
        s.table[b, :2] = s.table[0, :2]
    toks, length, tab = i32([1, 2, 3, 4, 5, 6]), i32([40] * 6), i32(s.table)
    cu, groups, prefix = i32(range(7)), i32([0, 4, 6]), i32([32, 0])
    sizes = (4, 32, 400)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        s.step(toks, cu, tab, length, groups, prefix, sizes, 5)
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        out = s.step(toks, cu, tab, length, groups, prefix, sizes, 5)
    for t in range(20):
        length.add_(1 + t % 3)
        toks.copy_((out[0][:, 0] + t) % V)
        prefix.copy_(i32([32 - t, 0]))
        groups.copy_(i32([0, 4 - t % 3, 6]))
        pool = s.pool.clone()
        graph.replay()
        torch.cuda.synchronize()
        got, after = [o.clone() for o in out], s.pool.clone()
        s.pool.copy_(pool)
        want = s.step(toks, cu, tab, length, groups, prefix, sizes, 5)
        assert torch.equal(after, s.pool) and all(torch.equal(a, b) for a, b in zip(got, want)), t
