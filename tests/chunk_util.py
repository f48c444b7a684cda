"""Batches of new tokens over a paged cache, and what the operations on them are, in 64 bits on the CPU."""
import numpy as np
import torch

import paper_2404_07947_amd as exe

DEV = "cuda:0"
TYPES = {"f32": (0, torch.float32), "bf16": (1, torch.bfloat16)}
U = 2.0 ** -24                                   # half a step of float
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}    # half a step of the storage type


BOUND = 1          # of the lengths, at least: sizes the launch, so a larger one brings small cases to the kernels of larger ones


class Batch:
    """Sequences of `seqs` = [(new tokens, positions with them)] over blocks in random order; what no sequence holds is NaN, the
    table's unused entries are far out of the pool."""

    def __init__(self, seqs, H, Hkv, dh, block, dtype, seed=0, extra_rows=0, table_pad=0):
        g = torch.Generator().manual_seed(seed)
        self.code, self.t = TYPES[dtype]
        self.dtype, self.seqs, self.H, self.Hkv, self.dh, self.block = dtype, seqs, H, Hkv, dh, block
        need = [-(-L // block) for _, L in seqs]
        self.max_blocks = max(need + [1]) + table_pad
        self.n_blocks = sum(need) + 3
        order = torch.randperm(self.n_blocks, generator=g).tolist()
        self.table = np.full((len(seqs), self.max_blocks), 1 << 30, dtype=np.int32)
        self.pool = torch.full((self.n_blocks, 2, Hkv, block, dh), float("nan"), dtype=self.t)
        self.k, self.v = [], []                  # per sequence [Hkv, L, dh]
        at = 0
        for b, (n, L) in enumerate(seqs):
            self.table[b, :need[b]] = order[at:at + need[b]]
            at += need[b]
            kv = torch.randn((2, Hkv, max(L, 0), dh), generator=g).to(self.t)
            self.k.append(kv[0])
            self.v.append(kv[1])
        self.T = sum(n for n, _ in seqs)
        self.rows = self.T + extra_rows
        self.cu = np.concatenate([[0], np.cumsum([n for n, _ in seqs])]).astype(np.int32)
        self.q = (torch.randn((self.rows, H * dh), generator=g) * 1.5).to(self.t)
        self.scale = dh ** -0.5

    def fill(self):
        """The cache's rows, as the appends of all positions would leave them."""
        for b, (_, L) in enumerate(self.seqs):
            for i in range(-(-L // self.block)):
                m = min(self.block, L - i * self.block)
                s = slice(i * self.block, i * self.block + m)
                self.pool[self.table[b, i], 0, :, :m] = self.k[b][:, s]
                self.pool[self.table[b, i], 1, :, :m] = self.v[b][:, s]
        return self

    def device(self):
        i32 = lambda a: torch.as_tensor(np.ascontiguousarray(a), dtype=torch.int32).to(DEV)
        self.d_pool, self.d_q = self.pool.to(DEV), self.q.to(DEV)
        self.d_table, self.d_cu, self.d_len = i32(self.table), i32(self.cu), i32([L for _, L in self.seqs])
        return self

    def attend(self, window=0, max_new=None, max_len=None, out=None, stream=None, workspace=None, scale=None):
        """The library's result (rows behind the last sequence hold 7)."""
        n = max([s[0] for s in self.seqs] + [1]) if max_new is None else max_new
        L = max([s[1] for s in self.seqs] + [BOUND]) if max_len is None else max_len
        w = self.H * self.dh
        if out is None:
            out = torch.full((self.rows, w), 7.0, dtype=self.t, device=DEV)
        if workspace is None:
            need = exe.exe_op_chunk_attention_paged_workspace(self.code, len(self.seqs), self.rows, n, L, self.H, self.Hkv, self.dh, window)
            workspace = torch.full((max(need, 16) // 4,), float("nan"), dtype=torch.float32, device=DEV)
        exe.exe_op_chunk_attention_paged(self.code, len(self.seqs), self.d_cu, self.rows, n, self.d_q, w, self.d_pool, self.n_blocks, self.d_table,
                                         self.max_blocks, self.block, self.d_len, L, self.H, self.Hkv, self.dh,
                                         self.scale if scale is None else scale, window, out, w, workspace, stream=stream)
        return out

    def want(self, window=0, scale=None):
        """(result, bound of the error) in 64 bits.  The bound: a score is dh products and sums in float (relative to the sum of their
        magnitudes), its exponent a few roundings of numbers as large as the scores; a probability of relative error e is off by e,
        and so is what it adds; the sums over the keys add half a step each; probabilities are rounded to the storage type (or to more
        bits), and the result is once more."""
        scale = self.scale if scale is None else scale
        out = torch.full((self.rows, self.H, self.dh), 7.0, dtype=torch.float64)
        tol = torch.zeros_like(out)
        G = self.H // self.Hkv
        q = self.q.double().view(self.rows, self.H, self.dh)
        for b, (n, L) in enumerate(self.seqs):
            for i in range(n):
                p, t = L - n + i, int(self.cu[b]) + i
                lo, hi = max(0, p - window + 1) if window else 0, p + 1
                if hi <= 0:
                    out[t] = 0.0
                    continue
                k = self.k[b][:, lo:hi].double().repeat_interleave(G, 0)
                v = self.v[b][:, lo:hi].double().repeat_interleave(G, 0)
                s = torch.einsum("hd,hkd->hk", q[t], k) * scale
                mag = torch.einsum("hd,hkd->hk", q[t].abs(), k.abs()) * abs(scale)
                pr = torch.softmax(s, -1)
                out[t] = torch.einsum("hk,hkd->hd", pr, v)
                e = 2 * (self.dh + 8) * U * mag.amax(-1) + 8 * U * (1 + s.abs().amax(-1)) + (hi - lo + 16) * 2 * U + HALF[self.dtype]
                tol[t] = e[:, None] * torch.einsum("hk,hkd->hd", pr, v.abs()) + HALF[self.dtype] * out[t].abs() + 1e-30
        return out.flatten(1), tol.flatten(1)


def check(got, want, tol, what=""):
    got = got.cpu().double()
    assert got.shape == want.shape
    assert not torch.isnan(got).any(), what
    over = (got - want).abs() - tol * (1 + 1e-6)
    assert bool((over <= 0).all()), (what, float(over.max()), int((over > 0).sum()))


def turned(x, pos, inv_freq, amplitude, rot, interleaved):
    """x [tokens, heads, dh] in 64 bits, and the bound: sine and cosine within 3 half steps of float, the products and their sum within 3
    more."""
    x = x.double()
    w = torch.polar(torch.full((len(pos), rot // 2), float(amplitude), dtype=torch.float64), pos.double()[:, None] * inv_freq[None])[:, None]
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:rot])
    z = torch.complex(a, b) * w
    y, e = x.clone(), torch.zeros_like(x)
    err = 6 * U * abs(amplitude) * (a.abs() + b.abs())
    if interleaved:
        y[..., 0:rot:2], y[..., 1:rot:2], e[..., 0:rot:2], e[..., 1:rot:2] = z.real, z.imag, err, err
    else:
        y[..., :rot // 2], y[..., rot // 2:rot], e[..., :rot // 2], e[..., rot // 2:rot] = z.real, z.imag, err, err
    return y, e
