"""Attention over prefixes that the sequences of a group share, against 64 bits.  What lies behind a sequence's end, and the blocks that only a
group's first sequence with new tokens is read through, are NaN or no blocks in all other tables."""
import numpy as np
import pytest
import torch

import chunk_util
import paper_2404_07947_amd as exe
from chunk_util import DEV, Batch, check

pytestmark = pytest.mark.gpu


BOUND = 1          # of own positions, at least: sizes the launch, so a larger one brings small cases to the kernels of larger ones


@pytest.fixture(autouse=True, params=[1, 1100], ids=["own", "parts"])
def bound(request, monkeypatch):
    """Calls of few and short sequences take one kernel: with a larger bound of the own positions, those of longer ones and the join."""
    monkeypatch.setitem(globals(), "BOUND", request.param)


class Groups(Batch):
    """groups = [(prefix, [(new tokens, own positions with them), ..]), ..]; `loose`: sequences behind the last group, (new, positions)."""

    def __init__(self, groups, H, Hkv, dh, block, dtype, loose=(), **kw):
        self.groups = groups
        self.prefix = [p for p, _ in groups]
        seqs = [(n, p + own) for p, s in groups for n, own in s] + list(loose)
        super().__init__(seqs, H, Hkv, dh, block, dtype, **kw)
        self.cu_groups = np.concatenate([[0], np.cumsum([len(s) for _, s in groups])]).astype(np.int32)
        for g, (p, _) in enumerate(groups):
            b0, b1 = self.cu_groups[g], self.cu_groups[g + 1]
            for b in range(b0 + 1, b1):
                self.k[b][:, :p], self.v[b][:, :p] = self.k[b0][:, :p], self.v[b0][:, :p]

    def fill(self):
        super().fill()
        for g, (p, _) in enumerate(self.groups):
            members = range(self.cu_groups[g], self.cu_groups[g + 1])
            front = next((b for b in members if self.seqs[b][0]), -1)
            for b in members:
                for i in range(p // self.block if b != front else 0):     # never looked at: no block, or one of NaN
                    self.pool[self.table[b, i]] = float("nan")
                    self.table[b, i] = self.n_blocks - 1 if i % 2 else -5
        return self

    def device(self):
        super().device()
        self.d_groups = torch.as_tensor(self.cu_groups).to(DEV)
        self.d_prefix = torch.tensor(self.prefix, dtype=torch.int32, device=DEV)
        for b, (n, _) in enumerate(self.seqs):                            # of a sequence without new tokens nothing is looked at
            if n == 0:
                self.d_len[b] = -9 if b % 2 else (1 << 31) - 1
        return self

    def sizes(self):
        new = [n for n, _ in self.seqs]
        return dict(max_new=max(new + [1]), max_group=max([sum(n for n, _ in s) for _, s in self.groups] + [1]), max_prefix=max(self.prefix + [0]),
                    max_own=max([o for _, s in self.groups for _, o in s] + [L for _, L in self.seqs[self.cu_groups[-1]:]] + [BOUND]))

    def attend(self, out=None, stream=None, workspace=None, scale=None, q=None, q_stride=None, out_stride=None, **change):
        z = {**self.sizes(), **change}
        w = self.H * self.dh
        if out is None:
            out = torch.full((self.rows, w), 7.0, dtype=self.t, device=DEV)
        if workspace is None:
            need = exe.exe_op_prefix_attention_paged_workspace(self.code, len(self.seqs), self.rows, z["max_new"], len(self.groups), z["max_group"], z["max_prefix"], z["max_own"],
                                                               self.H, self.Hkv, self.dh)
            workspace = torch.full((need // 4,), float("nan"), dtype=torch.float32, device=DEV) if need else None
        exe.exe_op_prefix_attention_paged(self.code, len(self.seqs), self.d_cu, self.rows, z["max_new"], len(self.groups), self.d_groups, self.d_prefix, z["max_group"],
                                          z["max_prefix"], self.d_q if q is None else q, q_stride or w, self.d_pool, self.n_blocks, self.d_table, self.max_blocks, self.block,
                                          self.d_len, z["max_own"], self.H, self.Hkv, self.dh, self.scale if scale is None else scale, out, out_stride or w, workspace,
                                          stream=stream)
        return out


ONES = lambda n, lo=1: [(1, lo + 7 * i) for i in range(n)]
CASES = {
    "one": [(5, [(1, 1)])], "pair": [(64, ONES(2))], "eight": [(300, ONES(8, 20))], "forty": [(777, ONES(40, 3))], "seventy": [(129, ONES(70))],
    "ragged": [(500, ONES(5)), (16, ONES(1)), (0, ONES(3)), (33, ONES(17, 40)), (1, ONES(2)), (1000, ONES(2))],
    "drafted": [(200, [(4, 9), (1, 1), (3, 3), (7, 50)]), (31, [(2, 2), (5, 5)])],
    "empty": [(100, [(0, 3), (1, 5), (0, 0), (2, 2)]), (50, []), (40, [(0, 1)]), (60, [(1, 1)])],
    "ended": [(90, [(0, 3), (0, 0)] + ONES(4)), (200, [(0, 9)] * 40 + ONES(35))],
    "chunks": [(150, [(40, 60), (1, 10), (33, 33)]), (15, [(100, 101)])],
    "long": [(5000, ONES(3, 600)), (2500, ONES(6, 2000))],
}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("case", list(CASES))
def test_groups(dtype, dh, case):
    for i, (H, Hkv) in enumerate([(4, 4), (8, 2), (5, 1)]):
        b = Groups(CASES[case], H, Hkv, dh, (16, 64, 8)[i], dtype, seed=i, extra_rows=i, loose=[(1, 70), (0, 4), (2, 3)] if i == 2 else []).fill().device()
        check(b.attend(), *b.want(), (H, Hkv))


@pytest.mark.parametrize("dtype,dh", [("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("heads", [(4, 4), (8, 2), (6, 2), (16, 1), (3, 3), (40, 8), (40, 40), (24, 8)])
def test_head_layouts(dtype, dh, heads):
    for i, groups in enumerate(([(120, ONES(3))], [(70, [(2, 5), (1, 30)]), (9, ONES(9))])):
        b = Groups(groups, *heads, dh, 32, dtype, seed=i).fill().device()
        check(b.attend(), *b.want())


@pytest.mark.parametrize("block", [8, 16, 128, 4096])
@pytest.mark.parametrize("prefix", [1, 7, 8, 15, 16, 17, 63, 64, 128, 129])
def test_prefixes_that_end_anywhere(block, prefix):
    for dtype, dh in (("bf16", 64), ("f32", 128)):
        b = Groups([(prefix, [(1, 1), (2, 20), (1, 129)])], 4, 2, dh, block, dtype, table_pad=2, loose=[(1, prefix)]).fill().device()
        check(b.attend(), *b.want())


@pytest.mark.parametrize("n", [62, 63, 64, 65, 130, 260])
def test_many_sequences_and_groups(n):
    """Every way to find a row's group: fewer than 64 of both, more sequences, more groups."""
    b = Groups([(40, ONES(n))], 2, 1, 64, 16, "bf16").fill().device()
    check(b.attend(), *b.want())
    rng = np.random.default_rng(n)
    groups = [(int(rng.integers(0, 90)), [(int(rng.integers(0, 3)), int(rng.integers(3, 40))) for _ in range(int(rng.integers(0, 3)))]) for _ in range(n)]
    b = Groups(groups, 2, 2, 64, 8, "bf16", seed=n, loose=[(1, 9)]).fill().device()
    check(b.attend(), *b.want())
    b = Groups([(20, [(1, 1)])] * n, 4, 1, 64, 16, "f32", seed=n).fill().device()
    check(b.attend(), *b.want())


def test_workgroups_of_two_waves():
    """40 heads, 8 sequences: sizes that one round of the chip holds in unequal parts."""
    b = Groups([(1500, [(1, 20 + 40 * i) for i in range(8)])], 40, 40, 128, 64, "bf16").fill().device()
    check(b.attend(), *b.want())
    b = Groups([(300 + 20 * g, [(1, 30), (1, 250 - 5 * g)]) for g in range(20)], 32, 4, 128, 16, "bf16").fill().device()
    check(b.attend(max_prefix=1500, max_own=288), *b.want())


def test_no_groups_and_no_prefix():
    b = Groups([], 4, 2, 64, 16, "bf16", loose=[(1, 50), (3, 3), (1, 700)]).fill().device()
    check(b.attend(), *b.want())
    none = torch.empty(0, dtype=torch.int32, device=DEV)
    b.d_groups, b.d_prefix = None, None
    check(b.attend(), *b.want())
    b = Groups([(0, ONES(3)), (0, ONES(2))], 4, 2, 64, 16, "bf16").fill().device()
    check(b.attend(), *b.want())
    b.d_prefix.fill_(-7)
    check(b.attend(), *b.want())


@pytest.mark.parametrize("claim", [41, 60, 1000, (1 << 31) - 1])
def test_a_prefix_beyond_the_shortest_context(claim):
    """What a call names beyond is each sequence's own: the shortest sequence's new token is at position 40."""
    for dtype in ("bf16", "f32"):
        b = Groups([(40, [(1, 1), (1, 30), (2, 100)])], 4, 2, 64, 8, dtype).fill().device()
        b.d_prefix.fill_(claim)
        check(b.attend(), *b.want())
        check(b.attend(max_prefix=min(claim, 4000)), *b.want())


def test_sizes_that_are_wrong_are_slower_not_wrong():
    b = Groups([(700, [(3, 300), (1, 40), (2, 2), (9, 500)]), (90, ONES(4))], 8, 2, 128, 16, "bf16", loose=[(5, 400)]).fill().device()
    for change in (dict(max_new=1), dict(max_group=1), dict(max_prefix=0), dict(max_own=1), dict(max_new=1, max_group=1, max_prefix=1, max_own=1), dict(max_prefix=1 << 30, max_own=1 << 30),
                   dict(max_new=1 << 30, max_group=1 << 30), dict(max_own=1 << 30, max_prefix=0)):
        check(b.attend(**change), *b.want(), change)


def test_rows_without_keys_and_missing_blocks():
    """Positions before 0 are 0; a missing block of the prefix is NaN for its group, of an own position for its sequence; others stay."""
    b = Groups([(64, ONES(3, 20)), (40, ONES(2, 3))], 4, 2, 64, 16, "bf16", loose=[(2, 20)]).fill()
    clean = b.device().attend().clone()
    b.d_len[5] = -1
    got = b.attend()
    assert bool((got[5:7] == 0).all()) and torch.equal(got[:5], clean[:5])
    b.d_len[5] = 1                                                         # one before position 0, one at it
    got = b.attend()
    assert bool((got[5] == 0).all()) and not bool(got[6].isnan().any()) and bool((got[6] != 0).any())
    b.d_len[5] = 20
    t = b.d_table.clone()
    for entry in (-1, 1 << 30, b.n_blocks):
        b.d_table[0, 2] = entry
        got = b.attend()
        assert bool(got[:3].isnan().all()) and torch.equal(got[3:], clean[3:])
        b.d_table.copy_(t)
        b.d_table[1, 64 // 16] = entry
        got = b.attend()
        assert bool(got[1].isnan().all()) and torch.equal(got[[0, 2, 3, 4, 5, 6]], clean[[0, 2, 3, 4, 5, 6]])
        b.d_table.copy_(t)
    short = b.d_table[:, :4].contiguous()                                  # a table that ends with the first prefix: its sequences' own positions are missing
    b.d_table, b.max_blocks = short, 4
    got = b.attend()
    assert bool(got[:3].isnan().all()) and torch.equal(got[3:], clean[3:])


@pytest.mark.parametrize("dtype,dh", [("bf16", 128), ("bf16", 64), ("f32", 64)])
@pytest.mark.parametrize("n", [2, 12, 40])
def test_infinities_nan_and_a_floats_end(dtype, dh, n):
    """Infinite or NaN values and keys of one sequence's own positions leave the others alone; in the prefix they are its group's; values near
    a float's end."""
    def batch():
        return Groups([(50, ONES(n, 4)), (33, ONES(2, 9))], 4, 2, dh, 16, dtype)
    for bad in (float("inf"), float("nan")):
        b = batch()
        want, tol = b.want()
        b.v[1][1, 52] = bad
        b.fill().device()
        got = b.attend().cpu().double().view(-1, 4, dh)
        w, t = want.view(-1, 4, dh), tol.view(-1, 4, dh)
        keep = torch.ones((len(w), 4), dtype=torch.bool)
        keep[1, 2:] = False
        assert bool(((got - w).abs() <= t * (1 + 1e-6))[keep].all()) and not bool(got[1, 2:].isfinite().any())
        b = batch()
        for s in range(n):
            b.k[s][0, 20] = bad
        b.fill().device()
        got = b.attend().cpu().double().view(-1, 4, dh)
        assert bool(got[:n, :2].isnan().all()) or bad == float("inf")
        assert bool(((got - w).abs() <= t * (1 + 1e-6))[:, 2:].all()) and bool(((got - w).abs() <= t * (1 + 1e-6))[n:].all())
    b = batch()
    big = 3.0e38
    for s in range(len(b.seqs)):
        b.v[s].fill_(big)
    b.fill().device()
    got = b.attend().cpu().double()
    # every value the same: the mean of them, to the roundings of the weights and the result
    assert bool(((got / float(torch.tensor(big).to(b.t))) - 1).abs().max() <= 3 * 2.0 ** -8 if dtype == "bf16" else 64 * 2.0 ** -24)


@pytest.mark.parametrize("scale", [0.0, -0.3, 4.0, 1e-3])
def test_scales(scale):
    for dtype in ("bf16", "f32"):
        b = Groups([(90, ONES(10, 5))], 4, 2, 64, 16, dtype).fill().device()
        check(b.attend(scale=scale), *b.want(scale=scale))


def test_strides_and_rows_left_alone():
    b = Groups([(90, ONES(6, 5))], 4, 2, 64, 16, "bf16", extra_rows=3).fill().device()
    want = b.attend()
    wide = torch.zeros((b.rows, 256 + 24), dtype=torch.bfloat16, device=DEV)
    wide[:, 8:264] = b.d_q
    out = torch.full((b.rows, 256 + 40), 7.0, dtype=torch.bfloat16, device=DEV)
    b.attend(q=wide[:, 8:], q_stride=280, out=out, out_stride=296)
    assert torch.equal(out[:, :256], want) and bool((out[:, 256:] == 7).all()) and bool((want[6:] == 7).all())


def test_blocks_beyond_2_31_elements():
    """A pool of more than 2^32 bytes whose last blocks are in use."""
    b = Groups([(200, ONES(4, 9))], 4, 2, 128, 64, "bf16").fill().device()
    want = b.attend()
    per = 2 * 2 * 64 * 128
    n = (1 << 31) // per + 50
    pool = torch.zeros((n, 2, 2, 64, 128), dtype=torch.bfloat16, device=DEV)
    pool[n - b.n_blocks:] = b.d_pool
    b.d_table = torch.where((b.d_table >= 0) & (b.d_table < b.n_blocks), b.d_table + (n - b.n_blocks), b.d_table)
    b.d_pool, b.n_blocks = pool, n
    assert torch.equal(b.attend(), want)


def test_against_the_chunk_attention_and_repeats():
    """Of full tables both calls give the same up to the bits of a probability; the same call gives the same bits; a group cut in two as well, nearly."""
    b = Groups([(640, ONES(9, 30))], 8, 2, 128, 32, "bf16")
    Batch.fill(b).device()
    a = b.attend()
    assert torch.equal(a, b.attend())
    c = Batch.attend(b)
    want, tol = b.want()
    assert bool(((a.double() - c.double()).abs().cpu() <= 2 * tol).all())


def test_two_streams_and_a_replayed_graph():
    """Two calls at once with a workspace each; a graph whose lengths, prefixes, groups and tables change between replays, against eager calls."""
    bs = [Groups([(300 + 50 * i, ONES(9, 5)), (80, ONES(4, 9))], 8, 2, 64, 16, "bf16", seed=i, table_pad=1).fill().device() for i in range(2)]
    want = [b.attend() for b in bs]
    streams = [torch.cuda.Stream() for _ in bs]
    torch.cuda.synchronize()
    got = [None, None]
    for _ in range(3):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i] = bs[i].attend()
    torch.cuda.synchronize()
    assert all(torch.equal(g, w) for g, w in zip(got, want))
    b = bs[0]
    Batch.fill(b).device()
    b.d_pool.nan_to_num_(nan=0.5)
    b.d_table.copy_(torch.arange(b.d_table.numel(), device=DEV).view(b.d_table.shape) % b.n_blocks)
    for s in range(1, 9):
        b.d_table[s, :18] = b.d_table[0, :18]
    need = exe.exe_op_prefix_attention_paged_workspace(b.code, 13, b.rows, 1, 2, 9, 400, max(100, BOUND), 8, 2, 64)
    assert (need == 0) == (BOUND == 1)
    ws, out = torch.empty(max(need, 16), dtype=torch.uint8, device=DEV), torch.empty((b.rows, 512), dtype=torch.bfloat16, device=DEV)
    sizes = dict(max_new=1, max_group=9, max_prefix=400, max_own=max(100, BOUND))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.attend(out=out, workspace=ws, **sizes)
    for step in range(6):
        b.d_len.add_(1)
        b.d_prefix.sub_(13)
        b.d_groups[1] = 9 - step
        b.d_q.copy_(torch.randn(b.d_q.shape, generator=torch.Generator().manual_seed(step)).bfloat16())
        graph.replay()
        torch.cuda.synchronize()
        replayed = out.clone()
        assert torch.equal(replayed, b.attend(**sizes)) and not bool(replayed.isnan().any())


@pytest.mark.parametrize("seed", range(24))
def test_random_batches(seed):
    rng = np.random.default_rng(seed)
    Hkv = int(rng.choice([1, 2, 3, 8]))
    H, dh, block = Hkv * int(rng.choice([1, 2, 4, 5])), int(rng.choice([64, 128])), int(rng.choice([8, 16, 64]))
    groups = [(int(rng.integers(0, 400)), [(int(rng.choice([0, 1, 1, 1, 2, 6])), int(rng.integers(6, 150))) for _ in range(int(rng.integers(0, 12)))])
              for _ in range(int(rng.integers(1, 7)))]
    loose = [(1, int(rng.integers(1, 200))) for _ in range(int(rng.integers(0, 3)))]
    b = Groups(groups, H, Hkv, dh, block, ["bf16", "f32"][seed % 2], seed=seed, loose=loose or [(1, 3)], extra_rows=int(rng.integers(0, 3))).fill().device()
    check(b.attend(), *b.want(), (groups, loose))


@pytest.mark.parametrize("heads", [(33, 1), (64, 1), (128, 1), (66, 2), (192, 3)])
def test_many_heads_over_one(heads):
    """Rows of one token in several tiles, and tiles that hold parts of two tokens."""
    for dtype, dh in (("bf16", 128), ("bf16", 64), ("f32", 64)):
        b = Groups([(90, [(1, 1), (0, 5), (3, 20)]), (257, [(1, 1)])], *heads, dh, 16, dtype, seed=heads[0], loose=[(1, 33)]).fill().device()
        check(b.attend(), *b.want())
        check(b.attend(max_group=1, max_new=1), *b.want())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh,n", [(64, 3), (128, 3), (64, 40), (128, 40)])
def test_values_near_a_floats_end(dtype, dh, n):
    """Values whose sums pass the largest float.  All the same: their mean, to a half step of float for each of a row's keys, 16 for each 64 of them (sums of
    weights, their inverse, the factor of what was there before) and 4 more; in bf16 a half step for the weights, the result and the tile's sum of weights too."""
    b = Groups([(50, ONES(n, 4)), (33, ONES(2, 9))], 4, 2, dh, 16, dtype)
    for v in b.v:
        v.fill_(3.0e38)
    b.fill().device()
    got = b.attend().cpu().double()
    keys = max(L for _, L in b.seqs)
    bound = (keys + 16 * -(-keys // 64) + 4) * 2.0 ** -24 + (3 * 2.0 ** -8 if dtype == "bf16" else 0.0)
    off = (got / float(torch.tensor(3.0e38).to(b.t)) - 1).abs().max()
    assert bool(off <= bound), (float(off), bound)
    b = Groups([(50, ONES(n, 4)), (33, ONES(2, 9))], 4, 2, dh, 16, dtype)
    for v in b.v:
        v.mul_(6e37)                                                      # of both signs, up to 5 times as large
    b.fill().device()
    check(b.attend(), *b.want())


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("heads,n", [((4, 4), 9), ((4, 4), 16), ((8, 2), 5), ((6, 2), 10), ((16, 1), 2)])
def test_probabilities_keep_16_bits_for_up_to_32_rows(dh, heads, n, monkeypatch):
    """bf16: the bound of `want` with what two numbers of 8 bits leave of a probability, 2^-16, in place of a half step, and that of the result.  Few keys and a small
    scale, so that the other roundings do not cover it."""
    b = Groups([(21, ONES(n))], *heads, dh, 16, "bf16").fill().device()
    monkeypatch.setitem(chunk_util.HALF, "bf16", 2.0 ** -16)
    want, tol = b.want(scale=1e-3)
    got = b.attend(scale=1e-3).cpu().double()
    over = (got - want).abs() - tol - 2.0 ** -8 * (want.abs() + tol) * (1 + 1e-6)
    assert bool((over <= 0).all()), float(over.max())


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("heads,n", [((4, 4), 40), ((8, 2), 33), ((16, 1), 9)])
def test_probabilities_keep_15_bits_for_more_rows(dh, heads, n, monkeypatch):
    """As above: what is cut off a probability after 8 bits, up to a whole step, is rounded to 8 bits of its own."""
    b = Groups([(21, ONES(n))], *heads, dh, 16, "bf16").fill().device()
    monkeypatch.setitem(chunk_util.HALF, "bf16", 2.0 ** -15)
    want, tol = b.want(scale=1e-3)
    got = b.attend(scale=1e-3).cpu().double()
    over = (got - want).abs() - tol - 2.0 ** -8 * (want.abs() + tol) * (1 + 1e-6)
    assert bool((over <= 0).all()), float(over.max())
