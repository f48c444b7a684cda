"""Attention of a chunk of new tokens over a paged cache, against 64 bits: every row of every case.  Whatever lies in the cache behind
a sequence's end is NaN in all of them, and the table's unused entries name no block."""
import numpy as np
import pytest
import torch

import chunk_util
from chunk_util import DEV, HALF, U, Batch, check

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, params=[1, 1100], ids=["own", "tiles"])
def bound(request, monkeypatch):
    """Calls of few rows and up to 1024 keys go to the streaming kernel: with a larger bound of the lengths, to the tile kernel."""
    monkeypatch.setattr(chunk_util, "BOUND", request.param)


HEADS = [(4, 4), (8, 2), (6, 2), (5, 1), (16, 1), (3, 3), (40, 8)]
# (new tokens, positions with them)
LENGTHS = {
    "one": [(1, 1)], "single_tokens": [(1, 17), (1, 64), (1, 65), (1, 500), (1, 1), (1, 129)],
    "whole_prompts": [(1, 1), (5, 5), (64, 64), (65, 65), (130, 130), (257, 257)],
    "chunks": [(3, 40), (16, 16), (17, 300), (64, 200), (100, 1000), (129, 131)],
    "mixed": [(1, 900), (0, 30), (33, 33), (1, 2), (0, 0), (200, 777), (2, 64)],
    "long": [(1, 5000), (7, 4097)],
}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("lengths", list(LENGTHS))
def test_lengths(dtype, dh, lengths):
    for i, (H, Hkv) in enumerate([(4, 4), (8, 2)]):
        b = Batch(LENGTHS[lengths], H, Hkv, dh, (16, 64)[i], dtype, seed=i, extra_rows=3).fill().device()
        check(b.attend(), *b.want(), (H, Hkv))


@pytest.mark.parametrize("dtype,dh", [("bf16", 128), ("bf16", 64), ("f32", 64), ("f32", 128)])
def test_single_tokens_beside_chunks(dtype, dh):
    """Many single tokens and one longer chunk (both kernels in one call, long ones in parts), and few single tokens among chunks (one)."""
    for seqs in ([(1, 1000 + 90 * i) for i in range(9)] + [(40, 900), (1, 3)], [(1, 5000), (30, 40), (1, 4500)], [(100, 300), (1, 800), (70, 70), (2, 2)]):
        b = Batch(seqs, 4, 2, dh, 16, dtype, seed=len(seqs), extra_rows=1).fill().device()
        check(b.attend(), *b.want(), seqs)


@pytest.mark.parametrize("G,n,L,Hkv", [(8, 128, 400, 8), (8, 64, 300, 2), (1, 600, 600, 3), (4, 300, 1500, 1)])
@pytest.mark.parametrize("dh", [64, 128])
def test_tiles_that_share_their_keys(G, n, L, Hkv, dh):
    """Tiles of 64 and of 128 rows, with and without a window, a second sequence that ends inside a tile."""
    for window in (0, 100):
        b = Batch([(n, L), (n // 2 + 1, n)], G * Hkv, Hkv, dh, 16, "bf16", seed=G).fill().device()
        check(b.attend(window=window), *b.want(window=window), window)


@pytest.mark.parametrize("dh,H,Hkv,n,L", [(64, 512, 64, 512, 520), (128, 64, 8, 300, 700), (128, 32, 8, 1100, 2300)])
@pytest.mark.parametrize("window", [0, 130])
def test_full_chips(dh, H, Hkv, n, L, window):
    """Launches that fill the chip with tiles of 128 rows; the reference is computed on the device, in 64 bits and 4 heads at a time."""
    b = Batch([(n, L)], H, Hkv, dh, 32, "bf16").fill().device()
    got = b.attend(window=window).double().view(n, H, dh)
    key, pos = torch.arange(L, device=DEV)[None], torch.arange(L - n, L, device=DEV)[:, None]
    seen = (key <= pos) & ((key > pos - window) if window else True)
    count = seen.sum(1).double()[:, None, None]
    for h in range(0, H, 4):
        kv = [h // (H // Hkv), (h + 3) // (H // Hkv) + 1]
        rep = 4 // (kv[1] - kv[0])
        k, v = (t[0][kv[0]:kv[1]].to(DEV).double().repeat_interleave(rep, 0) for t in (b.k, b.v))
        q = b.d_q.double().view(n, H, dh)[:, h:h + 4].transpose(0, 1).contiguous()
        s = torch.matmul(q, k.transpose(1, 2).contiguous()) * b.scale
        mag = (torch.matmul(q.abs(), k.abs().transpose(1, 2).contiguous()) * b.scale).masked_fill(~seen, 0).amax(-1)
        top = s.abs().masked_fill(~seen, 0).amax(-1)
        p = torch.softmax(s.masked_fill(~seen, -float("inf")), -1)
        want = torch.matmul(p, v).transpose(0, 1)
        e = (2 * (dh + 8) * U * mag + 8 * U * (1 + top)).t()[..., None] + (count + 16) * 2 * U + HALF["bf16"]
        tol = e * torch.matmul(p, v.abs()).transpose(0, 1) + HALF["bf16"] * want.abs() + 1e-30         # as Batch.want has it
        assert bool(((got[:, h:h + 4] - want).abs() <= tol * (1 + 1e-6)).all()), h


@pytest.mark.parametrize("dtype,dh", [("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("heads", HEADS)
def test_head_layouts(dtype, dh, heads):
    for i, lengths in enumerate(([(1, 300), (1, 77)], [(20, 100), (1, 200), (3, 3)])):
        b = Batch(lengths, *heads, dh, 32, dtype, seed=i).fill().device()
        check(b.attend(), *b.want(), lengths)


@pytest.mark.parametrize("block", [8, 16, 128, 4096])
@pytest.mark.parametrize("dtype,dh", [("bf16", 64), ("bf16", 128), ("f32", 128)])
def test_block_sizes(dtype, dh, block):
    b = Batch([(1, 150), (70, 300), (1, 8), (9, 9)], 4, 2, dh, block, dtype, table_pad=2).fill().device()
    check(b.attend(), *b.want())


@pytest.mark.parametrize("dtype,dh", [("bf16", 128), ("bf16", 64), ("f32", 64)])
@pytest.mark.parametrize("window", [1, 2, 63, 64, 65, 200, 1 << 30])
def test_windows(dtype, dh, window):
    b = Batch([(1, 400), (90, 500), (1, 1), (30, 30), (1, 64)], 4, 2, dh, 16, dtype).fill().device()
    check(b.attend(window=window), *b.want(window=window))
    b = Batch([(1, 1400), (2, 2000)], 8, 2, dh, 16, dtype).fill().device()
    check(b.attend(window=window), *b.want(window=window))


@pytest.mark.parametrize("dtype,dh", [("bf16", 128), ("bf16", 64), ("f32", 64), ("f32", 128)])
def test_bounds_that_size_the_launch_do_not_change_the_result_beyond_rounding(dtype, dh):
    b = Batch([(1, 700), (40, 300), (3, 1500)], 8, 2, dh, 16, dtype).fill().device()
    want, tol = b.want()
    for max_new, max_len in ((1, 1), (1, 1500), (3, 100), (40, 1), (1000, 100000), (40, 1500)):
        check(b.attend(max_new=max_new, max_len=max_len), want, tol, (max_new, max_len))


@pytest.mark.parametrize("dtype,dh", [("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("scale", [0.0, -0.2, 3.0, 1e-3])
def test_scales(dtype, dh, scale):
    b = Batch([(1, 100), (40, 77)], 4, 2, dh, 16, dtype).fill().device()
    check(b.attend(scale=scale), *b.want(scale=scale))


@pytest.mark.parametrize("dtype,dh", [("bf16", 128), ("bf16", 64), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_what_later_positions_and_the_window_hide_may_be_anything(dtype, dh, bad):
    """Keys and values of the last tokens (and of the first, behind the window) are infinite or NaN: rows that do not see them are as
    without them, the others are what a softmax of them is."""
    seqs = [(70, 300), (20, 20), (2, 200), (1, 200)]
    b = Batch(seqs, 8, 2, dh, 16, dtype)
    window = 150
    want, tol = b.want(window=window)
    clean = torch.ones(b.rows, dtype=torch.bool)
    for i, (n, L) in enumerate(seqs):
        late = max(L - n + 1, L - n // 3)                      # the positions late .. L - 1 and 0 .. 9 go bad
        for a in (b.k[i], b.v[i]):
            a[:, late:] = bad
            if L > window + n + 10:
                a[:, :10] = bad
        for j in range(n):
            clean[int(b.cu[i]) + j] = L - n + j < late
    got = b.fill().device().attend(window=window)
    check(got[clean], want[clean], tol[clean])
    assert int(clean.sum()) > 60 and int((~clean).sum()) > 0
    assert not bool(torch.isfinite(got.float().cpu()[~clean]).any())


@pytest.mark.parametrize("dtype,dh", [("bf16", 128), ("f32", 64)])
def test_rows_without_keys_are_zero(dtype, dh):
    b = Batch([(1, 40), (5, 12), (3, 3)], 4, 2, dh, 16, dtype).fill().device()
    b.seqs = [(1, 0), (5, 2), (3, -4)]                          # five new tokens of two positions: three lie before the first one
    b.k[1], b.v[1] = b.k[1][:, :2], b.v[1][:, :2]
    b.d_len = torch.tensor([0, 2, -4], dtype=torch.int32, device=DEV)
    got = b.attend(max_len=40)
    check(got, *b.want())
    assert bool((got[[0, 1, 2, 3, 6, 7, 8]] == 0).all()) and bool((got[[4, 5]] != 0).any())


@pytest.mark.parametrize("dtype,dh", [("bf16", 128), ("bf16", 64), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("entry", [-1, 1 << 30, None])
def test_positions_without_a_block_give_nan(dtype, dh, entry):
    """A table entry outside of the pool is not followed (None: the table is too short): rows that would read it are NaN, other
    sequences are as they were."""
    b = Batch([(1, 200), (80, 200), (1, 50), (80, 80)], 4, 2, dh, 16, dtype).fill()
    want, tol = b.want()
    if entry is None:
        b.table, b.max_blocks = b.table[:, :9], 9               # positions from 144 on have no entry
    else:
        b.table[:2, 9] = entry
    got = b.device().attend()
    rows = [0] + list(range(1 + 24, 81))                        # positions 144 and up
    assert bool(torch.isnan(got[rows].float()).all())
    other = list(range(81, b.rows))
    check(got[other], want[other], tol[other])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strided_rows(dtype):
    b = Batch([(1, 100), (40, 90)], 4, 2, 64, 16, dtype).fill().device()
    import paper_2404_07947_amd as exe
    w = b.H * b.dh
    wide = torch.zeros((b.rows, 3 * w + 16), dtype=b.t, device=DEV)
    wide[:, 2 * w:3 * w] = b.d_q
    out = torch.full((b.rows, w + 8), 7.0, dtype=b.t, device=DEV)
    ws = torch.empty(max(16, exe.exe_op_chunk_attention_paged_workspace(b.code, 2, b.rows, 40, 100, 4, 2, 64)), dtype=torch.uint8, device=DEV)
    exe.exe_op_chunk_attention_paged(b.code, 2, b.d_cu, b.rows, 40, wide[:, 2 * w:], 3 * w + 16, b.d_pool, b.n_blocks, b.d_table, b.max_blocks, 16,
                                     b.d_len, 100, 4, 2, 64, b.scale, 0, out, w + 8, ws)
    check(out[:, :w].contiguous(), *b.want())
    assert bool((out[:, w:] == 7).all())


def test_offsets_beyond_32_bits():
    """A pool of more than 2^32 elements, in which the blocks lie at its end."""
    H, Hkv, dh, block = 8, 8, 128, 64
    b = Batch([(1, 300), (70, 200)], H, Hkv, dh, block, "bf16").fill()
    per = 2 * Hkv * block * dh
    n = (1 << 32) // per + 40
    pool = torch.empty(n * per, dtype=torch.bfloat16, device=DEV)
    pool[(n - b.n_blocks) * per:] = b.pool.to(DEV).flatten()
    want = b.want()
    b.device()
    b.d_pool, b.d_table = pool, (b.d_table + (n - b.n_blocks)).clamp_(max=1 << 30)
    b.n_blocks = n
    check(b.attend(), *want)


@pytest.mark.parametrize("dtype,dh", [("bf16", 128), ("f32", 64)])
def test_graph_replays_follow_lengths_and_tables(dtype, dh):
    """A captured launch reads lengths, table and cu_seqlens from the device; two graphs share a workspace one after the other."""
    a = Batch([(1, 700), (30, 400)], 8, 2, dh, 16, dtype, seed=1, table_pad=40).fill().device()
    c = Batch([(30, 90), (1, 900)], 8, 2, dh, 16, dtype, seed=2).fill()
    import paper_2404_07947_amd as exe
    ws = torch.empty(max(16, exe.exe_op_chunk_attention_paged_workspace(a.code, 2, a.rows, 30, 1300, 8, 2, dh)), dtype=torch.uint8, device=DEV)
    outs = [torch.zeros((a.rows, 8 * dh), dtype=a.t, device=DEV) for _ in range(2)]
    for o in outs:
        a.attend(max_new=30, max_len=1300, out=o, workspace=ws)
    graphs = []
    for o in outs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            a.attend(max_new=30, max_len=1300, out=o, workspace=ws)
        graphs.append(g)
    first = outs[0].clone()
    for k in range(3):
        for g, o in zip(graphs, outs):
            o.fill_(3.0)
            g.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], first) and torch.equal(outs[1], first)
        check(outs[0], *a.want())
    # other contents, lengths and tables in the same places
    assert c.n_blocks <= a.n_blocks and c.max_blocks <= a.max_blocks
    table = torch.full_like(a.d_table, 1 << 30)
    a.d_pool[:c.n_blocks] = c.pool.to(DEV)
    table[:, :c.max_blocks] = torch.as_tensor(c.table).to(DEV)
    a.d_table.copy_(table)
    a.d_cu.copy_(torch.as_tensor(c.cu))
    a.d_len.copy_(torch.as_tensor([L for _, L in c.seqs], dtype=torch.int32))
    a.d_q.copy_(c.q.to(DEV))
    for g in graphs:
        g.replay()
    torch.cuda.synchronize()
    check(outs[0], *c.want())
    assert torch.equal(outs[0], outs[1])


def test_two_streams_and_repeats_give_the_same_bits():
    b = Batch([(1, 3000), (50, 900), (1, 40)], 8, 2, 128, 16, "bf16").fill().device()
    first = b.attend().clone()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = []
    for _ in range(3):
        for s in streams:
            with torch.cuda.stream(s):
                outs.append(b.attend())
    torch.cuda.synchronize()
    assert all(torch.equal(o, first) for o in outs)


def test_random_batches():
    rng = np.random.default_rng(77)
    for i in range(24):
        Hkv = int(rng.choice([1, 2, 3, 5]))
        H = Hkv * int(rng.choice([1, 2, 4, 7]))
        seqs = []
        for _ in range(int(rng.integers(1, 9))):
            n = int(rng.choice([0, 1, 1, 1, rng.integers(2, 20), rng.integers(2, 150)]))
            seqs.append((n, n + int(rng.choice([0, rng.integers(0, 80), rng.integers(0, 700)]))))
        if not sum(n for n, _ in seqs):
            seqs.append((2, 5))
        dtype, dh, block, window = str(rng.choice(["bf16", "f32"])), int(rng.choice([64, 128])), int(rng.choice([8, 16, 64])), int(rng.choice([0, 0, 37]))
        b = Batch(seqs, H, Hkv, dh, block, dtype, seed=i, extra_rows=int(rng.integers(0, 3))).fill().device()
        check(b.attend(window=window), *b.want(window=window), (i, seqs, H, Hkv, dtype, dh, block, window))
