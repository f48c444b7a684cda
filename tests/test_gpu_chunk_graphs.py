"""Rotary positions, append and attention in one captured graph: replays follow lengths, tables and contents, between eager calls."""
import numpy as np
import pytest
import torch

import paper_2404_07947_amd as exe
from chunk_util import DEV, Batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,dh", [("bf16", 128), ("f32", 64)])
def test_a_decode_loop_from_one_graph(dtype, dh):
    """Three sequences take a token a step, 40 steps across block boundaries and past the window, from a graph that was captured once; each step is
    bit by bit what eager calls make of it on a pool of their own.  Queries are turned in place, so attention reads them out of the packed rows."""
    H, Hkv, block, window = 4, 2, 16, 50
    b = Batch([(1, 15), (1, 64), (1, 130)], H, Hkv, dh, block, dtype, seed=9, table_pad=3)
    # room for 40 more positions of every sequence
    free = iter(np.random.default_rng(1).permutation(64).tolist())
    b.n_blocks, b.max_blocks = 64, 11
    table = torch.full((3, 11), -1, dtype=torch.int32)
    for i, (_, L) in enumerate(b.seqs):
        for j in range(-(-(L + 40) // block)):
            table[i, j] = next(free)
    table = table.to(DEV)
    width = (H + 2 * Hkv) * dh
    pools = [torch.zeros((64, 2, Hkv, block, dh), dtype=b.t, device=DEV) for _ in range(2)]
    cu = torch.arange(4, dtype=torch.int32, device=DEV)
    length = torch.tensor([L for _, L in b.seqs], dtype=torch.int32, device=DEV)
    f, amplitude = exe.exe_rotary_frequencies(dh)
    f = torch.as_tensor(f, device=DEV)
    rows = [torch.zeros((3, width), dtype=b.t, device=DEV) for _ in range(2)]
    outs = [torch.zeros((3, H * dh), dtype=b.t, device=DEV) for _ in range(2)]
    need = exe.exe_op_chunk_attention_paged_workspace(b.code, 3, 3, 1, 170, H, Hkv, dh, window)
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device=DEV)

    def step(i):
        exe.exe_op_rotary_append_paged(b.code, 3, cu, 3, rows[i], width, H, Hkv, dh, dh, 0, None, f, amplitude, pools[i], 64, table, 11, block, length,
                                       rows[i], width)
        exe.exe_op_chunk_attention_paged(b.code, 3, cu, 3, 1, rows[i], width, pools[i], 64, table, 11, block, length, 170, H, Hkv, dh, dh ** -0.5, window,
                                         outs[i], H * dh, ws)
        exe.exe_op_rotary(b.code, 3, outs[i], H * dh, H, dh, dh, 0, length, f, 1.0, outs[i], H * dh)

    graph = torch.cuda.CUDAGraph()
    step(0)
    pools[0].zero_()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step(0)
    g = torch.Generator().manual_seed(4)
    for _ in range(40):
        new = torch.randn((3, width), generator=g).to(b.t)
        for r in rows:
            r.copy_(new)
        graph.replay()
        step(1)
        torch.cuda.synchronize()
        assert torch.equal(outs[0], outs[1]) and torch.equal(rows[0], rows[1]) and torch.equal(pools[0], pools[1])
        assert bool(torch.isfinite(outs[0].float()).all()) and bool((outs[0] != 0).any())
        length += 1
