"""Copies of pages, forks of sequences that share them, and the operations on a paged cache run together."""
import numpy as np
import pytest
import torch

import paper_2404_07947_amd as exe
import workload as wl
from chunk_util import DEV, TYPES, Batch, check, turned
from gpu_util import kv_bytes_per_token, make_pair
from test_gpu_paged import oracle_tokens

pytestmark = pytest.mark.gpu


def copied(pool, copies):
    want = pool.clone()
    for s, d, n in copies:
        want[:, d, :, :, :n] = pool[:, s, :, :, :n]
    return want


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layers,Hkv,dh,block", [(1, 1, 64, 8), (3, 5, 64, 16), (2, 8, 128, 64), (1, 2, 128, 4096)])
def test_copies(dtype, layers, Hkv, dh, block):
    n = 40
    pool = torch.randn((layers, n, 2, Hkv, block, dh), generator=torch.Generator().manual_seed(1)).to(TYPES[dtype][1]).to(DEV)
    lists = [[(0, 1, block)], [(5, n - 1, 1)], [(3, 4, 0)], [], [(7, d, (d * 5) % (block + 1)) for d in range(10, 30)],
             [(d, d + 20, block) for d in range(20)], [(d, d + 20, 1 + d % block) for d in range(20)]]
    for copies in lists:
        got = pool.clone()
        exe.exe_op_kv_copy_blocks(TYPES[dtype][0], got, layers, n, block, Hkv, dh, copies)
        assert torch.equal(got, copied(pool, copies)), copies


def test_more_copies_than_a_launch_lists():
    n, block = 1500, 8
    pool = torch.randn((2, n, 2, 1, block, 64), device=DEV)
    order = np.random.default_rng(1).permutation(n)
    copies = [(int(order[i]), int(order[700 + i]), 1 + i % block) for i in range(700)]
    got = pool.clone()
    exe.exe_op_kv_copy_blocks(0, got, 2, n, block, 1, 64, copies)
    assert torch.equal(got, copied(pool, copies))


def test_captured_copies_keep_their_list():
    pool = torch.randn((2, 10, 2, 2, 16, 64), device=DEV)
    got = pool.clone()
    copies = np.array([(0, 5, 16), (1, 6, 3)], dtype=np.int32)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        exe.exe_op_kv_copy_blocks(0, got, 2, 10, 16, 2, 64, copies)
    copies[:] = -1
    for _ in range(3):
        got.copy_(pool)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, copied(pool, [(0, 5, 16), (1, 6, 3)]))


# ---------------------------------------------------------------- forks in the model

@pytest.mark.parametrize("block", [8, 16, 0])
@pytest.mark.parametrize("length", [21, 16, 1])
def test_forks_continue_on_their_own(block, length):
    """Three forks of a prompt are fed different tokens: each gives what the oracle gives for that continuation alone."""
    shape = wl.tiny_shape()
    m, o, _ = make_pair(shape, wl.BASE_SEED, "float", pool_tokens=512, max_seqs=8, max_batch_tokens=256, max_batch_seqs=8, kv_block_size=block)
    rng = np.random.default_rng(7)
    toks = wl.random_tokens(rng, length, shape.vocab)
    m.encode([2], [length], toks)
    used = m.kv_stats()["used_bytes"]
    m.seq_fork(2, [5, 0, 7])
    per = kv_bytes_per_token(shape)
    if block:
        assert m.kv_stats()["used_bytes"] - used == 3 * (block * per if length % block else 0)
    assert m.kv_stats()["live_seqs"] == 4 and all(m.seq_length(i) == length for i in (2, 5, 0, 7))
    ids = [2, 5, 0, 7]
    fed = wl.random_tokens(rng, 4 * 20, shape.vocab).reshape(20, 4)
    logits = torch.zeros((4, shape.vocab), device=DEV)
    got = []
    for s in range(20):
        if s == 9:
            m.seq_release([2])                              # the forks outlive the sequence that they come from
            ids = [5, 0, 7]
        k = len(ids)
        m.decode_step(ids, fed[s, 4 - k:], [length + s + 1] * k, out_device=logits[4 - k:])
        got.append(logits.cpu().numpy().copy())
    for col, steps in ((0, 9), (1, 20), (2, 20), (3, 20)):
        o.encode(0, toks)
        for s in range(steps):
            _, want = o.decode(0, int(fed[s, col]))
            assert np.max(np.abs(got[s][col] - want)) <= 1e-4 * np.max(np.abs(want)), (col, s)
        o.release(0)
    m.seq_release([5, 0])
    buf, st = m.seq_export(7)
    assert st["kv_len"] == length + 20
    m.seq_release([7])
    assert m.kv_stats()["used_bytes"] == 0 and m.kv_stats()["live_seqs"] == 0
    m.close()


def test_forks_of_forks_share_until_the_last_leaves():
    shape, block = wl.tiny_shape(), 8
    m, o, _ = make_pair(shape, wl.BASE_SEED, "float", pool_tokens=80, max_seqs=8, max_batch_tokens=256, max_batch_seqs=8, kv_block_size=block)
    per = block * kv_bytes_per_token(shape)
    used = lambda: m.kv_stats()["used_bytes"] // per
    rng = np.random.default_rng(8)
    toks = wl.random_tokens(rng, 19, shape.vocab)
    want = oracle_tokens(o, toks, 12)
    cur = m.encode([0], [19], toks)
    assert used() == 3
    m.seq_fork(0, [1])
    m.seq_fork(1, [2])
    assert used() == 5                                       # two full blocks once, three last ones
    m.seq_fork(2, [3, 4, 5, 6, 7])
    assert used() == 10
    m.seq_release([0, 3, 4, 5, 6, 7])
    assert used() == 4
    got = [int(cur[0])]
    both = np.array([cur[0], cur[0]])
    for s in range(1, 13):
        both = m.decode_step([1, 2], both, [19 + s] * 2)
        assert both[0] == both[1]
        got.append(int(both[0]))
    assert got == want and used() == 2 + 2 * 2
    m.seq_reserve(1, 60)
    m.seq_reserve(1, 31)
    assert used() == 6
    m.seq_release([1])
    assert used() == 4
    m.seq_release([2])
    assert used() == 0
    # every block is free again, once: the pool fills and refuses as a new one does
    m.encode([0, 2], [40, 40], wl.random_tokens(rng, 80, shape.vocab))          # (the position table ends at 64)
    assert used() == 10
    with pytest.raises(exe.ExeError) as e:
        m.encode([1], [1], [1])
    assert e.value.code == -3
    m.close()


def test_fork_refusals_change_nothing():
    shape = wl.tiny_shape()
    for block in (8, 0):
        m, _, _ = make_pair(shape, wl.BASE_SEED, "float", pool_tokens=48, max_seqs=6, max_batch_tokens=256, max_batch_seqs=8, kv_block_size=block)
        m.encode([0, 1], [20, 3], wl.random_tokens(np.random.default_rng(1), 23, shape.vocab), reserve_lengths=[24, 8])
        before = m.kv_stats()
        for src, ids, code in ((2, [3], -4), (-1, [3], -4), (6, [3], -4), (0, [1], -4), (0, [0], -4), (0, [2, 2], -4), (0, [6], -4), (0, [-1], -4),
                               (0, [2, 3, 4, 5], -3)):
            with pytest.raises(exe.ExeError) as e:
                m.seq_fork(src, ids)
            assert e.value.code == code, (block, src, ids)
            assert m.kv_stats() == before and m.seq_length(0) == 20
        m.seq_fork(0, [])
        assert m.kv_stats() == before
        m.close()


def test_fork_of_an_encoder_decoder_sequence():
    shape = wl.small_t5_shape(wl.DTYPE_F32)
    m, o, _ = make_pair(shape, 3, "float", pool_tokens=512, max_seqs=4, max_batch_tokens=256, max_batch_seqs=4)
    rng = np.random.default_rng(2)
    toks = wl.random_tokens(rng, 30, shape.vocab)
    m.encode([1], [30], toks, reserve_lengths=[40], want_tokens=False)
    o.encode(1, toks)
    logits = torch.zeros((2, shape.vocab), device=DEV)
    m.decode_step([1], [0], [1])
    o.decode(1, 0)
    m.seq_fork(1, [3])
    m.seq_release([1])
    for s, t in enumerate((5, 9, 2)):
        m.decode_step([3], [t], [s + 2], out_device=logits[:1])
        _, want = o.decode(1, t)
        assert np.max(np.abs(logits[0].cpu().numpy() - want)) <= 1e-4 * np.max(np.abs(want))
    m.close()


# ---------------------------------------------------------------- together

@pytest.mark.parametrize("dtype,dh,H,Hkv", [("bf16", 128, 4, 4), ("bf16", 64, 8, 2), ("f32", 64, 4, 4), ("f32", 128, 6, 3)])
def test_a_prompt_in_chunks_forked_and_decoded(dtype, dh, H, Hkv):
    """A prompt of 150 tokens goes in in chunks of 1, 64, 7, 70 and 8 tokens (append, then attention), is forked by copying its last
    page, and both branches take three tokens of their own.  Every output is that of attention over the whole sequence's turned
    keys; the last one of equal head numbers also that of the single-token decode attention."""
    block, code, t = 16, *TYPES[dtype]
    g = torch.Generator().manual_seed(11)
    total, w = 150, (H + 2 * Hkv) * dh
    rows = torch.randn((total + 6, w), generator=g).to(t)          # the prompt, then three tokens of each branch
    inv, amplitude = exe.exe_rotary_frequencies(dh, scaling=exe.ROPE_LINEAR, factor=2.0)
    f = torch.as_tensor(inv, device=DEV)
    n_blocks = 40
    pool = torch.full((1, n_blocks, 2, Hkv, block, dh), float("nan"), dtype=t, device=DEV)
    free = np.random.default_rng(1).permutation(n_blocks).tolist()
    tables = [[free.pop() for _ in range(10)]]
    outs = {}

    def step(qkv, lens_new, lens_all, tbl):
        cu = torch.tensor(np.concatenate([[0], np.cumsum(lens_new)]), dtype=torch.int32, device=DEV)
        L = torch.tensor(lens_all, dtype=torch.int32, device=DEV)
        tb = torch.tensor(tbl, dtype=torch.int32, device=DEV)
        T, n = qkv.shape[0], len(lens_new)
        x = qkv.to(DEV)
        q = torch.empty((T, H * dh), dtype=t, device=DEV)
        exe.exe_op_rotary_append_paged(code, n, cu, T, x, w, H, Hkv, dh, dh, 0, None, f, amplitude, pool, n_blocks, tb, 10, block, L, q, H * dh)
        out = torch.empty_like(q)
        ws = torch.empty(max(16, exe.exe_op_chunk_attention_paged_workspace(code, n, T, max(lens_new), 200, H, Hkv, dh)), dtype=torch.uint8, device=DEV)
        exe.exe_op_chunk_attention_paged(code, n, cu, T, max(lens_new), q, H * dh, pool, n_blocks, tb, 10, block, L, 200, H, Hkv, dh, dh ** -0.5, 0, out,
                                         H * dh, ws)
        return q, out, L, tb

    at, q_all, o_all = 0, [], []
    for n in (1, 64, 7, 70, 8):
        q, o, _, _ = step(rows[at:at + n], [n], [at + n], tables)
        q_all.append(q)
        o_all.append(o)
        at += n
    last = free.pop()
    exe.exe_op_kv_copy_blocks(code, pool, 1, n_blocks, block, Hkv, dh, [(tables[0][9], last, total % block)])
    tables.append(tables[0][:9] + [last])
    for s in range(3):
        q, o, L, tb = step(rows[[total + 2 * s, total + 2 * s + 1]], [1, 1], [total + s + 1] * 2, tables)
        q_all.append(q)
        o_all.append(o)
    if H == Hkv:
        d = torch.empty_like(o)
        exe.exe_op_decode_attention_paged(code, 2, q, H * dh, pool, tb, 10, block, L, L - 1, H, dh, dh ** -0.5, None, 0, 0, d)
        half = 2.0 ** -24 if dtype == "f32" else 2.0 ** -8
        # either is within its own bound of the result; both bounds are below 4 half steps of the values' sizes here
        assert float((d.float() - o.float()).abs().max()) <= (4 * half + 1e-5) * float(pool.float().nan_to_num().abs().max())
    # what the branches are: the prompt, then their own tokens
    branch = [torch.cat([rows[:total], rows[total + i::2]]) for i in range(2)]
    for i in range(2):
        b = Batch([(total + 3, total + 3)], H, Hkv, dh, block, dtype)
        x = branch[i].view(total + 3, H + 2 * Hkv, dh)
        # the library's own turned keys and queries (their error is tested elsewhere)
        b.q = torch.cat([torch.cat(q_all[:5]), torch.stack([q[i] for q in q_all[5:]])]).cpu()
        blocks = pool[0, torch.tensor(tables[i], device=DEV)].cpu()
        kv = blocks.permute(1, 2, 0, 3, 4).reshape(2, Hkv, 160, dh)[:, :, :total + 3]
        y, e = turned(x[:, H:H + Hkv], torch.arange(total + 3), torch.as_tensor(inv), amplitude, dh, 0)
        half = 2.0 ** -24 if dtype == "f32" else 2.0 ** -8
        assert bool(((kv[0].double() - y.transpose(0, 1)).abs() <= e.transpose(0, 1) + half * y.transpose(0, 1).abs() * (1 + 1e-6)).all())
        assert torch.equal(kv[1], x[:, H + Hkv:].transpose(0, 1))
        b.k, b.v = [kv[0]], [kv[1]]
        got = torch.cat([torch.cat(o_all[:5]), torch.stack([o[i] for o in o_all[5:]])])
        check(got, *b.want())
