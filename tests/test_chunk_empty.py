"""A batch without tokens, or without sequences, is nothing to do: an empty tensor has no address, and the longest chunk of none is 0."""
import pytest

import paper_2404_07947_amd as exe

# what an empty batch has in hand: no address of a packed array, a table or lengths
ROTARY = dict(dtype=1, T=0, x=None, x_stride=256, heads=4, dh=64, rot=64, interleaved=0, pos=None, inv_freq=None, amplitude=1.0, out=None, out_stride=256)
APPEND = dict(dtype=1, n_seqs=0, cu=None, T=0, qkv=None, row_stride=512, H=4, Hkv=2, dh=64, rot=64, interleaved=0, pos=None, inv_freq=None, amplitude=1.0,
              kv_blocks=None, n_blocks=4, table=None, max_blocks=2, block=16, length=None, q_out=None, q_stride=256)
ATTEND = dict(dtype=1, n_seqs=0, cu=None, T=0, max_new=0, q=None, q_stride=256, kv_blocks=None, n_blocks=4, table=None, max_blocks=2, block=16, length=None,
              max_len=0, H=4, Hkv=2, dh=64, scale=0.1, window=0, out=None, out_stride=256)


@pytest.mark.parametrize("fn,base", [(exe.exe_op_rotary, ROTARY), (exe.exe_op_rotary_append_paged, APPEND), (exe.exe_op_chunk_attention_paged, ATTEND)])
def test_no_address_is_asked_for(fn, base):
    fn(*base.values(), stream=1)
    if "n_seqs" in base:
        fn(*{**base, "n_seqs": 3}.values(), stream=1)           # sequences that bring nothing
        fn(*{**base, "T": 8}.values(), stream=1)                # rows behind the last of no sequences


@pytest.mark.parametrize("fn,base,change,code", [
    (exe.exe_op_rotary, ROTARY, dict(dtype=2), -1), (exe.exe_op_rotary, ROTARY, dict(dh=80), -2), (exe.exe_op_rotary, ROTARY, dict(rot=3), -2),
    (exe.exe_op_rotary, ROTARY, dict(x_stride=255), -2), (exe.exe_op_rotary, ROTARY, dict(T=4), -1),
    (exe.exe_op_rotary_append_paged, APPEND, dict(block=12), -1), (exe.exe_op_rotary_append_paged, APPEND, dict(T=-1), -1),
    (exe.exe_op_rotary_append_paged, APPEND, dict(T=4, n_seqs=1), -1), (exe.exe_op_rotary_append_paged, APPEND, dict(row_stride=511), -2),
    (exe.exe_op_chunk_attention_paged, ATTEND, dict(H=3), -2), (exe.exe_op_chunk_attention_paged, ATTEND, dict(max_new=-1), -1),
    (exe.exe_op_chunk_attention_paged, ATTEND, dict(max_len=-1), -1), (exe.exe_op_chunk_attention_paged, ATTEND, dict(q_stride=257), -2),
    (exe.exe_op_chunk_attention_paged, ATTEND, dict(T=4, n_seqs=1, max_new=4, max_len=4), -1)])
def test_sizes_are_looked_at_all_the_same(fn, base, change, code):
    with pytest.raises(exe.ExeError) as e:
        fn(*{**base, **change}.values(), stream=1)
    assert e.value.code == code


@pytest.mark.gpu
@pytest.mark.parametrize("n_seqs", [0, 3])
def test_empty_tensors(n_seqs):
    import torch
    d = dict(device="cuda:0")
    rows = lambda w: torch.empty((0, w), dtype=torch.bfloat16, **d)
    cu, length = torch.zeros(n_seqs + 1, dtype=torch.int32, **d), torch.zeros(n_seqs, dtype=torch.int32, **d)
    table = torch.zeros((n_seqs, 2), dtype=torch.int32, **d)
    pool = torch.ones((4, 2, 2, 16, 64), dtype=torch.bfloat16, **d)
    f = torch.ones(32, dtype=torch.float64, **d)
    exe.exe_op_rotary(1, 0, rows(256), 256, 4, 64, 64, 0, torch.zeros(0, dtype=torch.int32, **d), f, 1.0, rows(256), 256)
    exe.exe_op_rotary_append_paged(1, n_seqs, cu, 0, rows(512), 512, 4, 2, 64, 64, 0, None, f, 1.0, pool, 4, table, 2, 16, length, rows(256), 256)
    assert exe.exe_op_chunk_attention_paged_workspace(1, n_seqs, 0, 0, 0, 4, 2, 64) == 0
    exe.exe_op_chunk_attention_paged(1, n_seqs, cu, 0, 0, rows(256), 256, pool, 4, table, 2, 16, length, 0, 4, 2, 64, 0.125, 0, rows(256), 256)
    torch.cuda.synchronize()
    assert bool((pool == 1).all())
