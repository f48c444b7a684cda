"""The workspace of the chunk attention: a tensor, or an address and its size."""
import pytest

import paper_2404_07947_amd as exe

P = 4096            # an address that no call may follow
ATTEND = dict(dtype=1, n_seqs=1, cu=P, T=4, max_new=4, q=P, q_stride=4 * 64, kv_blocks=P, n_blocks=4, table=P, max_blocks=2, block=16, length=P,
              max_len=1 << 20, H=4, Hkv=2, dh=64, scale=0.1, window=0, out=2 * P, out_stride=4 * 64)


@pytest.mark.parametrize("workspace,short,says", [(None, None, "workspace too small"), (P, 1, "workspace too small"), (P + 8, 0, "aligned")])
def test_an_address_and_its_size_reach_the_library(workspace, short, says):
    need = exe.exe_op_chunk_attention_paged_workspace(1, 1, 4, 4, 1 << 20, 4, 2, 64)
    assert need > 0
    ws_bytes = None if short is None else need - short
    with pytest.raises(exe.ExeError, match=says) as e:
        exe.exe_op_chunk_attention_paged(*ATTEND.values(), workspace, stream=1, ws_bytes=ws_bytes)
    assert e.value.code == -1


def test_an_address_alone_is_refused():
    for ws_bytes in (None, -1):                     # as an unsigned number, -1 would be room for anything
        with pytest.raises(AssertionError, match="ws_bytes"):
            exe.exe_op_chunk_attention_paged(*ATTEND.values(), P, stream=1, ws_bytes=ws_bytes)


@pytest.mark.gpu
def test_the_result_is_the_same_by_address():
    import torch
    from chunk_util import Batch
    b = Batch([(1, 3000), (2, 900)], 8, 2, 64, 16, "bf16").fill().device()
    need = exe.exe_op_chunk_attention_paged_workspace(1, 2, 3, 2, 3000, 8, 2, 64)
    assert need > 0
    ws = torch.empty(need, dtype=torch.uint8, device="cuda:0")
    want = b.attend(workspace=ws).clone()
    w = 8 * 64
    args = (1, 2, b.d_cu, b.rows, 2, b.d_q, w, b.d_pool, b.n_blocks, b.d_table, b.max_blocks, 16, b.d_len, 3000, 8, 2, 64, b.scale, 0)
    for workspace, ws_bytes in ((ws.data_ptr(), need), (ws, need), (ws, None)):
        out = torch.zeros_like(want)
        exe.exe_op_chunk_attention_paged(*args, out, w, workspace, ws_bytes=ws_bytes)
        assert torch.equal(out, want)
    with pytest.raises(AssertionError):
        exe.exe_op_chunk_attention_paged(*args, out, w, ws, ws_bytes=need + 1)
