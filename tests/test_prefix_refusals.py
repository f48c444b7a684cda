"""What attention over shared prefixes refuses, before anything of the device is touched (CPU)."""
import pytest

import paper_2404_07947_amd as exe

P = 4096            # an address that no call may follow
GOOD = dict(dtype=1, n_seqs=2, cu=P, T=4, max_new=2, n_groups=1, cu_groups=P, prefix=P, max_group=4, max_prefix=900, q=P, q_stride=256, kv_blocks=P, n_blocks=4, table=P,
            max_blocks=2, block=16, length=P, max_own=9, H=4, Hkv=2, dh=64, scale=0.1, out=2 * P, out_stride=256)


def refused(code, ws=P, ws_bytes=1 << 40, **change):
    with pytest.raises(exe.ExeError) as e:
        exe.exe_op_prefix_attention_paged(*{**GOOD, **change}.values(), ws, stream=1, ws_bytes=ws_bytes)
    assert e.value.code == code, change


@pytest.mark.parametrize("change,code", [
    (dict(dtype=2), -1), (dict(dh=96), -2), (dict(Hkv=0), -1), (dict(n_blocks=0), -1), (dict(max_blocks=0), -1), (dict(block=12), -1), (dict(n_seqs=-1), -1), (dict(T=-1), -1),
    (dict(n_groups=-1), -1), (dict(max_new=0), -1), (dict(max_group=0), -1), (dict(max_prefix=-1), -1), (dict(max_own=0), -1), (dict(H=3), -2), (dict(H=1), -2), (dict(T=1 << 30), -2),
    (dict(q_stride=255), -2), (dict(q_stride=257), -2), (dict(out_stride=252), -2), (dict(cu=None), -1), (dict(q=None), -1), (dict(kv_blocks=None), -1), (dict(table=None), -1),
    (dict(length=None), -1), (dict(out=None), -1), (dict(cu_groups=None), -1), (dict(prefix=None), -1), (dict(q=P + 4), -1), (dict(out=P + 2), -1), (dict(kv_blocks=P + 8), -1),
    (dict(out=P), -1)])
def test_refusals(change, code):
    refused(code, **change)


def test_workspaces():
    good = (1, 2, 4, 2, 1, 4, 900, 9, 4, 2, 64)
    need = exe.exe_op_prefix_attention_paged_workspace(*good)
    assert need > 0
    refused(-1, ws_bytes=need - 1)
    refused(-1, ws=P + 8)
    refused(-1, ws=None, ws_bytes=None)
    for i, v in ((0, 2), (1, 0), (2, 0), (3, 0), (4, -1), (5, 0), (6, -1), (7, 0), (8, 3), (8, 0), (9, 0), (10, 96), (2, 1 << 30)):
        assert exe.exe_op_prefix_attention_paged_workspace(*good[:i], v, *good[i + 1:]) == 0
    assert exe.exe_op_prefix_attention_paged_workspace(1, 2, 4, 2, 0, 0, 0, 900, 4, 2, 64) > 0
    assert exe.exe_op_prefix_attention_paged_workspace(1, 2, 4, 2, 1, 4, 30, 9, 4, 2, 64) == 0          # few and short: one kernel


def test_nothing_to_do_is_no_error():
    none = dict.fromkeys(("cu", "cu_groups", "prefix", "q", "kv_blocks", "table", "length", "out"))
    for change in (dict(T=0), dict(n_seqs=0), dict(T=0, max_new=0, max_group=0, max_prefix=0, max_own=0)):
        exe.exe_op_prefix_attention_paged(*{**GOOD, **none, **change}.values(), None, stream=1)
