"""What norms of heads and log probabilities refuse, before anything of the device is touched (CPU)."""
import pytest

import paper_2404_07947_amd as exe

P = 4096            # an address that no call may follow
HEADS = dict(dtype=1, T=4, x=P, x_stride=256, heads=4, dh=64, rms=1, gain=P, gain_per_head=0, eps=1e-6, rot=64, interleaved=0, pos=P, inv_freq=P, amplitude=1.0, out=P,
             out_stride=256)
APPEND = dict(dtype=1, n_seqs=1, cu=P, T=4, qkv=P, row_stride=8 * 64, H=4, Hkv=2, dh=64, rms=1, q_gain=P, k_gain=P, gain_per_head=0, eps=1e-6, rot=64, interleaved=0,
              pos=None, inv_freq=P, amplitude=1.0, kv_blocks=P, n_blocks=4, table=P, max_blocks=2, block=16, length=P, q_out=2 * P, q_stride=4 * 64)
LOGPROBS = dict(dtype=0, logits=P, row_stride=100, rows=4, n=100, scale=1.0, tokens=P, n_tokens=1, logprobs=P, entropy=P, top_k=5, top_ids=P, top_logprobs=P)


def refused(fn, base, code, **change):
    with pytest.raises(exe.ExeError) as e:
        fn(*{**base, **change}.values(), stream=1)
    assert e.value.code == code, change


@pytest.mark.parametrize("change,code", [
    (dict(rms=2), -1), (dict(gain_per_head=-1), -1), (dict(eps=-1e-6), -1), (dict(eps=float("nan")), -1), (dict(eps=float("inf")), -1), (dict(rot=65), -2), (dict(rot=66), -2),
    (dict(rot=-2), -2), (dict(interleaved=2), -1), (dict(inv_freq=None), -1), (dict(dtype=2), -1), (dict(dh=96), -2), (dict(T=-1), -1)])
def test_what_both_norms_refuse(change, code):
    refused(exe.exe_op_head_norm_rotary, HEADS, code, **change)
    refused(exe.exe_op_head_norm_rotary_append_paged, APPEND, code, **change)


@pytest.mark.parametrize("change,code", [
    (dict(x=None), -1), (dict(out=None), -1), (dict(pos=None), -1), (dict(heads=0), -1), (dict(x_stride=255), -2), (dict(out_stride=255), -2), (dict(out=P, out_stride=300), -1),
    (dict(x=P + 1), -1), (dict(out=P + 1), -1), (dict(gain=P + 1), -1), (dict(heads=1 << 26, x_stride=1 << 40, out_stride=1 << 40), -2)])
def test_head_norm_refusals(change, code):
    refused(exe.exe_op_head_norm_rotary, HEADS, code, **change)


@pytest.mark.parametrize("change,code", [
    (dict(qkv=None), -1), (dict(H=-1), -1), (dict(row_stride=511), -2), (dict(q_stride=255), -2), (dict(qkv=P + 1), -1), (dict(q_out=P + 1), -1), (dict(qkv=P, q_out=P, q_stride=256), -1),
    (dict(q_gain=P + 1), -1), (dict(k_gain=P + 1), -1), (dict(H=1 << 26, row_stride=1 << 40, q_stride=1 << 40), -2), (dict(Hkv=0), -1), (dict(n_blocks=0), -1), (dict(max_blocks=0), -1),
    (dict(block=12), -1), (dict(n_seqs=-1), -1), (dict(cu=None), -1), (dict(kv_blocks=None), -1), (dict(kv_blocks=P + 8), -1), (dict(table=None), -1), (dict(length=None), -1)])
def test_append_refusals(change, code):
    refused(exe.exe_op_head_norm_rotary_append_paged, APPEND, code, **change)


@pytest.mark.parametrize("change,code", [
    (dict(dtype=2), -1), (dict(rows=-1), -1), (dict(n=0), -1), (dict(n_tokens=-1), -1), (dict(top_k=-1), -2), (dict(top_k=65), -2), (dict(n=4, top_k=5), -2), (dict(scale=0.0), -1),
    (dict(scale=-1.0), -1), (dict(scale=float("nan")), -1), (dict(scale=float("inf")), -1), (dict(scale=2.4e38), -1), (dict(row_stride=99), -2), (dict(logits=None), -1), (dict(tokens=None), -1),
    (dict(logprobs=None), -1), (dict(top_ids=None), -1), (dict(top_logprobs=None), -1), (dict(logits=P + 2), -1), (dict(dtype=1, logits=P + 1), -1), (dict(n=200000, row_stride=200000), -1)])
def test_logprob_refusals(change, code):
    refused(exe.exe_op_logprobs, LOGPROBS, code, **change)


def test_workspaces():
    need = exe.exe_op_logprobs_workspace(0, 3, 200000, 5)
    assert need > 0 and exe.exe_op_logprobs_workspace(0, 3, 100, 5) == 0
    for ws, size in ((P, need - 1), (P + 8, need)):
        with pytest.raises(exe.ExeError):
            exe.exe_op_logprobs(*{**LOGPROBS, "n": 200000, "row_stride": 200000, "rows": 3}.values(), ws, stream=1, ws_bytes=size)
    with pytest.raises(AssertionError):
        exe.exe_op_logprobs(*{**LOGPROBS, "n": 200000, "row_stride": 200000, "rows": 3}.values(), P, stream=1)
    good = (0, 3, 200000, 5)
    for i, v in ((0, 2), (1, 0), (1, -1), (2, 0), (3, -1), (3, 65)):
        assert exe.exe_op_logprobs_workspace(*good[:i], v, *good[i + 1:]) == 0
    # sizes do not shrink where rows begin on single elements, or rows and tokens are more
    assert exe.exe_op_logprobs_workspace(1, 1, 2 ** 31 - 1, 64) >= exe.exe_op_logprobs_workspace(1, 1, 2 ** 31 - 1, 0) > 0


def test_nothing_to_do_is_no_error():
    exe.exe_op_head_norm_rotary(*{**HEADS, "T": 0, "x": None, "out": None, "pos": None}.values(), stream=1)
    exe.exe_op_head_norm_rotary_append_paged(*{**APPEND, "T": 0}.values(), stream=1)
    exe.exe_op_head_norm_rotary_append_paged(*{**APPEND, "n_seqs": 0, "cu": None, "qkv": None}.values(), stream=1)
    exe.exe_op_logprobs(*{**LOGPROBS, "rows": 0, "logits": None}.values(), stream=1)
