"""What the operations on a paged cache refuse, before anything of the device is touched, and the rotary frequencies (CPU)."""
import ctypes as C

import numpy as np
import pytest

import paper_2404_07947_amd as exe

P = 4096            # an address that no call may follow

APPEND = dict(dtype=1, n_seqs=1, cu=P, T=4, qkv=P, row_stride=8 * 64, H=4, Hkv=2, dh=64, rot=64, interleaved=0, pos=None, inv_freq=P, amplitude=1.0,
              kv_blocks=P, n_blocks=4, table=P, max_blocks=2, block=16, length=P, q_out=P, q_stride=4 * 64)
ATTEND = dict(dtype=1, n_seqs=1, cu=P, T=4, max_new=4, q=P, q_stride=4 * 64, kv_blocks=P, n_blocks=4, table=P, max_blocks=2, block=16, length=P,
              max_len=32, H=4, Hkv=2, dh=64, scale=0.1, window=0, out=P, out_stride=4 * 64)
ROTARY = dict(dtype=1, T=4, x=P, x_stride=256, heads=4, dh=64, rot=64, interleaved=0, pos=P, inv_freq=P, amplitude=1.0, out=2 * P, out_stride=256)
COPY = dict(dtype=1, pool=P, layers=2, n_blocks=8, block=16, Hkv=2, dh=64, copies=[(0, 1, 16)])


def refused(fn, base, code, **change):
    with pytest.raises(exe.ExeError) as e:
        fn(*{**base, **change}.values(), stream=1)
    assert e.value.code == code, change


@pytest.mark.parametrize("change,code", [
    (dict(dtype=2), -1), (dict(dh=96), -2), (dict(Hkv=0), -1), (dict(n_blocks=0), -1), (dict(max_blocks=0), -1), (dict(block=12), -1), (dict(block=4), -1),
    (dict(block=8192), -1), (dict(block=0), -1), (dict(block=-16), -1), (dict(n_seqs=-1), -1), (dict(T=-1), -1), (dict(cu=None), -1), (dict(kv_blocks=None), -1), (dict(table=None), -1),
    (dict(length=None), -1), (dict(kv_blocks=P + 8), -1)])
def test_what_both_refuse(change, code):
    refused(exe.exe_op_rotary_append_paged, APPEND, code, **change)
    refused(exe.exe_op_chunk_attention_paged, ATTEND, code, **change)


@pytest.mark.parametrize("change,code", [
    (dict(qkv=None), -1), (dict(inv_freq=None), -1), (dict(rot=65), -2), (dict(rot=-2), -2), (dict(rot=66), -2), (dict(interleaved=2), -1), (dict(H=-1), -1),
    (dict(row_stride=511), -2), (dict(H=1 << 26, row_stride=1 << 40, q_stride=1 << 40), -2), (dict(q_stride=255), -2), (dict(qkv=P + 1), -1), (dict(q_out=P + 1), -1), (dict(qkv=P, q_out=P, q_stride=256), -1)])
def test_append_refusals(change, code):
    refused(exe.exe_op_rotary_append_paged, {**APPEND, "q_out": 2 * P}, code, **change)


@pytest.mark.parametrize("change,code", [
    (dict(q=None), -1), (dict(out=None), -1), (dict(max_new=0), -1), (dict(max_len=0), -1), (dict(window=-1), -1), (dict(H=3), -2), (dict(H=1), -2),
    (dict(q_stride=255), -2), (dict(q_stride=257), -2), (dict(T=1 << 30), -2), (dict(out_stride=252), -2), (dict(q=P + 4), -1), (dict(out=P + 2), -1)])
def test_attention_refusals(change, code):
    refused(exe.exe_op_chunk_attention_paged, ATTEND, code, **change)


@pytest.mark.parametrize("change,code", [
    (dict(dtype=-1), -1), (dict(T=-1), -1), (dict(x=None), -1), (dict(out=None), -1), (dict(pos=None), -1), (dict(inv_freq=None), -1), (dict(heads=0), -1), (dict(dh=32), -2),
    (dict(rot=3), -2), (dict(rot=66), -2), (dict(interleaved=-1), -1), (dict(x_stride=255), -2), (dict(out_stride=255), -2), (dict(out=P, out_stride=300), -1),
    (dict(x=P + 1), -1), (dict(out=P + 1), -1), (dict(heads=1 << 26, x_stride=1 << 40, out_stride=1 << 40), -2)])
def test_rotary_refusals(change, code):
    refused(exe.exe_op_rotary, ROTARY, code, **change)


@pytest.mark.parametrize("change,code", [
    (dict(pool=None), -1), (dict(pool=P + 4), -1), (dict(dtype=7), -1), (dict(layers=0), -1), (dict(n_blocks=0), -1), (dict(block=20), -1), (dict(dh=80), -2), (dict(Hkv=0), -1),
    (dict(copies=[(8, 1, 2)]), -1), (dict(copies=[(-1, 1, 2)]), -1), (dict(copies=[(0, 8, 2)]), -1), (dict(copies=[(0, -1, 2)]), -1), (dict(copies=[(0, 1, 17)]), -5),
    (dict(copies=[(0, 1, -1)]), -5), (dict(copies=[(0, 1, 2), (3, 1, 2)]), -1), (dict(copies=[(0, 1, 2), (1, 2, 2)]), -1), (dict(copies=[(0, 0, 2)]), -1),
    (dict(copies=[(0, 1, 1)] * 9), -1), (dict(Hkv=1 << 20, block=4096), -2)])
def test_copy_refusals(change, code):
    refused(exe.exe_op_kv_copy_blocks, COPY, code, **change)


def test_nothing_to_do_is_no_error():
    exe.exe_op_chunk_attention_paged(*{**ATTEND, "T": 0}.values(), stream=1)
    exe.exe_op_chunk_attention_paged(*{**ATTEND, "n_seqs": 0}.values(), stream=1)
    exe.exe_op_rotary_append_paged(*{**APPEND, "T": 0, "q_out": 2 * P}.values(), stream=1)
    exe.exe_op_rotary(*{**ROTARY, "T": 0}.values(), stream=1)
    exe.exe_op_kv_copy_blocks(*{**COPY, "copies": []}.values(), stream=1)


def test_workspace_of_bad_arguments_is_none():
    good = (1, 4, 8, 2, 5000, 8, 2, 128, 0)
    for i, v in ((0, 2), (7, 96), (1, 0), (2, 0), (3, 0), (4, 0), (5, 0), (5, 3), (6, 0), (6, -1), (8, -1)):
        assert exe.exe_op_chunk_attention_paged_workspace(*good[:i], v, *good[i + 1:]) == 0


def test_fork_of_no_model():
    assert exe.lib().exe_seq_fork(None, 0, 0, None) == -1


@pytest.mark.parametrize("rot", [2, 32, 64, 100, 128])
def test_frequencies(rot):
    i = np.arange(rot // 2)
    plain = 10000.0 ** (-2.0 * i / rot)
    close = lambda a, b: np.testing.assert_allclose(a, b, rtol=1e-14)
    f, a = exe.exe_rotary_frequencies(rot)
    close(f, plain)
    assert a == 1.0
    f, a = exe.exe_rotary_frequencies(rot, scaling=exe.ROPE_LINEAR, factor=4.0)
    close(f, plain / 4)
    assert a == 1.0
    if rot > 2:
        f, a = exe.exe_rotary_frequencies(rot, scaling=exe.ROPE_BASE, factor=8.0)
        np.testing.assert_allclose([f[0], f[-1]], [1.0, plain[-1] / 8], rtol=1e-13)      # the fastest left, the slowest divided
        assert a == 1.0
    f, a = exe.exe_rotary_frequencies(rot, base=500000.0, scaling=exe.ROPE_RAMP, factor=8.0, original_positions=8192, turns_slow=1.0, turns_fast=4.0)
    plain = 500000.0 ** (-2.0 * i / rot)
    turns = 8192 * plain / (2 * np.pi)
    keep = np.clip((turns - 1) / 3, 0, 1)
    close(f, plain * keep + plain / 8 * (1 - keep))
    assert a == np.float32(0.1 * np.log(8.0) + 1)


@pytest.mark.parametrize("kw", [dict(rot=0), dict(rot=3), dict(rot=130), dict(rot=-2), dict(rot=64, base=0.0), dict(rot=64, base=float("inf")), dict(rot=64, base=float("nan")),
                                dict(rot=64, scaling=4), dict(rot=64, scaling=-1), dict(rot=64, scaling=1, factor=0.0), dict(rot=64, scaling=1, factor=float("nan")),
                                dict(rot=2, scaling=2, factor=2.0), dict(rot=64, scaling=3, factor=2.0, original_positions=0),
                                dict(rot=64, scaling=3, factor=2.0, original_positions=10, turns_slow=3.0, turns_fast=3.0)])
def test_frequency_refusals(kw):
    with pytest.raises(exe.ExeError) as e:
        exe.exe_rotary_frequencies(**kw)
    assert e.value.code == -1
    assert exe.lib().exe_rotary_frequencies(64, C.c_double(1e4), 0, C.c_double(1), 0, C.c_double(1), C.c_double(2), None, None) == -1


def test_tensors_of_the_host_are_refused():
    torch = pytest.importorskip("torch")
    x = torch.zeros((4, 256), dtype=torch.bfloat16)
    f = torch.zeros(32, dtype=torch.float64)
    pos = torch.zeros(4, dtype=torch.int32)
    for change in (dict(x=x), dict(out=x), dict(pos=pos), dict(inv_freq=f)):
        with pytest.raises(AssertionError):
            exe.exe_op_rotary(*{**ROTARY, **change}.values(), stream=1)
    with pytest.raises(AssertionError):
        exe.exe_op_kv_copy_blocks(*{**COPY, "pool": x}.values(), stream=1)
    with pytest.raises(AssertionError):
        exe.exe_op_chunk_attention_paged(*{**ATTEND, "table": pos}.values(), stream=1)


def test_results_over_the_queries_are_refused():
    with pytest.raises(exe.ExeError, match="cannot be the same"):
        exe.exe_op_chunk_attention_paged(*ATTEND.values(), stream=1)


def test_rows_whose_elements_no_int_counts_are_refused():
    refused(exe.exe_op_chunk_attention_paged, {**ATTEND, "out": 2 * P}, -2, T=1, H=1 << 26, q_stride=1 << 40, out_stride=1 << 40)


def test_tensors_that_hold_less_than_they_show_are_refused(monkeypatch):
    torch = pytest.importorskip("torch")
    from paper_2404_07947_amd import binding
    monkeypatch.setattr(binding, "_torch", torch)
    host = -1                                       # a host tensor's device number
    one = torch.zeros(1, 64)
    assert binding._rows(one.repeat(8, 1), host, 0, 8, 64, 64)
    assert binding._rows(torch.zeros(8, 128)[:, 64:], host, 0, 8, 64, 128)
    with pytest.raises(AssertionError):             # 8 rows to look at, memory of one
        binding._rows(one.expand(8, 64), host, 0, 8, 64, 64)
    with pytest.raises(AssertionError):             # the last row ends behind the memory
        binding._rows(torch.zeros(8, 128)[:, 64:], host, 0, 8, 65, 128)


def test_streams_and_workspaces_of_another_device_are_refused(monkeypatch):
    torch = pytest.importorskip("torch")
    from paper_2404_07947_amd import binding
    monkeypatch.setattr(binding, "_torch", torch)
    monkeypatch.setattr(binding, "_current", lambda: (0, None))

    class Other:
        device_index, cuda_stream = 1, 7

    class Own:
        device_index, cuda_stream = 0, 7

    assert binding._where(Own()) == (0, 7)
    with pytest.raises(AssertionError):
        binding._where(Other())
    with pytest.raises(AssertionError):
        exe.exe_op_chunk_attention_paged(*{**ATTEND, "out": 2 * P}.values(), workspace=torch.zeros(16), stream=1)
