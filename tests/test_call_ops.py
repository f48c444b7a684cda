"""csrc/call.c's operations on tensors: every argument reaches the library's function in its place and type, and what the library would misread is refused.

A function of ctypes stands for the library's; CPU tensors and stand-ins with a device number stand for device tensors.
"""
import ctypes as C

import pytest
import torch

from paper_2404_07947_amd import binding

P, I, L, F, U = C.c_void_p, C.c_int32, C.c_int64, C.c_float, C.c_uint64
# the arguments behind the stream, as include/exe.h declares them; in the last one a workspace with its bytes
SIGNATURES = {
    "head_norm_rotary": [I, I, P, L, I, I, I, P, I, F, I, I, P, P, F, P, L],
    "head_norm_rotary_append_paged": [I, I, P, I, P, L, I, I, I, I, P, P, I, F, I, I, P, P, F, P, I, P, I, I, P, P, L],
    "prefix_attention_paged": [I, I, P, I, I, I, P, P, I, I, P, L, P, I, P, I, I, P, I, I, I, I, F, P, L, P, U],
    "logprobs": [I, P, L, I, I, F, P, I, P, P, I, P, P, P, U],
}


@pytest.fixture(scope="module")
def call():
    binding.lib()
    from paper_2404_07947_amd import _call
    _call.types(torch.float32, torch.bfloat16, torch.int32, torch.float64)
    return _call


def recorder(name, seen):
    return C.CFUNCTYPE(I, P, *SIGNATURES[name])(lambda *a: seen.append(a) or 0)


class OnDevice:
    """A tensor that says it lies on device 3."""

    def __init__(self, t):
        self.t = t

    def get_device(self):
        return 3

    def __getattr__(self, name):
        return getattr(self.t, name)


@pytest.mark.parametrize("name", SIGNATURES)
def test_places_and_types(call, name):
    seen = []
    f = recorder(name, seen)
    kinds = SIGNATURES[name]
    given = [{P: 0x7fff00000000 + 16 * i, I: 100 + i, L: (1 << 40) + i, U: (1 << 41) + i, F: 0.25 * i}[k] for i, k in enumerate(kinds)]
    assert getattr(call, name)(C.cast(f, P).value, None, 0x1230, *given) == 0
    assert seen == [(0x1230, *given)]
    given = [None if k is P else 0 for k in kinds]
    assert getattr(call, name)(C.cast(f, P).value, None, None, *given) == 0
    assert seen[1] == (None, *given)


@pytest.mark.parametrize("name", SIGNATURES)
def test_numbers_are_not_cut(call, name):
    f = recorder(name, [])
    kinds = SIGNATURES[name]
    for i, k in enumerate(kinds):
        given = [None if k is P else 0 for k in kinds]
        for bad, error in {I: [(1 << 31, OverflowError), (-(1 << 31) - 1, OverflowError), (1.5, TypeError), (None, TypeError)], L: [(1 << 63, OverflowError), ("1", TypeError)],
                           U: [(1 << 64, OverflowError)], F: [("x", TypeError)], P: [(1 << 64, OverflowError)]}[k]:
            given[i] = bad
            with pytest.raises(error):
                getattr(call, name)(C.cast(f, P).value, None, None, *given)
    for count in (len(kinds) - 1, len(kinds) + 1):
        with pytest.raises(TypeError):
            getattr(call, name)(C.cast(f, P).value, None, None, *[0] * count)


def norm_args(x, gain=None, pos=None, freq=None, out=None, T=4, heads=2, dh=64, stride=128, dtype=0, rot=0, per_head=0):
    return [dtype, T, x, stride, heads, dh, 1, gain, per_head, 1e-5, rot, 0, pos, freq, 1.0, out, stride]


def test_tensors(call):
    seen = []
    f = recorder("head_norm_rotary", seen)

    def run(dev, **a):
        return call.head_norm_rotary(C.cast(f, P).value, dev, None, *norm_args(**a))

    x = torch.zeros(4, 128)
    on = OnDevice(x)
    assert run(3, x=on, out=on, gain=OnDevice(x[0, :64]), pos=OnDevice(torch.zeros(4, dtype=torch.int32)), freq=OnDevice(torch.zeros(32, dtype=torch.float64)), rot=64) == 0
    assert seen[0][3] == x.data_ptr() and seen[0][17 - 1] == x.data_ptr()
    # a view between wider rows, whose last row ends with the storage; one element further on is beyond it
    wide = torch.zeros(4 * 192)
    assert run(3, x=OnDevice(wide[64:]), stride=192) == 0 and seen[1][3] == wide.data_ptr() + 256
    assert run(3, x=OnDevice(wide.view(4, 192)[:, 64:]), stride=192) == 0 and seen[2][3] == wide.data_ptr() + 256
    assert run(3, x=OnDevice(x[:0]), T=0) == 0                                # no rows
    n = len(seen)
    for dev, a in [
        (2, dict(x=on)),                                                      # another device
        (None, dict(x=on)),                                                   # no device
        (None, dict(x=x)), (-1, dict(x=x)),                                   # host memory
        (3, dict(x=x)),
        (3, dict(x=on, dtype=1)), (3, dict(x=OnDevice(x.bfloat16()))), (3, dict(x=OnDevice(x.double()))),
        (3, dict(x=on, T=5)), (3, dict(x=on, stride=129)), (3, dict(x=OnDevice(wide[65:]), stride=192)),
        (3, dict(x=on, out=OnDevice(x[:3].clone()))),
        (3, dict(x=on, gain=OnDevice(x[0, :63]))), (3, dict(x=on, gain=OnDevice(x[:, 0].expand(4)))), (3, dict(x=on, gain=OnDevice(x[0, :64]), per_head=1)),
        (3, dict(x=on, gain=OnDevice(torch.zeros(128)[::2]))),                # elements that do not follow each other
        (3, dict(x=on, pos=OnDevice(torch.zeros(3, dtype=torch.int32)))), (3, dict(x=on, pos=OnDevice(torch.zeros(4, dtype=torch.int64)))),
        (3, dict(x=on, freq=OnDevice(torch.zeros(31, dtype=torch.float64)), rot=64)), (3, dict(x=on, freq=OnDevice(torch.zeros(32)), rot=64)),
        # counts whose product passes 64 bits
        (3, dict(x=on, T=2**31 - 1, stride=2**62)), (3, dict(x=on, heads=2**31 - 1, dh=2**31 - 1, stride=2**62)),
    ]:
        with pytest.raises(AssertionError):
            run(dev, **a)
    with pytest.raises(AttributeError):
        run(3, x="text")
    assert len(seen) == n


def test_workspaces(call):
    seen = []
    f = recorder("logprobs", seen)

    def run(ws, size):
        return call.logprobs(C.cast(f, P).value, 3, None, 0, None, 0, 0, 0, 1.0, None, 0, None, None, 0, None, None, ws, size)

    t = torch.zeros(10)
    for ws, size, want in [(None, None, (None, 0)), (None, 7, (None, 0)), (64, 7, (64, 7)), (OnDevice(t), None, (t.data_ptr(), 40)), (OnDevice(t), 24, (t.data_ptr(), 24)),
                           (OnDevice(t[4:]), 24, (t.data_ptr() + 16, 24))]:
        assert run(ws, size) == 0 and seen[-1][-2:] == want
    n = len(seen)
    for ws, size in [(64, None), (64, -1), (OnDevice(t), 41), (OnDevice(t), -1), (OnDevice(t[::2]), None), (t, None)]:
        with pytest.raises(AssertionError):
            run(ws, size)
    assert len(seen) == n
