"""The sines and cosines of rotary positions alone, against 64 bits."""
import pytest
import torch

import paper_2404_07947_amd as exe

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("interleaved", [0, 1])
def test_sines_and_cosines(interleaved):
    """2^22 angles of up to 2^16 radians.  What is left of an angle, an eighth of a turn at most, is rounded to float, by 2^-28 turns at most,
    2 pi 2^-28 radians; a sine or cosine of it is off by 2 steps of 2^-24 (two units in the last place of numbers below 1) at most.  The 64-bit
    side: positions times frequencies are off by 2^16 * 2^-53 at most."""
    T, dh = 1 << 16, 128
    g = torch.Generator(device="cuda:0").manual_seed(3)
    pos = torch.randint(-(1 << 16), 1 << 16, (T,), generator=g, device="cuda:0", dtype=torch.int32)
    f = torch.rand(dh // 2, generator=g, device="cuda:0", dtype=torch.float64)
    x = torch.zeros((T, dh), device="cuda:0")
    one = x[:, 0::2] if interleaved else x[:, :dh // 2]
    one.fill_(1.0)                                              # pairs (1, 0) become (cos, sin)
    out = torch.empty_like(x)
    exe.exe_op_rotary(0, T, x, dh, 1, dh, dh, interleaved, pos, f, 1.0, out, dh)
    got = (out[:, 0::2], out[:, 1::2]) if interleaved else (out[:, :dh // 2], out[:, dh // 2:])
    angle = pos.double()[:, None] * f[None]
    bound = 2 * 3.141592653589793 * 2.0 ** -28 + 2 * 2.0 ** -24 + 2.0 ** -36
    for a, want in zip(got, (angle.cos(), angle.sin())):
        off = float((a.double() - want).abs().max())
        assert off <= bound, off
