"""Rotary positions and the append of a chunk's keys and values, against 64 bits."""
import numpy as np
import pytest
import torch

import paper_2404_07947_amd as exe
from chunk_util import DEV, HALF, TYPES, Batch, turned

pytestmark = pytest.mark.gpu


def rotate(x, heads, dh, rot, interleaved, pos, f, amplitude, out=None):
    code = 0 if x.dtype == torch.float32 else 1
    out = torch.full_like(x, 7.0) if out is None else out
    exe.exe_op_rotary(code, x.shape[0], x, x.stride(0), heads, dh, rot, interleaved, pos, f, amplitude, out, out.stride(0))
    return out


def close(got, want, err, dtype):
    got = got.cpu().double()
    assert bool(((got - want).abs() <= err + HALF[dtype] * want.abs() * (1 + 1e-6) + 1e-30).all()), float(((got - want).abs() - err).max())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("interleaved", [0, 1])
@pytest.mark.parametrize("dh,rot", [(64, 64), (64, 32), (64, 0), (64, 2), (128, 128), (128, 64), (128, 70), (128, 126), (64, 24)])
def test_rotary(dtype, interleaved, dh, rot):
    for T, heads in ((1, 1), (3, 5), (130, 2), (1000, 48)):
        g = torch.Generator().manual_seed(T)
        x = torch.randn((T, heads * dh), generator=g).to(TYPES[dtype][1])
        pos = torch.randint(-5, 1 << 20, (T,), generator=g, dtype=torch.int32)
        f = torch.as_tensor(exe.exe_rotary_frequencies(rot)[0]) if rot else torch.zeros(0, dtype=torch.float64)
        d = x.to(DEV)
        got = rotate(d, heads, dh, rot, interleaved, pos.to(DEV), f.to(DEV), 1.2)
        y, e = turned(x.view(T, heads, dh), pos, f, np.float32(1.2), rot, interleaved)
        close(got, y.flatten(1), e.flatten(1), dtype)
        rest = got.cpu().view(T, heads, dh)[..., rot:]
        assert torch.equal(rest, x.view(T, heads, dh)[..., rot:])          # passed through bit by bit
        assert torch.equal(rotate(d, heads, dh, rot, interleaved, pos.to(DEV), f.to(DEV), 1.2, out=d), got)      # in place


@pytest.mark.parametrize("pos", [0, 1, -1, 1 << 24, (1 << 31) - 1, -(1 << 31)])
def test_far_positions_keep_their_angles(pos):
    """Against integer arithmetic: the angle of a frequency of 2 pi * k / 2^20 radians, k odd, is k * pos mod 2^20 of 2^20 parts of a turn."""
    k = np.arange(1, 129, 2)
    f = torch.as_tensor(2 * np.pi * k / 2.0 ** 20)
    x = torch.zeros((1, 128), dtype=torch.float32)
    x[0, :64] = 1.0
    got = rotate(x.to(DEV), 1, 128, 128, 0, torch.tensor([pos], dtype=torch.int32, device=DEV), f.to(DEV), 1.0).cpu().double()[0]
    part = (k.astype(object) * pos) % (1 << 20)
    angle = torch.as_tensor(np.array(part, dtype=np.float64) / 2.0 ** 20 * 2 * np.pi)
    # the frequency itself is rounded to 64 bits: 2^-53 of the angle
    off = abs(pos) * float(f.max()) * 2.0 ** -52 + 4 * 2.0 ** -24
    assert float((got[:64] - angle.cos()).abs().max()) <= off and float((got[64:] - angle.sin()).abs().max()) <= off


def test_strides_and_alignments():
    """Rows that begin anywhere: every start and stride of single elements, in front of and behind what is left alone."""
    for dtype in ("f32", "bf16"):
        t = TYPES[dtype][1]
        for start in (0, 1, 3, 8):
            for extra in (0, 1, 8):
                T, heads, dh, rot = 5, 3, 64, 64
                w = heads * dh
                buf = torch.randn((T * (w + extra) + start,), generator=torch.Generator().manual_seed(start)).to(t)
                x = torch.as_strided(buf, (T, w), (w + extra, 1), start)
                d = buf.to(DEV)
                dx = torch.as_strided(d, (T, w), (w + extra, 1), start)
                pos = torch.arange(T, dtype=torch.int32, device=DEV) * 77
                f = torch.as_tensor(exe.exe_rotary_frequencies(rot)[0], device=DEV)
                for il in (0, 1):
                    y, e = turned(x.reshape(T, heads, dh), pos.cpu(), f.cpu(), 1.0, rot, il)
                    o = torch.full((T * (w + 5) + 2,), 7.0, dtype=t, device=DEV)
                    exe.exe_op_rotary(TYPES[dtype][0], T, dx, w + extra, heads, dh, rot, il, pos, f, 1.0, o[1:], w + 5)
                    got = torch.as_strided(o, (T, w), (w + 5, 1), 1)
                    close(got, y.flatten(1), e.flatten(1), dtype)
                    left = o.clone()
                    torch.as_strided(left, (T, w), (w + 5, 1), 1).fill_(7.0)
                    assert bool((left == 7).all())


@pytest.mark.parametrize("interleaved", [0, 1])
def test_gradient_is_the_call_at_negated_positions(interleaved):
    """The transpose of the turn: against the formula's gradient and against differences."""
    T, heads, dh, rot, amplitude = 6, 2, 64, 48, 1.25
    g = torch.Generator().manual_seed(3)
    x, dy = torch.randn((T, heads * dh), generator=g), torch.randn((T, heads * dh), generator=g)
    pos = torch.randint(0, 5000, (T,), generator=g, dtype=torch.int32)
    f = torch.as_tensor(exe.exe_rotary_frequencies(rot)[0])
    got = rotate(dy.to(DEV), heads, dh, rot, interleaved, (-pos).to(DEV), f.to(DEV), amplitude).cpu().double()
    xr = x.double().requires_grad_(True)
    y, e = turned(xr.view(T, heads, dh), pos, f, amplitude, rot, interleaved)
    (want,) = torch.autograd.grad((y.flatten(1) * dy.double()).sum(), xr)
    _, e = turned(dy.view(T, heads, dh), pos, f, amplitude, rot, interleaved)
    close(got, want, e.flatten(1), "f32")
    # a turn is linear: a difference along a direction is exact but for the roundings of both sides
    v = torch.randn((T, heads * dh), generator=g)
    up = rotate((x + v).to(DEV), heads, dh, rot, interleaved, pos.to(DEV), f.to(DEV), amplitude).cpu().double()
    dn = rotate((x - v).to(DEV), heads, dh, rot, interleaved, pos.to(DEV), f.to(DEV), amplitude).cpu().double()
    slope = float(((up - dn) / 2 * dy.double()).sum())
    size = float((amplitude * 2 * (x.abs() + v.abs()).double() * 2 * dy.abs().double()).sum())
    assert abs(slope - float((got * v.double()).sum())) <= 16 * 2.0 ** -24 * size


def append(b, qkv, rot, interleaved, pos, f, amplitude, q_out, stride=None, q_stride=None):
    exe.exe_op_rotary_append_paged(b.code, len(b.seqs), b.d_cu, b.rows, qkv, stride or qkv.shape[1], b.H, b.Hkv, b.dh, rot, interleaved, pos, f, amplitude,
                                   b.d_pool, b.n_blocks, b.d_table, b.max_blocks, b.block, b.d_len, q_out, q_stride or b.H * b.dh)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("interleaved", [0, 1])
@pytest.mark.parametrize("H,Hkv,dh,rot,block", [(4, 4, 64, 64, 8), (8, 2, 128, 128, 16), (5, 1, 128, 64, 4096), (3, 3, 64, 0, 16), (6, 2, 128, 90, 64)])
def test_append(dtype, interleaved, H, Hkv, dh, rot, block):
    for seqs in ([(1, 1)], [(1, 9), (0, 4), (1, 64), (40, 65), (0, 0), (3, 3)], [(1, 17 * i + 1) for i in range(70)] + [(300, 333)]):
        b = Batch(seqs, H, Hkv, dh, block, dtype, extra_rows=2).fill().device()
        g = torch.Generator().manual_seed(5)
        qkv = torch.randn((b.rows, (H + 2 * Hkv) * dh), generator=g).to(b.t)
        f = torch.as_tensor(exe.exe_rotary_frequencies(rot, scaling=exe.ROPE_RAMP, factor=4.0, original_positions=100)[0]) if rot else torch.zeros(1, dtype=torch.float64)
        before = b.d_pool.clone()
        for pos in (None, torch.randint(0, 100000, (b.rows,), generator=g, dtype=torch.int32)):
            q_out = torch.full((b.rows, H * dh), 7.0, dtype=b.t, device=DEV)
            b.d_pool.copy_(before)
            append(b, qkv.to(DEV), rot, interleaved, None if pos is None else pos.to(DEV), f.to(DEV), 1.1, q_out)
            at = torch.cat([torch.arange(L - n, L) for n, L in seqs]) if pos is None else pos[:b.T]
            x = qkv[:b.T].view(b.T, H + 2 * Hkv, dh)
            y, e = turned(x[:, :H + Hkv], at, f[:rot // 2], np.float32(1.1), rot, interleaved)
            close(q_out[:b.T], y[:, :H].flatten(1), e[:, :H].flatten(1), dtype)
            assert bool((q_out[b.T:] == 7).all())
            after, want = b.d_pool.cpu(), before.cpu()
            t = 0
            for s, (n, L) in enumerate(seqs):
                for p in range(L - n, L):
                    blk, row = int(b.table[s, p // block]), p % block
                    close(after[blk, 0, :, row], y[t, H:], e[t, H:], dtype)
                    assert torch.equal(after[blk, 1, :, row], x[t, H + Hkv:])
                    want[blk, :, :, row] = after[blk, :, :, row]
                    t += 1
            assert torch.equal(torch.nan_to_num(after, nan=99.0), torch.nan_to_num(want, nan=99.0))      # nothing else moved


def test_append_in_place_without_queries_and_unaligned():
    b = Batch([(3, 20), (1, 5)], 4, 2, 64, 16, "bf16").fill().device()
    f = torch.as_tensor(exe.exe_rotary_frequencies(64)[0], device=DEV)
    qkv = torch.randn((4, 8 * 64), generator=torch.Generator().manual_seed(1)).bfloat16().to(DEV)
    q_out = torch.empty((4, 256), dtype=torch.bfloat16, device=DEV)
    append(b, qkv, 64, 0, None, f, 1.0, q_out)
    pool = b.d_pool.clone()
    b.d_pool.fill_(3.0)
    append(b, qkv, 64, 0, None, f, 1.0, None)                              # keys and values only
    rows = [(0, p) for p in (17, 18, 19)] + [(1, 4)]
    at = lambda t: torch.stack([t[int(b.table[s, p // 16]), :, :, p % 16] for s, p in rows])
    assert torch.equal(at(b.d_pool), at(pool)) and int((b.d_pool != 3).any(-1).sum()) == 4 * 4
    wide = torch.zeros((4, 8 * 64 + 3), dtype=torch.bfloat16, device=DEV)
    wide[:, 1:8 * 64 + 1] = qkv
    b.d_pool.fill_(3.0)
    append(b, wide[:, 1:], 64, 0, None, f, 1.0, wide[:, 1:], stride=8 * 64 + 3, q_stride=8 * 64 + 3)       # in place, odd rows
    assert torch.equal(at(b.d_pool), at(pool)) and torch.equal(wide[:, 1:257], q_out) and torch.equal(wide[:, 257:513], qkv[:, 256:])


@pytest.mark.parametrize("entry", [-1, 1 << 30, -(1 << 31), None])
def test_positions_without_a_block_are_not_stored(entry):
    b = Batch([(40, 60), (1, 10)], 4, 2, 64, 16, "bf16").fill()
    if entry is None:
        b.table, b.max_blocks = b.table[:, :2].copy(), 2
        lost = range(32, 60)
    else:
        b.table[0, 2] = entry
        lost = range(32, 48)
    b.device()
    b.d_len[1] = -3                                                         # and a token before position 0
    before = b.d_pool.clone()
    qkv = torch.randn((41, 8 * 64), generator=torch.Generator().manual_seed(1)).bfloat16().to(DEV)
    q_out = torch.full((41, 256), 7.0, dtype=torch.bfloat16, device=DEV)
    append(b, qkv, 0, 0, None, torch.zeros(1, dtype=torch.float64, device=DEV), 1.0, q_out)
    assert torch.equal(q_out, qkv[:, :256])
    changed = torch.zeros((b.n_blocks, 16), dtype=torch.bool)
    for p in range(20, 60):
        if p not in lost:
            changed[int(b.table[0, p // 16]), p % 16] = True
    same = ((b.d_pool == before) | (b.d_pool.isnan() & before.isnan())).all(-1).all(1).all(1).cpu()
    assert torch.equal(~same, changed)


def test_tensors_that_would_be_misread_are_refused():
    x = torch.zeros((4, 256), dtype=torch.bfloat16, device=DEV)
    pos, f = torch.zeros(4, dtype=torch.int32, device=DEV), torch.zeros(32, dtype=torch.float64, device=DEV)
    good = dict(dtype=1, T=4, x=x, x_stride=256, heads=4, dh=64, rot=64, interleaved=0, pos=pos, inv_freq=f, amplitude=1.0, out=x, out_stride=256)
    exe.exe_op_rotary(**good)
    for change in (dict(x=x.float(), out=x.float()), dict(dtype=0), dict(pos=pos.long()), dict(inv_freq=f.float()), dict(pos=pos[:3]), dict(inv_freq=f[:31]), dict(T=5, pos=torch.zeros(5, dtype=torch.int32, device=DEV)),
                   dict(x=x[:, 1:]), dict(pos=torch.zeros(8, dtype=torch.int32, device=DEV)[::2]), dict(x=x.cpu()), dict(pos=pos.cpu())):
        with pytest.raises(AssertionError):
            exe.exe_op_rotary(**{**good, **change})
