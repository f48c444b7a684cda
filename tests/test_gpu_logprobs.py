"""Log probabilities of given tokens, entropy and the largest ones, against 64 bits."""
import math

import numpy as np
import pytest
import torch

import paper_2404_07947_amd as exe
import workload as wl
from chunk_util import DEV, TYPES, U

pytestmark = pytest.mark.gpu


def call(x, n, scale=1.0, tokens=None, k=0, entropy=True, stride=None, stream=None, ws=None):
    """x: device tensor, rows of x.shape[0] (or a flat one with `stride`)."""
    rows = x.shape[0]
    stride = x.stride(0) if stride is None else stride
    code = 0 if x.dtype == torch.float32 else 1
    m = 0 if tokens is None else tokens.shape[1]
    lp = torch.full((rows, m), 7.0, device=DEV) if m else None
    en = torch.full((rows,), 7.0, device=DEV) if entropy else None
    ids = torch.full((rows, k), -7, dtype=torch.int32, device=DEV) if k else None
    top = torch.full((rows, k), 7.0, device=DEV) if k else None
    if ws is None:
        ws = torch.full((max(16, exe.exe_op_logprobs_workspace(code, rows, n, k)) // 4,), float("nan"), device=DEV)
    exe.exe_op_logprobs(code, x, stride, rows, n, scale, tokens, m, lp, en, k, ids, top, ws, stream=stream)
    return lp, en, ids, top


def best(x, k):
    """The k largest above minus infinity, the lowest index on ties: ids, -1 where there are fewer."""
    x = x.double().numpy()
    out = np.full((len(x), k), -1, dtype=np.int32)
    for r, v in enumerate(x):
        i = np.flatnonzero(v > -math.inf)
        i = i[np.argsort(-v[i], kind="stable")][:k]
        out[r, :len(i)] = i
    return torch.as_tensor(out)


def check(x, scale, tokens, k, got):
    """The bound, with y = scale * (x - max): z is off by 2 half steps of float relative to itself (its factor's rounding and its own), 2^z by 2
    more; up to 80 additions one after the other or in trees; the logarithm and the products after it by 4 of their size.  So the sum's logarithm is off by
    (90 + 2 E|y|) half steps, where E is over the probabilities, and the entropy's sum by as much of E|y| and by 2 E y^2."""
    lp, en, ids, top = got
    x = x.double()
    y = (x - x.amax(-1, keepdim=True)) * float(np.float32(scale))
    p = torch.softmax(y, -1)
    L = torch.logsumexp(y, -1, keepdim=True)
    a = torch.where(p > 0, y.abs(), 0.0)
    e1, e2 = (p * a).sum(-1, keepdim=True), (p * a * a).sum(-1, keepdim=True)
    full = y - L
    tol = U * (96 + 2 * e1 + 6 * torch.where(y > -math.inf, y.abs(), 0.0) + 6 * L.abs())
    if lp is not None:
        t = tokens.long().cpu()
        assert bool(((lp.cpu().double() - full.gather(1, t)).abs() <= tol.gather(1, t)).logical_or(lp.cpu().double() == full.gather(1, t)).all())
    if en is not None:
        want = (L + e1)[:, 0]
        bound = U * (96 + 6 * L + 100 * e1 + 2 * e1 * e1 + 4 * e2)[:, 0]
        assert bool(((en.cpu().double() - want).abs() <= bound).all()), float(((en.cpu().double() - want).abs() - bound).max())
    if k:
        want = best(x, k)
        assert torch.equal(ids.cpu(), want)
        i = want.long().clamp_min(0)
        there = want >= 0
        off = (top.cpu().double() - full.gather(1, i)).abs() <= tol.gather(1, i)
        assert bool(torch.where(there, off, top.cpu() == -math.inf).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 2, 3, 63, 64, 255, 1000, 1024, 1025, 2047, 4096, 8191, 8192, 8193, 20011, 50272])
@pytest.mark.parametrize("rows", [1, 5, 130])
def test_sizes(dtype, n, rows):
    g = torch.Generator().manual_seed(n + rows)
    x = (torch.randn((rows, n), generator=g) * 2.5).to(TYPES[dtype][1])
    for k, m, scale in ((min(n, 20), 1, 1.0), (0, 3, 0.7), (min(n, 64), 0, 1.25), (1, 1, 2.0)):
        tokens = torch.randint(0, n, (rows, m), generator=g, dtype=torch.int32).to(DEV) if m else None
        check(x, scale, tokens, k, call(x.to(DEV), n, scale, tokens, k))


@pytest.mark.parametrize("dtype,rows,n", [("f32", 300, 8200), ("f32", 300, 50272), ("f32", 257, 53249), ("f32", 3, 53248), ("f32", 3, 53249), ("bf16", 300, 32768), ("bf16", 300, 32769),
                                          ("bf16", 2, 65536), ("bf16", 2, 65537), ("bf16", 200, 70001), ("bf16", 80, 70001)])
def test_launches(dtype, rows, n):
    """Each number of threads, one launch and two; rows on either side of what a workgroup holds."""
    g = torch.Generator().manual_seed(n)
    x = (torch.randn((rows, n), generator=g) * 2.5).to(TYPES[dtype][1])
    x[0], x[1, :n - 50] = 0.25, -math.inf
    tokens = torch.randint(n - 50, n, (rows, 1), generator=g, dtype=torch.int32).to(DEV)
    check(x, 1.0, tokens, 20, call(x.to(DEV), n, 1.0, tokens, 20))
    check(x[:3], 1.0, tokens[:3], 50, call(x[:3].to(DEV), n, 1.0, tokens[:3], 50))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [600000, 4300001])
def test_long_rows(dtype, n):
    """More than 64 parts a row, and more than 64 times as many."""
    g = torch.Generator().manual_seed(n)
    x = (torch.randn((2, n), generator=g) * 2.5).to(TYPES[dtype][1])
    tokens = torch.tensor([[0, n - 1], [n // 2, 5]], dtype=torch.int32, device=DEV)
    check(x, 1.0, tokens, 40, call(x.to(DEV), n, 1.0, tokens, 40))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("k", [1, 4, 20, 64])
@pytest.mark.parametrize("n", [300, 9000, 30000])
def test_ties_and_orders(dtype, k, n):
    """All equal; rising and falling; few values; the largest all in one place; 0 and -0; two values one step apart."""
    t = TYPES[dtype][1]
    i = torch.arange(n, dtype=torch.float32)
    g = torch.Generator().manual_seed(n)
    few = torch.randint(0, 3, (n,), generator=g).float()
    one = torch.zeros(n)
    one[n // 3:n // 3 + 200] = 5.0
    lane = torch.where((i / 4).floor() % 256 == 7, 9.0 + i / n, -i / n)
    zeros = torch.where(i % 3 == 0, -0.0, 0.0)
    step = torch.where(torch.rand(n, generator=g) < 0.5, 1.0, 1.0 + 2.0 ** -7)
    rows = [torch.full((n,), -3.25), i / n, -i / n, few, one, lane, zeros, step, -1e30 * few, (i * 7919 % n) / n]
    x = torch.stack(rows).to(t)
    tokens = torch.tensor([[0, n - 1]] * len(rows), dtype=torch.int32, device=DEV)
    check(x, 1.0, tokens, k, call(x.to(DEV), n, 1.0, tokens, k))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [500, 33000])
def test_ruled_out(dtype, n):
    """Minus infinity: half, all but a few (fewer than are asked for), all but one, whole stretches; never an alternative."""
    g = torch.Generator().manual_seed(n)
    x = torch.randn((6, n), generator=g).to(TYPES[dtype][1])
    keep = torch.rand((6, n), generator=g) < 0.5
    keep[1] = torch.arange(n) % (n // 9) == 3
    keep[2] = torch.arange(n) == n - 1
    keep[3] = torch.arange(n) < n // 2
    keep[4] = (torch.arange(n) // 4 % 256) < 60               # whole waves of the kernel without one
    keep[5] = torch.arange(n) >= n - 300
    x.masked_fill_(~keep, -math.inf)
    tokens = torch.stack([torch.tensor([int(r.nonzero()[0]), int((~r).nonzero()[0])]) for r in keep]).int().to(DEV)
    for k in (0, 5, 64):
        got = call(x.to(DEV), n, 1.3, tokens, k)
        check(x, 1.3, tokens, k, got)
        assert bool((got[0][:, 1] == -math.inf).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [700, 40000])
def test_rows_without_a_distribution(dtype, n):
    """NaN, plus infinity, nothing at all: NaN, alternatives by what is a number; the rows beside them as they are alone."""
    g = torch.Generator().manual_seed(1)
    x = torch.randn((7, n), generator=g).to(TYPES[dtype][1])
    tokens = torch.randint(0, n, (7, 2), generator=g, dtype=torch.int32).to(DEV)
    clean = call(x.to(DEV), n, 1.0, tokens, 10)
    x[1, n // 2], x[2, 3], x[3], x[4] = math.nan, math.inf, -math.inf, math.nan
    x[5, :n - 1] = math.nan
    lp, en, ids, top = call(x.to(DEV), n, 1.0, tokens, 10)
    for r in (0, 6):
        assert all(torch.equal(a[r], b[r]) for a, b in zip((lp, en, ids, top), clean))
    for r in (1, 2, 3, 4, 5):
        assert bool(lp[r].isnan().all()) and bool(en[r].isnan())
    assert int(ids[2, 0]) == 3 and torch.equal(ids.cpu()[1:3], best(torch.nan_to_num(x[1:3].float(), nan=-math.inf, posinf=1e38), 10))
    assert bool((ids[3:5] == -1).all()) and bool((top[3:5] == -math.inf).all())
    assert ids[5].tolist() == [n - 1] + [-1] * 9 and bool(top[5, 0].isnan())


def test_largest_numbers_and_scales():
    big = float(np.finfo(np.float32).max)
    x = torch.tensor([[big, -big, 0.0, big], [1e-45, 0.0, -1e-45, 1e-38], [88.0, -88.0, 1000.0, 999.0]])
    tokens = torch.tensor([[0, 1]] * 3, dtype=torch.int32, device=DEV)
    check(x, 0.5, tokens, 4, call(x.to(DEV), 4, 0.5, tokens, 4))
    y = x[1:]
    for scale in (1e-6, 30.0):
        check(y, scale, tokens[1:], 4, call(y.to(DEV), 4, scale, tokens[1:], 4))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strides_and_alignments(dtype):
    """Rows that begin anywhere, with NaN and infinities between them and in front of the first."""
    t = TYPES[dtype][1]
    for n, extra, start in ((5, 0, 1), (1000, 1, 0), (1001, 3, 5), (9001, 0, 7), (9001, 7, 0), (17, 8, 2)):
        rows = 4
        g = torch.Generator().manual_seed(n)
        buf = torch.full((start + rows * (n + extra) + 9,), math.inf).to(t)
        buf[::2] = math.nan
        v = torch.as_strided(buf, (rows, n), (n + extra, 1), start)
        v.copy_(torch.randn((rows, n), generator=g))
        d = buf.to(DEV)
        dv = torch.as_strided(d, (rows, n), (n + extra, 1), start)
        tokens = torch.randint(0, n, (rows, 1), generator=g, dtype=torch.int32).to(DEV)
        check(v.contiguous(), 1.0, tokens, min(n, 7), call(dv, n, 1.0, tokens, min(n, 7), stride=n + extra))


def test_tokens_that_are_none_are_not_looked_up():
    x = torch.randn((2, 100), generator=torch.Generator().manual_seed(1)).to(DEV)
    tokens = torch.tensor([[-1, 100, 5], [1 << 30, -(1 << 31), 99]], dtype=torch.int32, device=DEV)
    lp, _, _, _ = call(x, 100, 1.0, tokens)
    assert bool(lp[:, :2].isnan().all())
    assert torch.equal(lp[:, 2:], call(x, 100, 1.0, tokens[:, 2:].contiguous())[0])


def test_many_tokens_of_a_row():
    x = torch.randn((3, 5000), generator=torch.Generator().manual_seed(1))
    tokens = torch.randint(0, 5000, (3, 4001), generator=torch.Generator().manual_seed(2), dtype=torch.int32).to(DEV)
    check(x, 1.0, tokens, 0, call(x.to(DEV), 5000, 1.0, tokens))


def test_rows_do_not_depend_on_each_other_and_repeat():
    """A row alone, among others, and again: the same bits where the rows of both calls are cut alike; the first alternative is argmax's."""
    x = (torch.randn((300, 8000), generator=torch.Generator().manual_seed(1)) * 3).to(DEV)
    a = call(x, 8000, 1.0, None, 8)
    b = call(x[100:].contiguous(), 8000, 1.0, None, 8)
    for s, t in zip(a[1:], b[1:]):
        assert torch.equal(s[100:], t)
    for s, t in zip(a[1:], call(x, 8000, 1.0, None, 8)[1:]):
        assert torch.equal(s, t)
    m = torch.empty(300, dtype=torch.int32, device=DEV)
    exe.exe_op_argmax(x, 300, 8000, m)
    assert torch.equal(m, a[2][:, 0])


def test_rows_beyond_2_31_elements():
    stride = (1 << 30) + 8
    buf = torch.zeros(2 * stride + 2000, dtype=torch.bfloat16, device=DEV)
    x = torch.randn((3, 2000), generator=torch.Generator().manual_seed(2)).bfloat16()
    v = torch.as_strided(buf, (3, 2000), (stride, 1))
    v.copy_(x.to(DEV))
    tokens = torch.tensor([[1], [2], [1999]], dtype=torch.int32, device=DEV)
    check(x, 1.0, tokens, 5, call(v, 2000, 1.0, tokens, 5, stride=stride))


def test_two_streams_and_a_replayed_graph():
    """Two calls at once with a workspace each; a graph replayed with other logits, tokens among them, against eager calls."""
    xs = [(torch.randn((3, 60000), generator=torch.Generator().manual_seed(i)) * 3).to(DEV) for i in range(2)]
    want = [call(x, 60000, 1.0, None, 16) for x in xs]
    streams = [torch.cuda.Stream() for _ in xs]
    torch.cuda.synchronize()
    got = [None, None]
    for _ in range(3):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i] = call(xs[i], 60000, 1.0, None, 16)
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert all(torch.equal(a, b) for a, b in zip(g[1:], w[1:]))
    x, n, k = xs[0], 60000, 16
    tokens = torch.zeros((3, 2), dtype=torch.int32, device=DEV)
    ws = torch.empty(exe.exe_op_logprobs_workspace(0, 3, n, k), dtype=torch.uint8, device=DEV)
    out = (torch.empty((3, 2), device=DEV), torch.empty(3, device=DEV), torch.empty((3, k), dtype=torch.int32, device=DEV), torch.empty((3, k), device=DEV))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        exe.exe_op_logprobs(0, x, n, 3, n, 1.0, tokens, 2, out[0], out[1], k, out[2], out[3], ws)
    for step in range(5):
        x.copy_(torch.randn((3, n), generator=torch.Generator().manual_seed(50 + step)) * 3)
        tokens.fill_(step)
        graph.replay()
        torch.cuda.synchronize()
        replayed = [o.clone() for o in out]
        assert all(torch.equal(a, b) for a, b in zip(replayed, call(x, n, 1.0, tokens, k)))


def test_tensors_that_would_be_misread_are_refused():
    x = torch.zeros((4, 100), device=DEV)
    tok, f, ids = torch.zeros((4, 1), dtype=torch.int32, device=DEV), torch.zeros((4, 2), device=DEV), torch.zeros((4, 2), dtype=torch.int32, device=DEV)
    good = dict(dtype=0, logits=x, row_stride=100, rows=4, n=100, scale=1.0, tokens=tok, n_tokens=1, logprobs=f, entropy=f, top_k=2, top_ids=ids, top_logprobs=f)
    exe.exe_op_logprobs(**good)
    for change in (dict(logits=x.half()), dict(dtype=1), dict(tokens=tok.long()), dict(logprobs=f.double()), dict(entropy=f[0]), dict(top_ids=ids.long()), dict(rows=5), dict(logits=x.cpu()),
                   dict(n=101, row_stride=101)):
        with pytest.raises(AssertionError):
            exe.exe_op_logprobs(**{**good, **change})
    with pytest.raises(exe.ExeError):
        exe.exe_op_logprobs(**{**good, "logits": torch.zeros((4, 60000), device=DEV), "row_stride": 60000, "n": 60000})      # no workspace


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [5000, 40000, 600000])
def test_far_apart_at_a_small_scale(dtype, n):
    """Logits whose differences pass the largest float, which the scale brings back to a few units: in one wave, of several and of several parts."""
    g = torch.Generator().manual_seed(n)
    x = torch.full((3, n), -3e38)
    x[0, n // 2], x[1, -1] = 3e38, 2e38
    x[2] = (2 * torch.rand(n, generator=g) - 1) * 3e38
    x = x.to(TYPES[dtype][1])
    tokens = torch.tensor([[0, n // 2, n - 1]] * 3, dtype=torch.int32, device=DEV)
    check(x, 2e-38, tokens, 8, call(x.to(DEV), n, 2e-38, tokens, 8))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [300, 3000, 9000, 40000, 600000])
def test_signalling_nan_beside_the_largest(dtype, n):
    """A signalling NaN at every place of a 16-byte chunk, the largest logit at every other one; beside plus infinity; all of a chunk but one."""
    t = TYPES[dtype][1]
    bits, nan, minus_nan = (torch.int32, 0x7f800001, 0xff800001 - (1 << 32)) if dtype == "f32" else (torch.int16, 0x7f81, 0xff81 - (1 << 16))
    chunk = 16 // t.itemsize
    places = [(i, j) for i in range(chunk) for j in range(chunk) if i != j]
    x = torch.randn((len(places) + 2, n), generator=torch.Generator().manual_seed(n)).to(t)
    at = n // 2 // chunk * chunk
    raw = x.view(bits)
    for r, (i, j) in enumerate(places):
        x[r, at + j] = 100.0
        raw[r, at + i] = nan
    x[-2, at], x[-2, at + 1], x[-1, at + chunk - 1] = math.inf, 50.0, 60.0
    raw[-2, at + 3], raw[-1, at:at + chunk - 1] = nan, minus_nan
    tokens = torch.full((len(x), 1), at, dtype=torch.int32, device=DEV)
    for k in (1, 5, 40):
        lp, en, ids, top = call(x.to(DEV), n, 1.0, tokens, k)
        assert torch.equal(ids.cpu(), best(x, k))
        assert bool(lp.isnan().all()) and bool(en.isnan().all()) and bool(top.isnan().all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 700, 3000, 9000, 40000, 60000, 600000])
def test_no_probability_above_one_and_no_entropy_below_zero(dtype, n):
    """Rows with one token left, of many magnitudes; rows so peaked that the others vanish, or nearly."""
    g = torch.Generator().manual_seed(n)
    rows = 64 if n < 100000 else 16
    at = torch.randint(0, n, (rows, 1), generator=g)
    left = torch.full((rows, n), -math.inf).scatter_(1, at, torch.randn((rows, 1), generator=g) * 10.0 ** torch.linspace(-3, 30, rows)[:, None])
    peaked = torch.randn((rows, n), generator=g).scatter_(1, at, torch.linspace(5, 120, rows)[:, None])
    tokens = at.int().to(DEV)
    for x in (left.to(TYPES[dtype][1]), peaked.to(TYPES[dtype][1])):
        for scale in (1.0, 0.7, 1.3, 3.0):
            got = call(x.to(DEV), n, scale, tokens, 1)
            lp, en, ids, top = got
            assert bool((lp <= 0).all()) and bool((top <= 0).all()) and bool((en >= 0).all())
            check(x, scale, tokens, 1, got)


def test_logits_of_a_models_own_steps():
    """What exe_encode and exe_decode_step hand out goes straight in: the first alternative is the token that they return."""
    shape = wl.tiny_shape()
    m = exe.Model(exe.config_from_shape(shape, kv_pool_bytes=1 << 24, max_seqs=8, max_batch_tokens=128, max_batch_seqs=8), [t.to(DEV) for t in wl.make_weights(shape, seed=1)])
    lens = np.array([9, 20, 5], dtype=np.int32)
    logits = torch.empty((3, shape.vocab), device=DEV)
    tokens = np.random.default_rng(0).integers(0, shape.vocab, lens.sum()).astype(np.int32)
    nxt = m.encode([0, 1, 2], lens, tokens, reserve_lengths=lens + 16, out_device=logits)
    for step in range(1, 5):
        given = torch.as_tensor(nxt[:, None].copy()).to(DEV)
        got = call(logits, shape.vocab, 0.8, given, 5)
        check(logits.cpu(), 0.8, given, 5, got)
        assert np.array_equal(got[2][:, 0].cpu().numpy(), nxt) and torch.equal(got[0][:, 0], got[3][:, 0])
        nxt = m.decode_step([0, 1, 2], nxt, lens + step, out_device=logits)
    m.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [257, 300, 495, 511, 512, 513, 1023, 1100, 2100])
def test_rows_that_few_threads_hold(dtype, n):
    """Parts in which fewer than k threads, or 64ths of them, have a logit; as many candidates as are sorted at once, and one more."""
    g = torch.Generator().manual_seed(n)
    x = (torch.randn((5, n), generator=g) * 2.5).to(TYPES[dtype][1])
    x[1], x[2] = 0.5, torch.arange(n).to(x.dtype) / n
    x[3, torch.rand(n, generator=g) < 0.5] = -math.inf
    x[4, 30:] = -math.inf
    tokens = torch.full((5, 1), 7, dtype=torch.int32, device=DEV)
    x[3, 7] = 1.0
    for k in (2, 17, 20, 32, 33, 40, 64):
        check(x, 1.0, tokens, k, call(x.to(DEV), n, 1.0, tokens, k))
