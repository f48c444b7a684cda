"""Attention of a chunk over a paged cache where values are large, against 64 bits, and where rows are NaN."""
import pytest
import torch

import chunk_util
from chunk_util import Batch, check

pytestmark = pytest.mark.gpu

TYPES = [("bf16", 64), ("bf16", 128), ("f32", 64), ("f32", 128)]


@pytest.fixture(autouse=True, params=[1, 1100], ids=["own", "tiles"])
def bound(request, monkeypatch):
    """As in test_gpu_chunk_attention.py: small cases to their own kernel, and to the tile kernel."""
    monkeypatch.setattr(chunk_util, "BOUND", request.param)


@pytest.mark.parametrize("dtype,dh", TYPES)
@pytest.mark.parametrize("seqs", [[(1, 1), (40, 300), (3, 77), (1, 200)], [(1, 3000), (5, 2000)], [(1, 600), (90, 2500)]], ids=["whole", "tokens_in_parts", "chunks_in_parts"])
def test_values_whose_sum_passes_a_floats_end(dtype, dh, seqs):
    """Values of 2^126 to 2^127, of one sign and of either: results are finite, sums of three or more of them are not.  The bound is the
    one of all values (Batch.want): a running mean rounds 3 times more for each 64 keys, (n / 64) * 3 half steps, of the 2 * n that it
    allows for n keys."""
    b = Batch(seqs, 8, 2, dh, 16, dtype)
    g = torch.Generator().manual_seed(5)
    for i, v in enumerate(b.v):
        big = 2.0 ** 126 * (1 + torch.rand(v.shape, generator=g, dtype=torch.float64))
        big[1] *= torch.where(torch.rand(v.shape[1:], generator=g) < 0.5, -1.0, 1.0)
        b.v[i] = big.to(b.t)
    check(b.fill().device().attend(), *b.want())


@pytest.mark.parametrize("dtype,dh", TYPES)
@pytest.mark.parametrize("what", ["queries", "keys", "infinite keys", "scores of minus infinity"])
def test_rows_that_are_nan_cost_no_more_than_others(dtype, dh, what):
    """Nothing is gained by computing a row again whose own scores are no numbers.  (It took 42 to 166 times as long; 4 leaves room for a
    card that is not at its clock.)"""
    b = Batch([(200, 900), (1, 3000)], 8, 2, dh, 16, dtype).fill().device()
    out, ws = torch.empty_like(b.d_q), torch.empty(1 << 24, dtype=torch.uint8, device=chunk_util.DEV)

    def time():
        best = 1e9
        for _ in range(5):
            ends = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
            ends[0].record()
            for _ in range(10):
                b.attend(out=out, workspace=ws)
            ends[1].record()
            torch.cuda.synchronize()
            best = min(best, ends[0].elapsed_time(ends[1]))
        return best

    time()
    clean = time()
    if what == "queries":
        b.d_q.fill_(float("nan"))
    elif what == "scores of minus infinity":
        b.d_q.fill_(1.0)
        b.d_pool[:, 0] = -float("inf")
    else:
        b.d_pool[:, 0] = float("nan") if what == "keys" else float("inf")
    spoilt = time()
    assert bool(torch.isnan(out.float()).all())
    assert spoilt < 4 * clean, (clean, spoilt)
