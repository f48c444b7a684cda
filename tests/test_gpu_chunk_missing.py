"""Attention of a chunk over a paged cache of which some blocks are not there, for rows that do not see them."""
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
@pytest.mark.parametrize("block", [8, 16, 32])
@pytest.mark.parametrize("seqs", [[(40, 400), (1, 500), (100, 777)], [(1, 1900), (1, 300), (4, 2100)]], ids=["chunks", "tokens"])
def test_blocks_in_front_of_the_window_may_be_given_back(dtype, dh, block, seqs):
    """Hidden positions have probability 0, whose product with any number is 0: bits are the same with and without the blocks."""
    window = 101
    b = Batch(seqs, 8, 2, dh, block, dtype).fill().device()
    want = b.want(window=window)
    full = b.attend(window=window)
    for i, (n, L) in enumerate(seqs):
        gone = (L - n - window + 1) // block                    # blocks wholly in front of what the first new token sees
        assert gone > 0
        b.d_table[i, :gone] = -1
    got = b.attend(window=window)
    check(got, *want)
    assert torch.equal(got, full)


@pytest.mark.parametrize("dtype,dh", TYPES)
def test_rows_in_front_of_a_missing_block_keep_their_bits(dtype, dh):
    b = Batch([(80, 200), (30, 60)], 4, 2, dh, 16, dtype).fill().device()
    full = b.attend()
    b.d_table[0, 9] = -1                                        # positions 144 .. 159 of the first, whose rows 24 .. see them
    b.d_table[1, 3] = 1 << 29                                   # 48 .. 59 of the second, rows 18 ..
    got = b.attend()
    blind = torch.tensor(list(range(24)) + list(range(80, 98)))
    assert torch.equal(got[blind], full[blind])
    rest = torch.ones(110, dtype=torch.bool)
    rest[blind] = False
    assert bool(torch.isnan(got[rest].float()).all())
