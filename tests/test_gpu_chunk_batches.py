"""Attention of a chunk over a paged cache: batches of many sequences, every row against 64 bits.

More than 256 pairs of a sequence and a key/value head run 4 waves a workgroup, whole or in parts; from 64 sequences on, a workgroup of
the tile kernel, of its join and of the tiles of 16 rows finds its sequence by a search."""
import numpy as np
import pytest
import torch

import paper_2404_07947_amd as exe
from chunk_util import Batch, check

pytestmark = pytest.mark.gpu

TYPES = [("bf16", 64), ("bf16", 128), ("f32", 64), ("f32", 128)]


def in_parts(b, max_new, max_len, window=0):
    return exe.exe_op_chunk_attention_paged_workspace(b.code, len(b.seqs), b.rows, max_new, max_len, b.H, b.Hkv, b.dh, window) > 0


@pytest.mark.parametrize("dtype,dh", TYPES)
@pytest.mark.parametrize("Hkv,G,n,long,parts", [(4, 2, 70, 1500, True), (8, 1, 70, 1100, True), (4, 1, 90, 250, False), (8, 4, 260, 600, False)])
def test_many_single_tokens(dtype, dh, Hkv, G, n, long, parts):
    rng = np.random.default_rng(n + long)
    seqs = [(1, int(L)) for L in rng.integers(1, 200, n)]
    for i in (0, n // 2, n - 1):
        seqs[i] = (1, long)
    seqs[3] = (0, 40)                                            # and sequences that bring nothing
    seqs[n - 2] = (0, 0)
    b = Batch(seqs, Hkv * G, Hkv, dh, 16, dtype, seed=n, extra_rows=2).fill().device()
    assert n * Hkv > 256 and in_parts(b, 1, long) == parts
    check(b.attend(), *b.want())


def mixed(n, most, rng, longest):
    """n sequences: a quarter of them empty, a quarter single tokens, the others of 2 to `most` new tokens."""
    seqs = []
    for i in range(n):
        new = (0, 1, int(rng.integers(2, 9)), int(rng.integers(2, most + 1)))[i % 4]
        seqs.append((new, new + int(rng.integers(0, 120))))
    order = rng.permutation(n)
    seqs = [seqs[i] for i in order]
    seqs[n // 3] = (most, longest)
    return seqs


@pytest.mark.parametrize("dtype,dh", TYPES)
@pytest.mark.parametrize("n", [63, 64, 65, 130])
@pytest.mark.parametrize("kernel", ["tiles", "tiles in parts", "tiles of 16"])
def test_many_sequences(dtype, dh, n, kernel):
    """Float x 128 has no tiles of 16 rows and runs tiles in their place."""
    rng = np.random.default_rng(n)
    most, longest = {"tiles": (150, 1100), "tiles in parts": (17, 2600), "tiles of 16": (17, 700)}[kernel]
    Hkv, G = (2, 4) if kernel == "tiles" else (1, 4)
    b = Batch(mixed(n, most, rng, longest), Hkv * G, Hkv, dh, 16, dtype, seed=n, extra_rows=1).fill().device()
    if kernel == "tiles in parts":
        assert in_parts(b, most, longest)
    check(b.attend(), *b.want())
    check(b.attend(window=50), *b.want(window=50))


@pytest.mark.parametrize("new", [2, 5, 8])
def test_drafted_tokens(new):
    """A decode batch that brings a few tokens each, in parts."""
    rng = np.random.default_rng(new)
    seqs = [(new, int(L)) for L in rng.integers(new, 1400, 66)]
    b = Batch(seqs, 8, 2, 128, 16, "bf16", seed=new).fill().device()
    check(b.attend(), *b.want())
    seqs = [(new, 1600 + i) for i in range(66)]
    b = Batch(seqs, 4, 1, 64, 16, "bf16", seed=new).fill().device()
    assert in_parts(b, new, 1700)
    check(b.attend(), *b.want())
