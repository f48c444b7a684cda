"""Into how many parts the chunk attention cuts keys, as its workspace tells (CPU)."""
import pytest

import paper_2404_07947_amd as exe


def parts(dtype, n, new, L, H, Hkv, dh):
    """Of n sequences of `new` tokens each, which all go to the tile kernel."""
    return exe.exe_op_chunk_attention_paged_workspace(dtype, n, n * new, new, L, H, Hkv, dh) // (n * new * H * (dh + 2) * 4) or 1


@pytest.mark.parametrize("dtype,dh", [(1, 128), (1, 64), (0, 64), (0, 128)])
@pytest.mark.parametrize("n,few,full,H,Hkv,L", [(32, 5, 16, 32, 8, 4000), (8, 24, 64, 40, 40, 4000), (32, 20, 64, 40, 40, 2000), (4, 9, 16, 32, 8, 9000),
                                                (64, 5, 16, 8, 2, 3000)])
def test_a_partly_filled_tile_is_a_tile(dtype, dh, n, few, full, H, Hkv, L):
    """`few` and `full` tokens make as many tiles of 64 rows over as many keys: as many parts fill the chip."""
    assert few * H // Hkv <= 64 == full * H // Hkv
    assert parts(dtype, n, few, L, H, Hkv, dh) == parts(dtype, n, full, L, H, Hkv, dh)
