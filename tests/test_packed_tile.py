"""The tile that corey_pack_tile gives for batches of many sequences."""
import pytest

from paper_2604_10597_amd.binding import corey_pack_tile


@pytest.mark.parametrize("long, S, D", [(16384, 201, 5120), (16384, 120, 5120), (800, 201, 5120), (16384, 300, 2048), (8192, 2001, 1536)])
def test_one_long_prompt_among_single_tokens(long, S, D):
    """Many sequences do not make a tile long: the tiles of the one that has nearly all tokens have to fill the GPU by themselves, with
    half a wave a SIMD at least (1024 SIMDs; a tile is a wave per 64 channels)."""
    T = long + S - 1
    tile = corey_pack_tile(S, T, D)
    assert tile % 16 == 0 and tile >= 32
    assert -(-long // tile) * (D // 64) >= 512 or tile <= 64, tile


@pytest.mark.parametrize("mean", [1, 3, 16, 50, 128, 250])
@pytest.mark.parametrize("S, D", [(160, 5120), (300, 2048), (2000, 1536)])
def test_many_sequences_of_like_lengths_are_walked_whole(mean, S, D):
    """Lengths over a factor of 20, even over the logarithm, reach 20 ln 20 / 19 = 3.15 times their mean."""
    tile = corey_pack_tile(S, S * mean, D)
    assert min(1024, 3.15 * mean) <= tile <= max(32, 4 * mean + 16)
