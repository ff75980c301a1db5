"""The cache of 8 bits without a GPU: the room that a workspace has for parts of tiles of many new tokens."""
import pytest

import paper_2410_18248_amd as P

PLACES = 512                     # workgroups of such tiles that the chip holds at once


@pytest.mark.parametrize("H,Hkv,D,columns", [(32, 8, 128, 128), (32, 32, 128, 128), (40, 40, 128, 128), (1, 1, 128, 128), (8, 2, 64, 128), (16, 16, 64, 128), (6, 2, 128, 128),
                                             (17, 1, 64, 128), (16, 16, 256, 64), (16, 4, 256, 64), (16, 1, 256, 64), (17, 1, 256, 128), (32, 1, 256, 128)])
def test_a_launch_is_cut_into_as_many_parts_for_every_geometry(H, Hkv, D, columns):
    """Up to twice the places, of a tile's columns each: outputs, reference and sum, and a word for the hand-over."""
    cfg = P.LampsConfig(1, H, Hkv, D, 16, 4, 4, 4, P.LAMPS_E4M3)
    cfg.staging_bytes = block = P.lamps_block_bytes(cfg)
    assert P.lamps_workspace_bytes(cfg) - 2 * block >= 2 * PLACES * (columns * (D + 2) * 4 + 8)


def test_only_a_cache_of_8_bits_asks_for_it():
    for H, Hkv in ((32, 32), (16, 16)):
        wide, codes = (P.LampsConfig(1, H, Hkv, 128, 16, 4, 4, 4, dtype) for dtype in (P.LAMPS_BF16, P.LAMPS_E4M3))
        wide.staging_bytes, codes.staging_bytes = P.lamps_block_bytes(wide), P.lamps_block_bytes(wide)
        assert P.lamps_workspace_bytes(wide) < 20 << 20 < P.lamps_workspace_bytes(codes)
