"""The sizes that the GPU tests of the cross-entropy of a linear layer rely on still take the tiles that they are there for: no GPU needed."""
import ctypes as C

import pytest

import paper_2405_10951_amd as P
from linear_ce_sizes import FEW, L, MID, PIECES, SHORT, SMALL, TILES


@pytest.mark.parametrize("size,want", TILES + PIECES)
def test_sizes_take_their_tiles(size, want):
    N, D, V, dtype, dw, aligned = size
    t = P.bsr_linear_ce_tiles(N, D, V, dtype, aligned, dw)
    forward, gradient, products, forward_pieces, pieces = want
    assert (t.forward, t.gradient, t.products) == (forward, gradient, products)
    assert t.forward_pieces >= forward_pieces and t.pieces >= pieces
    if (size, want) in PIECES and max(forward_pieces, pieces) > 1:
        assert D % 64 or dtype == "fp32"                       # (w is packed)


def test_every_tile_is_taken():
    for i, tiles in ((0, {L, SHORT, SMALL, MID, FEW}), (1, {L, SHORT, SMALL, MID, FEW}), (2, {L, SMALL})):
        for kind in (("bf16", "bf16"), ("bf16", "fp32"), ("fp32", "fp32")):
            got = {w[i] for s, w in TILES + PIECES if s[3] == kind[0] and (i == 0 or s[4] == kind[1])}
            assert tiles <= got, (i, kind)


def test_few_rows_and_little_work_take_none():
    assert P.bsr_linear_ce_tiles(32, 768, 100, "fp32") == (0,) * 9
    assert P.bsr_linear_ce_tiles(20, 1024, 50000, "bf16").pieces == 0
    t = P.bsr_linear_ce_tiles(130, 96, 400, "bf16")
    assert t.forward == t.gradient == 0 and t.products == SMALL


def test_arguments():
    lib, out = P.load_library(), (C.c_int32 * 3)(7, 7, 7)
    assert lib.bsr_linear_ce_tiles(0, 2048, 768, 21841, 1, 0, out, 2) == 9 and out[0] == L and out[1] == 1 and out[2] == 7
    assert lib.bsr_linear_ce_tiles(0, 2048, 768, 21841, 1, 0, None, 0) == 9
    for bad in ((2, 10, 10, 10, 1, 0), (0, 0, 10, 10, 1, 0), (0, 10, 0, 10, 1, 0), (0, 10, 10, 0, 1, 0), (0, 10, 10, 10, 1, 2), (1, 10, 10, 10, 1, 0), (0, (1 << 22) + 1, 1, 1, 1, 0)):
        assert lib.bsr_linear_ce_tiles(*bad, out, 3) < 0
    assert lib.bsr_linear_ce_tiles(0, 10, 10, 10, 1, 0, None, 3) < 0 and lib.bsr_linear_ce_tiles(0, 10, 10, 10, 1, 0, out, -1) < 0
