"""Host logic of the orthogonalised update's product kernel: the unit plan (no GPU).  Every piece of 64 columns of every row block, from
the diagonal on in symmetric products, must be computed exactly once, and units come widest first."""
import itertools

import numpy as np
import pytest

from paper_1810_00952_b200 import binding as B


def check_plan(rows, cols, symmetric, k_blocks, batch, pairs):
    units = B.relay_debug_orthogonalize_units(rows, cols, symmetric, k_blocks, batch, pairs)
    tiles, pieces = -(-rows // 256), -(-cols // 64)
    if units is None:
        assert sum(-(-(pieces - (4 * m if symmetric else 0)) // 8) for m in range(tiles)) > 640      # even the widest are too many
        return
    cover = np.zeros((tiles, pieces + 8), dtype=np.int32)
    for m, at, width in units:
        assert 0 <= m < tiles and width in (1, 2, 4, 6, 8) and 0 <= at < pieces and at + width <= pieces + 1, (m, at, width)
        cover[m, at:at + width] += 1
    for m in range(tiles):
        first = 4 * m if symmetric else 0
        assert (cover[m, first:pieces] == 1).all() and not cover[m, :first].any(), (rows, cols, symmetric, k_blocks, batch, pairs, m)
    widths = [w for _, _, w in units]
    assert widths == sorted(widths, reverse=True)


@pytest.mark.parametrize("pairs", [74, 66, 8, 1])
@pytest.mark.parametrize("symmetric", [False, True])
def test_plan_covers_every_piece_once(symmetric, pairs):
    sizes = (1, 63, 64, 129, 256, 257, 333, 500, 600, 1024, 1500, 4096, 9000, 65536)
    for rows, cols, batch, k_blocks in itertools.product(sizes, sizes, (1, 3, 8, 200), (1, 8, 64)):
        if not symmetric:
            check_plan(rows, cols, False, k_blocks, batch, pairs)
        elif rows == cols:
            check_plan(rows, rows, True, k_blocks, batch, pairs)


def test_bad_arguments_are_refused():
    with pytest.raises(ValueError):
        B.relay_debug_orthogonalize_units(100, 200, True, 4, 1, 74)
    with pytest.raises(ValueError):
        B.relay_debug_orthogonalize_units(0, 64, False, 4, 1, 74)
