"""Host logic of the gated recurrence: which form of its kernels takes a call (no GPU; descriptors are not dereferenced).  Tiles and
spans keep a place within a step's row as 32-bit byte offsets, so no row of 2^32 bytes or more may reach them."""
import itertools

import pytest

from paper_1810_00952_b200 import binding as B

STEPS, SPANS, TILES = 0, 1, 2
SIZE = {B.F32: 4, B.BF16: 2}


def form(T, Bn, D, dt=B.BF16, out_dt=None, packed=False, ragged=False):
    d = B.desc_of_type
    f = d(dt, (T, Bn, 2 * D if packed else D))
    return B.relay_debug_recurrence_form(f, None if packed else d(dt, (T, Bn, D)), d(dt if out_dt is None else out_dt, (T, Bn, D)), ragged)


def test_ordinary_sizes():
    assert [form(T, 64, 1024) for T in (1, 12, 13, 4096)] == [STEPS, STEPS, TILES, TILES]
    assert [form(T, 13, 333, B.F32, ragged=True) for T in (1, 32, 33, 4096)] == [STEPS, STEPS, SPANS, SPANS]
    assert form(100, 8, 333) == TILES and form(100, 8, 333, ragged=True) == SPANS      # one row of 2664 channels, or rows of 333
    assert form(100, 8, 332, packed=True) == SPANS and form(100, 8, 336, packed=True) == TILES
    assert form(4, 0, 8) == STEPS


@pytest.mark.parametrize("dt,out_dt", [(B.F32, B.F32), (B.BF16, B.BF16), (B.BF16, B.F32)])
@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("ragged", [False, True])
def test_rows_of_32_bits_and_more_run_step_by_step(dt, out_dt, packed, ragged):
    for bits, Bn, T, less in itertools.product(range(26, 34), (1, 8), (13, 40), (0, 1)):
        D = ((1 << bits) // Bn // 16 - less) * 16
        row = Bn * D * SIZE[dt] * (2 if packed else 1)
        assert form(T, Bn, D, dt, out_dt, packed, ragged) == (TILES if row < 1 << 32 else STEPS), (bits, Bn, T, D)
        if not packed and not ragged:
            D |= 1                                             # no whole 16-byte pieces: spans in the tiles' place
            wide = max(Bn * D * SIZE[dt], Bn * D * SIZE[out_dt]) >= 1 << 32
            if Bn == 1:
                assert form(T, 1, D, dt, out_dt) == (STEPS if wide or T <= 32 else SPANS), (bits, T, D)
    # 13 steps of 2^30 packed fp32 columns: 168 GB with its gradients, which a GPU can hold
    assert form(13, 1, 1 << 29, B.F32, packed=True) == STEPS
    assert form(13, 1, (1 << 29) - 4, B.F32, packed=True) == TILES


def test_refused_types_have_no_form():
    with pytest.raises(ValueError):
        B.relay_debug_recurrence_form(B.desc_of_type(B.I32, (4, 2, 8)), None, B.desc_of_type(B.F32, (4, 2, 4)))
