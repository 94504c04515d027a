"""CPU-only checks of what the paged cache's entry points refuse and what they let pass: sizes that belong together."""
import ctypes

import pytest

from paper_2509_09754_amd import lava

FAKE = 0x10000                        # never dereferenced: every case fails validation first
ARG, SHAPE = lava.LAVA_ERR_INVALID_ARG, lava.LAVA_ERR_SHAPE


@pytest.mark.parametrize("blocks,want", [(1, SHAPE), (3, SHAPE), (5, SHAPE), (-1, ARG), (4, None), (0, None)])
def test_gather_takes_tables_of_the_pools_width_only(blocks, want):
    """A table of another number of blocks would be read with the wrong stride, or behind its end.  The second problem is always refused, so
    nothing is launched where the first one passes."""
    desc = lava.LayerDesc.make(32, 8, 128, 32, "bf16")
    pool = lava.PagePoolStruct(10, 32, 4, FAKE, FAKE, FAKE)
    good = lava.PagedCompactProblem(100, None, FAKE, FAKE, None, FAKE, FAKE, 64, FAKE, None)
    good.table_blocks = blocks
    bad = lava.PagedCompactProblem(100, None, FAKE, FAKE, None, FAKE, FAKE, 801, FAKE, None, 4)
    table = (lava.PagedCompactProblem * 2)(good, bad)
    got = lava.lib.lava_compact_paged(ctypes.byref(desc), 2, ctypes.byref(table), ctypes.byref(pool), None)
    assert got == (lava.LAVA_ERR_BUDGET if want is None else want)
