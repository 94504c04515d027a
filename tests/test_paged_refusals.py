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


def test_no_tokens_need_no_buffers():
    """Empty tensors have no address; a step without tokens is nothing all the same, but for what is wrong whatever the tokens."""
    desc, rot = lava.LayerDesc.make(32, 8, 128, 32, "bf16"), lava.RotaryDesc.make(128)
    pool = lava.PagePoolStruct(10, 32, 4, FAKE, FAKE, FAKE)
    turn = lambda tokens, heads=8, r=rot: lava.lib.lava_rotary(ctypes.byref(r), FAKE, lava.LAVA_BF16, 128, tokens, heads, None, None, 1024, 128,
                                                               None, 1024, 128, 0, None)
    append = lambda tokens, p=pool: lava.lib.lava_rotary_append(ctypes.byref(desc), ctypes.byref(rot), FAKE, tokens, None, None, 4096, None, 1024,
                                                                None, 1024, None, ctypes.byref(p), None, None)
    assert turn(0) == lava.LAVA_OK and append(0) == lava.LAVA_OK
    assert turn(1) == ARG and append(1) == ARG and turn(-1) == ARG and append(-1) == ARG
    assert turn(0, heads=0) == ARG and turn(0, r=lava.RotaryDesc.make(130)) == SHAPE
    assert append(0, lava.PagePoolStruct(10, 33, 4, FAKE, FAKE, FAKE)) == SHAPE


def test_a_selection_of_nothing_needs_no_indices():
    desc = lava.LayerDesc.make(32, 8, 128, 32, "bf16")
    pool = lava.PagePoolStruct(10, 32, 4, FAKE, FAKE, FAKE)
    call = lambda capacity: lava.lib.lava_compact_paged(
        ctypes.byref(desc), 1, ctypes.byref(lava.PagedCompactProblem(100, None, FAKE, FAKE, None, FAKE, None, capacity, FAKE, None, 4)),
        ctypes.byref(pool), None)
    assert call(0) == lava.LAVA_OK and call(1) == ARG


@pytest.mark.parametrize("cap,refused", [(1e-40, True), (1e-39, True), (9e-31, True), (2e30, True), (float("inf"), True), (1e-30, False), (1e30, False),
                                         (0.0, False)])
def test_caps_have_a_reciprocal(cap, refused):
    """A cap whose reciprocal overflows would make NaN of a logit of zero.  Without a workspace nothing is launched."""
    desc = lava.LayerDesc.make(32, 8, 128, 32, "bf16")
    pool, options = lava.PagePoolStruct(10, 32, 4, FAKE, FAKE, FAKE), lava.DecodeOptions(cap, 0, None)
    got = lava.lib.lava_paged_decode(ctypes.byref(desc), 1, FAKE, ctypes.byref(pool), FAKE, FAKE, ctypes.byref(options), None, FAKE, FAKE, None, 0, None)
    assert got == (ARG if refused else lava.LAVA_ERR_WORKSPACE)
