"""CPU-only checks of the paged cache's entry points: arguments are refused on the host before anything is launched, the table
of angles agrees with the frequencies' definition, the binding refuses tensors it cannot pass on."""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import paged_oracle as P
from paper_2509_09754_amd import lava

FAKE, ODD = 0x10000, 0x10008          # never dereferenced: every case fails validation first
ARG, SHAPE, BUDGET, SPACE = lava.LAVA_ERR_INVALID_ARG, lava.LAVA_ERR_SHAPE, lava.LAVA_ERR_BUDGET, lava.LAVA_ERR_WORKSPACE


def desc(**kw):
    return lava.LayerDesc.make(**{**dict(n_q_heads=32, n_kv_heads=8, head_dim=128, window=32, dtype="bf16"), **kw})


def pool(**kw):
    return lava.PagePoolStruct(**{**dict(n_pages=10, page_rows=32, max_blocks=4, k=FAKE, v=FAKE, pos=FAKE), **kw})


def tables(state_over=None, sizes=None, **kw):
    state = lava.PageStateStruct(*([FAKE] * 9))
    for name, value in (state_over or {}).items():
        setattr(state, name, value)
    a = dict(batch=2, heads=8, n_new=FAKE, counts=None, release=None, tokens=4, slots=FAKE, positions=FAKE, ws=FAKE, ws_bytes=1 << 20)
    a.update(kw)
    return lava.lib.lava_page_tables(ctypes.byref(sizes or pool(k=None, v=None, pos=None)), a["batch"], a["heads"], ctypes.byref(state),
                                     a["n_new"], a["counts"], a["release"], a["tokens"], a["slots"], a["positions"], a["ws"],
                                     a["ws_bytes"], None)


@pytest.mark.parametrize("kw,want", [
    (dict(batch=0), ARG), (dict(heads=0), ARG), (dict(tokens=-1), ARG), (dict(tokens=0), ARG), (dict(counts=FAKE), ARG),
    (dict(batch=65536), SHAPE), (dict(heads=65), SHAPE), (dict(batch=32768, heads=64), SHAPE), (dict(tokens=1 << 28), SHAPE),
    (dict(ws=None), SPACE), (dict(ws=FAKE + 16), SPACE), (dict(ws_bytes=300), SPACE),
    (dict(state_over=dict(block_table=None)), ARG), (dict(state_over=dict(n_free_out=None)), ARG),
    (dict(sizes=pool(page_rows=24)), SHAPE), (dict(sizes=pool(page_rows=512)), SHAPE), (dict(sizes=pool(page_rows=8)), SHAPE),
    (dict(sizes=pool(n_pages=0)), ARG), (dict(sizes=pool(n_pages=1 << 31)), SHAPE), (dict(sizes=pool(max_blocks=0)), ARG),
    (dict(sizes=pool(max_blocks=1 << 26)), SHAPE)])
def test_tables_refuse(kw, want):
    assert tables(**kw) == want


def test_tables_workspace():
    size = lava.lava_page_tables_workspace_bytes
    assert size(0, 8) == size(1, 65) == size(65536, 1) == size(65535, 64) == 0
    assert 0 < size(1, 1) <= size(64, 8) <= size(2048, 8) <= size(16384, 64)
    assert tables(ws_bytes=size(2, 8) - 1) == SPACE


def test_compact_refuses():
    p = lava.PagedCompactProblem(100, None, FAKE, FAKE, None, FAKE, FAKE, 64, FAKE, None)
    call = lambda d, n, pr, po: lava.lib.lava_compact_paged(ctypes.byref(d), n, ctypes.byref(pr) if pr else None,
                                                            ctypes.byref(po) if po else None, None)
    assert call(desc(), 0, p, pool()) == ARG and call(desc(), 1, None, pool()) == ARG and call(desc(), 1, p, None) == ARG
    assert call(desc(head_dim=96), 1, p, pool()) == SHAPE and call(desc(), 1, p, pool(k=ODD)) == ARG
    assert call(desc(), 1, p, pool(v=None)) == ARG and call(desc(), 1, p, pool(max_blocks=0)) == ARG
    for name, value, want in (("k_src", None, ARG), ("v_src", ODD, ARG), ("head_offsets", None, ARG), ("kept_idx", None, ARG),
                              ("block_table", None, ARG), ("src_rows", 0, ARG), ("capacity", -1, ARG), ("capacity", 801, BUDGET)):
        q = lava.PagedCompactProblem.from_buffer_copy(p)
        setattr(q, name, value)
        assert call(desc(), 1, q, pool()) == want, name


def turn(rot=None, dtype=lava.LAVA_BF16, d=128, tokens=4, heads=8, x=FAKE, xs=(1024, 128), out=FAKE + (1 << 20), os=(1024, 128),
         turns=FAKE, positions=FAKE):
    return lava.lib.lava_rotary(ctypes.byref(rot or lava.RotaryDesc.make(128)), turns, dtype, d, tokens, heads, positions, x, *xs,
                                out, *os, 0, None)


@pytest.mark.parametrize("kw,want", [
    (dict(dtype=2), ARG), (dict(d=96), SHAPE), (dict(tokens=-1), ARG), (dict(heads=0), ARG), (dict(x=ODD), ARG), (dict(out=None), ARG),
    (dict(turns=None), ARG), (dict(positions=None), ARG), (dict(xs=(1020, 128)), ARG), (dict(os=(1024, 100)), ARG),
    (dict(os=(1024, 64)), ARG), (dict(os=(512, 128)), ARG), (dict(os=(128, 256)), ARG), (dict(xs=(-1024, 128)), ARG),
    (dict(out=FAKE, os=(128, 1024)), ARG), (dict(heads=1025), SHAPE), (dict(tokens=1 << 31), SHAPE),
    (dict(rot=lava.RotaryDesc.make(130)), SHAPE), (dict(rot=lava.RotaryDesc.make(7)), SHAPE), (dict(rot=lava.RotaryDesc.make(0)), ARG),
    (dict(rot=lava.RotaryDesc.make(64, magnitude=-1.0)), ARG), (dict(rot=lava.RotaryDesc.make(64, magnitude=math.nan)), ARG),
    (dict(rot=lava.RotaryDesc(64, 2, 1.0, 0, 1e4, 1.0, 1.0, 4.0)), ARG)])
def test_rotary_refuses(kw, want):
    assert turn(**kw) == want


def test_rotary_without_tokens_is_nothing():
    assert turn(tokens=0) == lava.LAVA_OK and append(tokens=0) == lava.LAVA_OK


def append(d=None, rot=None, turns=FAKE, tokens=4, positions=FAKE, q=FAKE, qs=6144, k=FAKE, ks=6144, v=FAKE, vs=6144, q_out=FAKE + (1 << 20),
           p=None, slots=FAKE):
    return lava.lib.lava_rotary_append(ctypes.byref(d or desc()), ctypes.byref(rot or lava.RotaryDesc.make(128)), turns, tokens, positions,
                                       q, qs, k, ks, v, vs, q_out, ctypes.byref(p or pool()), slots, None)


@pytest.mark.parametrize("kw,want", [
    (dict(d=desc(head_dim=96)), SHAPE), (dict(rot=lava.RotaryDesc.make(130)), SHAPE), (dict(turns=None), ARG), (dict(tokens=-1), ARG),
    (dict(positions=None), ARG), (dict(q=None), ARG), (dict(q_out=None), ARG), (dict(q=ODD), ARG), (dict(qs=6140), ARG), (dict(k=None), ARG),
    (dict(ks=-6144), ARG), (dict(v=None), ARG), (dict(vs=3), ARG), (dict(slots=None), ARG), (dict(q_out=FAKE), ARG), (dict(q_out=ODD), ARG),
    (dict(p=pool(k=None)), ARG), (dict(p=pool(page_rows=33)), SHAPE), (dict(p=pool(n_pages=-1)), ARG), (dict(tokens=1 << 28), SHAPE)])
def test_append_refuses(kw, want):
    assert append(**kw) == want


def decode(d=None, batch=2, q=FAKE, p=None, table=FAKE, rows=FAKE, o=None, q_pos=None, out=FAKE, lse=FAKE, ws=FAKE, ws_bytes=1 << 30):
    return lava.lib.lava_paged_decode(ctypes.byref(d or desc()), batch, q, ctypes.byref(p or pool()), table, rows,
                                      ctypes.byref(o) if o else None, q_pos, out, lse, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,want", [
    (dict(d=desc(n_q_heads=72)), SHAPE), (dict(d=desc(dtype="f32", head_dim=32)), SHAPE), (dict(batch=0), ARG), (dict(q=None), ARG),
    (dict(q=ODD), ARG), (dict(table=None), ARG), (dict(rows=None), ARG), (dict(out=None), ARG), (dict(p=pool(v=ODD)), ARG),
    (dict(p=pool(max_blocks=0)), ARG), (dict(o=lava.DecodeOptions(-1.0, 0, None)), ARG), (dict(o=lava.DecodeOptions(0.0, -1, None)), ARG),
    (dict(o=lava.DecodeOptions(math.nan, 0, None)), ARG), (dict(o=lava.DecodeOptions(0.0, 5, None)), ARG),
    (dict(o=lava.DecodeOptions(0.0, 0, FAKE)), ARG), (dict(o=lava.DecodeOptions(0.0, 5, None), q_pos=FAKE, p=pool(pos=None)), ARG),
    (dict(o=lava.DecodeOptions(0.0, 5, None), q_pos=FAKE, p=pool(pos=ODD)), ARG), (dict(p=pool(max_blocks=1 << 25), batch=130), SHAPE),
    (dict(batch=65536), SHAPE), (dict(batch=8193), SHAPE), (dict(ws=None), SPACE), (dict(ws=FAKE + 128), SPACE), (dict(ws_bytes=255), SPACE)])
def test_decode_refuses(kw, want):
    assert decode(**kw) == want


def test_decode_workspace():
    size = lava.lava_paged_decode_workspace_bytes
    assert size(desc(n_q_heads=72)) == 0 and size(desc(head_dim=32)) == 0
    for kw in ({}, dict(dtype="f32"), dict(n_q_heads=8), dict(n_q_heads=64), dict(head_dim=64)):
        assert size(desc(**kw)) > 0
        assert decode(d=desc(**kw), ws_bytes=size(desc(**kw)) - 1) == SPACE


@pytest.mark.parametrize("rot,kw", [(128, dict(base=10000.0)), (64, dict(base=500000.0, factor=8.0)), (2, dict(base=10.0)),
                                    (38, dict(base=1e6, factor=4.0, original_context=4096, low_turns=1.0, high_turns=32.0)),
                                    (128, dict(base=500000.0, factor=8.0, original_context=8192, low_turns=1.0, high_turns=4.0))])
def test_turns(rot, kw):
    t = lava.lava_rotary_turns(lava.RotaryDesc.make(rot, **kw)).numpy().view(np.uint64).astype(np.float64) / 2.0 ** 64
    f = P.rotary_frequencies(rot, **kw) / (2 * math.pi)
    # pow, a division and the blend of the oracle, each within 2^-52; 2^-65 for the rounding to 2^-64 turns
    assert (np.abs(t - f) <= 24 * 2.0 ** -53 * f + 2.0 ** -64).all()


@pytest.mark.parametrize("kw", [dict(base=1.0), dict(base=0.0), dict(base=math.nan), dict(base=math.inf), dict(factor=0.5), dict(factor=math.nan),
                                dict(original_context=-1), dict(original_context=5, low_turns=4.0, high_turns=4.0),
                                dict(original_context=5, low_turns=-1.0)])
def test_turns_refuse(kw):
    with pytest.raises(lava.LavaError):
        lava.lava_rotary_turns(lava.RotaryDesc.make(64, **kw))


def test_binding_refuses_host_tensors():
    """No tensor on the host is ever handed to the library."""
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)
    with pytest.raises(ValueError):
        lava.PagePool(torch.zeros(4, 16, 128), torch.zeros(4, 16, 128))
    with pytest.raises(ValueError):
        lava.PageState(i32(1, 2, 3), i32(1, 2), i32(1), i32(8), i32(1), 16)
    with pytest.raises(ValueError):
        lava.lava_rotary(lava.RotaryDesc.make(64), torch.zeros(32, dtype=torch.int64), i32(4), torch.zeros(4, 2, 64))
    with pytest.raises(ValueError):
        lava.DecodeOptions.make(slopes=torch.zeros(32))
