"""CPU-only checks of the entry points of sequences that share pages: arguments are refused on the host before anything is launched, sizes that
are none have no workspace."""
import ctypes

import pytest

from paper_2509_09754_amd import lava

FAKE, ODD = 0x10000, 0x10008          # never dereferenced: every case fails validation first
ARG, SHAPE, SPACE = lava.LAVA_ERR_INVALID_ARG, lava.LAVA_ERR_SHAPE, lava.LAVA_ERR_WORKSPACE


def desc(**kw):
    return lava.LayerDesc.make(**{**dict(n_q_heads=32, n_kv_heads=8, head_dim=128, window=32, dtype="bf16"), **kw})


def pool(**kw):
    return lava.PagePoolStruct(**{**dict(n_pages=10, page_rows=32, max_blocks=4, k=FAKE, v=FAKE, pos=FAKE), **kw})


def state(**kw):
    s = lava.PageStateStruct(*([FAKE] * 9))
    for name, value in kw.items():
        setattr(s, name, value)
    return s


def beam(**kw):
    a = dict(dtype=lava.LAVA_BF16, batch=2, beams=4, vocab=1000, logits=FAKE, stride=1000, scores=FAKE, done=None, end=-1, pad=0, n_out=4, parents=FAKE,
             tokens=FAKE, scores_out=FAKE + 256, done_out=None, sources=None, n_tables=0, ws=FAKE, ws_bytes=1 << 30)
    a.update(kw)
    return lava.lib.lava_beam_step(*a.values(), None)


@pytest.mark.parametrize("kw,want", [
    (dict(dtype=2), ARG), (dict(batch=0), ARG), (dict(beams=0), ARG), (dict(vocab=0), ARG), (dict(n_out=0), ARG), (dict(batch=65536), SHAPE),
    (dict(beams=65), SHAPE), (dict(n_out=65), SHAPE), (dict(vocab=1 << 31, stride=1 << 31), SHAPE),
    (dict(batch=65535, beams=64, vocab=1 << 30, stride=1 << 30), SHAPE), (dict(batch=32768, vocab=128 * 8192, stride=1 << 20), SHAPE), (dict(logits=None), ARG), (dict(logits=FAKE + 1), ARG),
    (dict(dtype=lava.LAVA_F32, logits=FAKE + 2), ARG), (dict(scores=None), ARG), (dict(parents=None), ARG), (dict(tokens=None), ARG),
    (dict(scores_out=None), ARG), (dict(pad=-1), ARG), (dict(pad=1000), ARG), (dict(stride=999), ARG), (dict(stride=-1), ARG), (dict(stride=1 << 40), SHAPE),
    (dict(n_out=3, scores_out=FAKE), ARG), (dict(n_out=3, done=FAKE, done_out=FAKE), ARG), (dict(sources=FAKE), ARG), (dict(n_tables=1), ARG),
    (dict(n_tables=-1), ARG), (dict(sources=FAKE, n_tables=1025), SHAPE), (dict(batch=60000, beams=64, sources=FAKE, n_tables=1000), SHAPE),
    (dict(ws=None), SPACE), (dict(ws=FAKE + 16), SPACE), (dict(ws_bytes=100), SPACE)])
def test_beam_step_refuses(kw, want):
    assert beam(**kw) == want


def test_beam_step_lets_pass():
    """Odd addresses of 16-bit logits, one row of any stride, the buffers in place: refused for the missing workspace only."""
    assert beam(logits=FAKE + 2, ws=None) == SPACE
    assert beam(batch=1, beams=1, stride=0, n_out=64, ws=None) == SPACE
    assert beam(batch=32768, beams=4, vocab=127 * 8192, stride=1 << 20, ws=None) == SPACE
    assert beam(scores_out=FAKE, done=FAKE, done_out=FAKE, ws=None) == SPACE
    size = lava.lava_beam_step_workspace_bytes
    assert size(0, 4, 10, 4) == size(1, 65, 10, 4) == size(1, 4, 0, 4) == size(1, 4, 10, 0) == size(65535, 64, 1 << 30, 1) == 0
    assert 0 < size(1, 1, 1, 1) <= size(2, 4, 1000, 4) <= size(2, 4, 100000, 4) <= size(2, 4, 100000, 64)
    assert beam(ws_bytes=size(2, 4, 1000, 4) - 1) == SPACE


def fork(d=None, po=None, st=None, **kw):
    a = dict(batch=2, source=FAKE, table=None, free=None, ws=FAKE, ws_bytes=1 << 30)
    a.update(kw)
    return lava.lib.lava_page_fork(ctypes.byref(d or desc()), ctypes.byref(po or pool()), a["batch"], ctypes.byref(st or state()), a["source"], a["table"],
                                   a["free"], a["ws"], a["ws_bytes"], None)


def compact(d=None, po=None, st=None, **kw):
    a = dict(batch=2, counts=FAKE, kept=FAKE, capacity=100, evict=None, table=None, free=None, ws=FAKE, ws_bytes=1 << 30)
    a.update(kw)
    return lava.lib.lava_page_compact(ctypes.byref(d or desc()), ctypes.byref(po or pool()), a["batch"], ctypes.byref(st or state()), a["counts"], a["kept"],
                                      a["capacity"], a["evict"], a["table"], a["free"], a["ws"], a["ws_bytes"], None)


@pytest.mark.parametrize("call", [fork, compact])
@pytest.mark.parametrize("kw,want", [
    (dict(batch=0), ARG), (dict(batch=65536), SHAPE), (dict(ws=None), SPACE), (dict(ws=FAKE + 16), SPACE), (dict(ws_bytes=1000), SPACE),
    (dict(d=desc(head_dim=96)), SHAPE), (dict(d=desc(n_q_heads=64, n_kv_heads=64), batch=32768), SHAPE),
    (dict(po=pool(page_rows=24)), SHAPE), (dict(po=pool(n_pages=0)), ARG), (dict(po=pool(n_pages=1 << 31)), SHAPE), (dict(po=pool(max_blocks=0)), ARG),
    (dict(po=pool(max_blocks=1 << 26)), SHAPE), (dict(po=pool(page_rows=16, max_blocks=(1 << 27) - 1), batch=3), SHAPE), (dict(po=pool(k=None)), ARG),
    (dict(po=pool(v=ODD)), ARG), (dict(st=state(block_table=None)), ARG), (dict(st=state(head_rows=None)), ARG), (dict(st=state(seq_pos_out=None)), ARG),
    (dict(st=state(free_pages=None)), ARG), (dict(st=state(n_free_out=None)), ARG)])
def test_changes_refuse(call, kw, want):
    assert call(**kw) == want


def test_changes_refuse_what_is_their_own():
    assert fork(source=None) == ARG
    assert compact(counts=None) == ARG and compact(kept=None) == ARG and compact(capacity=-1) == ARG and compact(capacity=1 << 40) == SHAPE
    assert compact(kept=None, capacity=0, ws=None) == SPACE and fork(st=state(error=None), ws=None) == SPACE
    size = lava.lava_page_fork_workspace_bytes
    assert size(0, 8, 4, 10) == size(1, 65, 4, 10) == size(1, 8, 0, 10) == size(1, 8, 4, 0) == size(65535, 64, 4, 10) == size(65535, 8, 1 << 20, 10) == 0
    assert 0 < size(1, 1, 1, 1) <= size(2, 8, 4, 10) <= size(64, 8, 4, 10) <= size(64, 8, 4, 1 << 20) <= size(64, 8, 4000, 1 << 20)
    assert fork(ws_bytes=size(2, 8, 4, 10) - 1) == SPACE


def shared(d=None, po=None, options=None, **kw):
    a = dict(batch=4, q=FAKE, table=FAKE, rows=FAKE, n_groups=2, start=FAKE, q_pos=FAKE, out=FAKE, lse=None, ws=FAKE, ws_bytes=1 << 40)
    a.update(kw)
    return lava.lib.lava_shared_decode(ctypes.byref(d or desc()), a["batch"], a["q"], ctypes.byref(po or pool()), a["table"], a["rows"], a["n_groups"],
                                       a["start"], ctypes.byref(options) if options else None, a["q_pos"], a["out"], a["lse"], a["ws"], a["ws_bytes"], None)


@pytest.mark.parametrize("kw,want", [
    (dict(batch=0), ARG), (dict(q=None), ARG), (dict(q=ODD), ARG), (dict(table=None), ARG), (dict(rows=None), ARG), (dict(out=None), ARG),
    (dict(n_groups=0), ARG), (dict(n_groups=5), ARG), (dict(n_groups=-1), ARG), (dict(start=None), ARG), (dict(batch=65536), SHAPE),
    (dict(d=desc(n_q_heads=128, n_kv_heads=8)), SHAPE), (dict(d=desc(head_dim=80)), SHAPE), (dict(po=pool(page_rows=8)), SHAPE),
    (dict(po=pool(max_blocks=(1 << 26) - 1)), SHAPE), (dict(po=pool(v=None)), ARG),
    (dict(options=lava.DecodeOptions(0.0, 5, None), q_pos=None), ARG), (dict(options=lava.DecodeOptions(0.0, 5, None), po=pool(pos=ODD)), ARG),
    (dict(options=lava.DecodeOptions(-1.0, 0, None)), ARG), (dict(options=lava.DecodeOptions(float("nan"), 0, None)), ARG),
    (dict(options=lava.DecodeOptions(0.0, -1, None)), ARG), (dict(ws=None), SPACE), (dict(ws=FAKE + 128), SPACE), (dict(ws_bytes=1000), SPACE)])
def test_shared_decode_refuses(kw, want):
    assert shared(**kw) == want


def test_shared_decode_workspace():
    size = lava.lava_shared_decode_workspace_bytes
    assert size(desc(), 0, 4) == size(desc(), 65536, 4) == size(desc(), 4, 0) == size(desc(head_dim=80), 4, 4) == size(desc(), 65535, 4) == 0
    assert size(desc(), 4, 1 << 27) == 0
    assert lava.lava_paged_decode_workspace_bytes(desc()) < size(desc(), 1, 1) <= size(desc(), 4, 4) <= size(desc(), 64, 4) <= size(desc(), 64, 4096)
    assert shared(ws_bytes=size(desc(), 4, 4) - 1) == SPACE
