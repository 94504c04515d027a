"""Decode over pages where the right answer is a count (oracle/paged_counts.py): no row of any head may be lost, read twice or paired with
another's value, in each of the three cuts, for groups of every padded size, both types and head sizes, with and without the strided order
of a window.  Which cut a case takes is worked out here with the kernel's rule, for every number of workgroups a compute unit may hold,
so that a case that no longer takes the cut it is for is noticed."""
import math

import numpy as np
import pytest

from oracle.paged_counts import SCALE, Pages

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
DEV = "cuda"


@pytest.fixture(scope="module")
def lava():
    from paper_2509_09754_amd import lava as L
    return L


def cut(rows, workgroups, window=0, q_pos=0):
    """(cut, whether a head's tiles take their places strided): the rule of the kernel, in its words."""
    places, strided = [], False
    for n in np.asarray(rows).reshape(-1).tolist():
        tiles = -(-n // 32)
        if window and tiles >= 68:
            tiles, strided = -(-tiles // 17) * 17, True
        if window:
            seen = q_pos + 1
            tiles = -(-tiles // (8 if seen >= 8 * window else 4 if seen >= 4 * window else 2 if seen >= 2 * window else 1))
        places.append(tiles)
    total, full, longest = sum(places), sum(p > 0 for p in places), max(places)
    least = int(math.sqrt(0.25 * longest))
    even, line = max(-(-total // workgroups), least), max(-(-(total + 6 * full) // workgroups), least)
    if 8 * longest * -(-full // (4 * workgroups)) <= 3 * line:
        return "wavefronts", strided
    for share in (even, line):
        share = (share + 3) & ~3
        if sum(-(-p // share) for p in places) <= workgroups:
            return "heads", strided
    return "line", strided


def between(seed, batch, heads, lo, hi, idle=0):
    rows = np.random.default_rng(seed).integers(lo, hi + 1, (batch, heads))
    rows[batch - idle:] = 0
    return rows


LOADS = {                                                            # rows of every head, the cut they are for
    "wavefronts, ten tiles": (between(1, 256, 8, 250, 330), "wavefronts"),
    "wavefronts, one and two tiles": (between(2, 512, 8, 1, 60), "wavefronts"),
    "wavefronts, more than a block of pages": (between(3, 512, 8, 2180, 2400), "wavefronts"),
    "line, ragged": (between(4, 61, 8, 100, 4000, idle=2), "line"),
    "line, some heads of none": (between(5, 230, 5, 0, 900), "line"),
    "one head": (np.array([[70000]]), "heads"),
    "eight heads": (np.full((1, 8), 8190), "heads"),
    "two sequences of uneven heads": (np.array([[9000, 40, 1, 700, 31, 20000, 33, 5], [64, 3000, 8, 12000, 0, 65, 4097, 100]]), None),
}
SHAPES = [(1, 128, "bf16", 16), (4, 128, "bf16", 64), (7, 128, "bf16", 16), (8, 64, "bf16", 32), (2, 64, "bf16", 256), (5, 64, "f32", 16),
          (8, 128, "f32", 128), (1, 64, "f32", 32)]


@pytest.mark.parametrize("G,d,dtype,page", SHAPES)
@pytest.mark.parametrize("load", LOADS)
@pytest.mark.parametrize("kw", [{}, dict(window=300), dict(window=130, softcap=50.0, bias=True)], ids=["plain", "window", "all"])
def test_every_row_counts_once(lava, G, d, dtype, page, load, kw):
    rows, expected = LOADS[load]
    print(f"counts: {load}, {G} heads a group, d {d} {dtype}, pages of {page}, {kw}", flush=True)
    batch, Hkv = rows.shape
    n_pages, q_last = 400, 999
    window, softcap = kw.get("window", 0), kw.get("softcap", 0.0)
    cus = torch.cuda.get_device_properties(0).multi_processor_count
    cuts = {cut(rows, n * cus, window, q_last) for n in (1, 2, 3, 4)}
    if not window and expected:
        assert cuts == {(expected, False)}
    elif window and expected in ("heads", "wavefronts") and load != "wavefronts, one and two tiles":
        assert {c for c, _ in cuts} == {expected}
    if window and rows.max() > 68 * 32:
        assert all(strided for _, strided in cuts)
    pages = Pages(G + page, n_pages, page, d, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(len(load))
    blocks = int(rows.max() - 1) // page + 1
    table = torch.randint(0, n_pages, (batch, Hkv, blocks), generator=g, device=DEV, dtype=torch.int32)
    # the new tokens' positions: the last one for the first sequence, half of them earlier
    q_pos = torch.where(torch.arange(batch, device=DEV) % 2 == 0, q_last, 700).to(torch.int32)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    desc = lava.LayerDesc.make(G * Hkv, Hkv, d, 1, dtype, softmax_scale=SCALE)
    pool = lava.PagePool(pages.k.to(dt), pages.v.to(dt), pages.pos, max_blocks=blocks)
    slopes = torch.zeros(G * Hkv, device=DEV) if kw.get("bias") else None
    options = lava.DecodeOptions.make(softcap, window, slopes) if kw else None
    q = pages.queries(batch, G * Hkv, G).to(dt)
    ws = torch.full((lava.lava_paged_decode_workspace_bytes(desc),), 0xFF, dtype=torch.uint8, device=DEV)
    out, lse = lava.lava_paged_decode(desc, q, pool, table, dev_rows(rows), options, q_pos if window else None, workspace=ws)
    want, want_lse, tol, tol_lse = pages.attend(table, rows, G, window, q_pos, softcap)
    torch.cuda.synchronize()
    some = torch.isfinite(want_lse)
    assert bool((torch.isfinite(lse) == some).all())
    worst = ((out.double() - want).abs() / tol.clamp(min=1e-300)).max()
    print(f"   cuts {sorted(c for c, _ in cuts)}, worst {float(worst):.3f} of the bound", flush=True)
    assert bool(((out.double() - want).abs() <= tol).all())
    assert bool(((lse.double() - want_lse).abs() <= tol_lse)[some].all())


def dev_rows(rows):
    return torch.from_numpy(np.ascontiguousarray(rows, dtype=np.int32)).to(DEV)
