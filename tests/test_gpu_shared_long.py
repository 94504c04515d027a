"""Decode over shared pages on the GPU, heads of millions of rows: a workgroup's unit has more stages than it holds pages for at a time (64), with and
without a window that leaves most of them out.  A table may name a page again and again, so that a small pool is as long as is needed."""
import numpy as np
import pytest

from oracle.paged_counts import SCALE, Pages
from test_gpu_shared import dev

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
DEV = "cuda"


@pytest.fixture(scope="module")
def lava():
    from paper_2509_09754_amd import lava as L
    return L


def run(lava, dtype, d, G, pages, table, rows, window, q_pos):
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    desc = lava.LayerDesc.make(G, 1, d, 1, dtype, softmax_scale=SCALE)
    pool = lava.PagePool(pages.k.to(dt), pages.v.to(dt), pages.pos, max_blocks=table.shape[2])
    options = lava.DecodeOptions.make(window=window) if window else None
    batch = len(rows)
    out, lse = lava.lava_shared_decode(desc, pages.queries(batch, G, G).to(dt), pool, dev(table), dev(rows),
                                       dev(np.array([0, batch], np.int32)), options, q_pos)
    want, want_lse, tol, tol_lse = pages.attend(dev(table), rows, G, window, q_pos if window else None)
    torch.cuda.synchronize()
    assert bool(torch.isfinite(want_lse).all())
    # rows that are off weigh nothing, counts below 2^24 are exact: one division more, of the two parts put together
    assert bool(((out.double() - want).abs() <= tol + want * 2.0 ** -21).all()), float((out.double() - want).abs().max())
    assert bool(((lse.double() - want_lse).abs() <= 2.0 * tol_lse).all())


# rows of a stage: 64 KiB of keys and values
@pytest.mark.parametrize("dtype,d,stage", [("f32", 128, 64), ("bf16", 128, 128), ("f32", 64, 128)])
@pytest.mark.parametrize("form", ["plain", "own rows", "windowed", "nothing in the first 64"])
def test_units_of_many_stages(lava, dtype, d, stage, form):
    cus = torch.cuda.get_device_properties(0).multi_processor_count
    windowed, rng, page = form not in ("plain", "own rows"), np.random.default_rng(60), stage
    each = 70                                                         # stages of a unit
    units = 2 * cus if windowed else cus - 1                          # of one item: twice the workgroups where there is a window
    stages = each * units - 3
    n_pages = 240
    pages = Pages(61, n_pages, page, d, device=DEV)
    shown = np.isin(np.arange(stages) % each, [0, 63, 64, 69] if form == "windowed" else [66, 69])
    if windowed:                                                      # the window shows the pages from 120 on only, and of those some rows
        pages.pos[:120] = pages.pos[:120] % 400
        pages.pos[120:] = 600 + pages.pos[120:] % 400
        common = np.where(shown, rng.integers(120, n_pages - 8, stages), rng.integers(0, 120, stages))
    else:
        common = rng.integers(0, n_pages - 8, stages)
    table = np.full((2, 1, stages + 3), -1, np.int32)
    table[:, 0, :stages] = common
    if form == "own rows":                                            # nothing in common
        table[1, 0, 0] = n_pages - 5
    own = np.array([[page + 5], [1]])
    table[0, 0, stages: stages + 2], table[1, 0, stages] = [n_pages - 8, n_pages - 7], n_pages - 6
    rows = (stages * page + own).astype(np.int32)
    print(f"{form}: {dtype} d {d}, {rows[0, 0]} rows, {stages} stages", flush=True)
    run(lava, dtype, d, 4, pages, table, rows, 350 if windowed else 0, torch.tensor([999, 950], dtype=torch.int32, device=DEV))


@pytest.mark.parametrize("window", [0, 1000], ids=["plain", "window"])
def test_as_many_rows_as_can_be(lava, window):
    """2^31 - 256 rows: the first, the last and one between have a value, and one of the two queries is no number."""
    page, d, blocks = 256, 64, (1 << 23) - 1
    desc = lava.LayerDesc.make(1, 1, d, 1, "bf16")
    k = torch.zeros(4, page, d, dtype=torch.bfloat16, device=DEV)
    v = torch.ones(4, page, d, dtype=torch.bfloat16, device=DEV)
    k[1:, ::page // 2] = 1.0                                          # two rows of page 1 to 3
    pos = torch.zeros(4, page, dtype=torch.int32, device=DEV)
    for i in (1, 2, 3):
        v[i, ::page // 2] = 8.0 * i
        pos[i, ::page // 2] = 5000
    table = torch.zeros(2, 1, blocks, dtype=torch.int32, device=DEV)
    table[:, 0, 0], table[:, 0, 5_000_001], table[:, 0, -1] = 1, 2, 3
    rows = torch.full((2, 1), blocks * page, dtype=torch.int32, device=DEV)
    q = torch.full((2, 1, d), 8.0, dtype=torch.bfloat16, device=DEV)   # logit 64 for those six rows, 0 for 2^31: e^-64 of them each, 3.4e-19 in all
    q[1] = float("nan")
    pool = lava.PagePool(k, v, pos, max_blocks=blocks)
    options = lava.DecodeOptions.make(window=window) if window else None
    q_pos = torch.full((2,), 5500, dtype=torch.int32, device=DEV)
    start = torch.tensor([0, 2], dtype=torch.int32, device=DEV)
    out, lse = lava.lava_shared_decode(desc, q, pool, table, rows, start, options, q_pos)
    torch.cuda.synchronize()
    assert bool(torch.isnan(out[1]).all()) and bool(torch.isnan(lse[1]).all())
    assert bool(((out[0] - 16.0).abs() <= 16.0 * 2.0 ** -20).all()), out[0, 0, :4].tolist()
    assert abs(float(lse[0, 0]) - (64.0 + np.log(6.0))) <= 66 * 2.0 ** -21
