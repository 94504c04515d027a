"""Which launches the paged cache's calls take, as the library's own launch counts say, where the choice decides how long a call takes."""
import numpy as np
import pytest

from oracle import paged_oracle as P
from test_paged_oracle_pins import random_state

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
DEV = "cuda"


@pytest.fixture(scope="module")
def lava():
    from paper_2509_09754_amd import lava as L
    return L


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


@pytest.mark.parametrize("batch,heads,page,max_blocks,new_hi,launches", [(1, 8, 16, 1030, 16000, 2), (16, 8, 64, 40, 2000, 2), (4, 8, 64, 12, 4, 1)])
def test_growth_without_maps(lava, batch, heads, page, max_blocks, new_hi, launches):
    """New tokens without slots or positions: nothing bounds how many pages a head takes but its table, so the table decides whether one
    workgroup does the step alone."""
    print(f"tables without maps: {batch} x {heads} heads, {max_blocks} blocks", flush=True)
    rng = np.random.default_rng(batch + max_blocks)
    n_pages = batch * heads * max_blocks
    table, rows, pos, free, n_free = random_state(rng, batch, heads, max_blocks, page, n_pages, 0.2)
    new = np.minimum(rng.integers(0, new_hi + 1, batch), max_blocks * page - rows.max(1)).astype(np.int32)
    st = lava.PageState(*(dev(a) for a in (table, rows, pos, free, np.array([n_free], np.int32))), page)
    torch.cuda.synchronize()
    lava.prof_enable(True), lava.prof_reset()
    lava.lava_page_tables(st, dev(new))
    torch.cuda.synchronize()
    count = {name: n for name, (_, n) in lava.prof_read().items()}
    lava.prof_enable(False)
    want = P.page_tables(page, n_pages, table, rows, pos, free, n_free, new)
    for got, a in zip((st.block_table, st.head_rows, st.seq_pos, st.free_pages), want):
        assert np.array_equal(got.cpu().numpy(), a)
    assert int(st.n_free[0]) == want[4]
    assert (count["page_plan"], count["page_fill"]) == (1, launches - 1)
