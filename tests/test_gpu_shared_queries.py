"""Decode over shared pages on the GPU: queries that are no numbers, of sequences that hold nothing and of sequences that do, and what they cost the
sequences beside them (nothing, bit for bit)."""
import numpy as np
import pytest

from test_gpu_shared import Case, shared_tables

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

IDLE = pytest.mark.parametrize("idle", [0, 260], ids=["few", "many"])   # own rows of more than 512 heads are decoded by themselves


@pytest.fixture(scope="module")
def lava():
    from paper_2509_09754_amd import lava as L
    return L


def case(lava, dtype, d, idle, kw):
    """Two groups whose sequences 1, 2 and 8 hold nothing, and more that hold nothing."""
    rng = np.random.default_rng(41)
    sizes = [6, 5, idle]
    table, rows, n_pages = shared_tables(rng, sizes, 2, 16, lambda i, g: 40 + 3 * g, 1, 60, idle=[1, 2, 8, *range(11, 11 + idle)])
    return Case(lava, rng, 8, 2, d, dtype, 16, sizes, table, rows, n_pages, **kw)


@IDLE
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("kw", [{}, dict(window=1500, bias=True, softcap=20.0)], ids=["plain", "all"])
def test_queries_of_sequences_that_hold_nothing(lava, dtype, d, idle, kw):
    """Whatever stands there (memory that nobody wrote), the others' results do not move by a bit."""
    c = case(lava, dtype, d, idle, kw)
    empty = c.rows[:, 0] == 0
    c.q[empty] = 0.0
    want, want_lse = c.run()
    for value in (float("nan"), float("inf"), torch.finfo(c.q.dtype).max):
        c.q[empty] = value
        c.q_pos[empty] = -5
        out, lse = c.run()
        assert torch.equal(out, want) and torch.equal(lse, want_lse), value
    c.q[empty] = 0.0
    c.check(out, lse)


