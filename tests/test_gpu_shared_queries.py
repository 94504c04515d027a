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




@IDLE
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("kw", [{}, dict(window=1500, softcap=20.0)], ids=["plain", "window and cap"])
def test_one_query_that_is_no_number(lava, dtype, d, idle, kw):
    """The sequence's own results are NaN where it sees rows.  The others' are what they are beside a query of zeros, whose logits' maximum moves no
    more often either: at the first rows that are seen."""
    c = case(lava, dtype, d, idle, kw)
    c.q_pos.fill_(2000)
    c.q[4], c.q[9, :4] = 0.0, 0.0                                      # all heads of one sequence, one KV head's of another
    want, want_lse = c.run()
    assert bool(torch.isfinite(want_lse[[0, 3, 4, 9]]).all())
    c.q[4], c.q[9, :4] = float("nan"), float("nan")
    out, lse = c.run()
    hit = torch.zeros(c.batch, 8, dtype=torch.bool, device=out.device)
    hit[4], hit[9, :4] = True, True
    assert torch.equal(torch.isnan(lse), hit) and torch.equal(torch.isnan(out), hit[..., None].expand_as(out))
    assert torch.equal(out[~hit], want[~hit]) and torch.equal(lse[~hit], want_lse[~hit])


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("kw", [dict(window=300), dict(window=300, bias=True, softcap=20.0)], ids=["window", "all"])
def test_values_that_one_sequence_does_not_see(lava, dtype, d, kw):
    """An infinity that the window of one group member leaves out: that member is looked at row by row, and gets what it gets without it."""
    c = case(lava, dtype, d, 0, kw)
    c.pos.copy_(torch.randint(0, 200, c.pos.shape, device=c.pos.device, generator=torch.Generator(c.pos.device).manual_seed(3)))
    c.q_pos.fill_(199)
    c.q_pos[3] = 420                                                   # sees positions from 121 on
    c.check(*c.run())
    low = c.pos < 100
    v = c.v.clone()
    c.v[low] = float("inf")
    out, lse = c.run()
    c.v[low] = v[low]
    want, want_lse, tol, tol_lse = c.want()
    some = want_lse.isfinite()
    assert bool(((out[3].double().cpu() - want[3]).abs() <= tol[3] + 2.0 ** -22 * 6).all())
    assert bool(((lse.double().cpu() - want_lse).abs()[some] <= (tol_lse + want_lse.abs() * 2.0 ** -21)[some]).all())
    assert not bool(torch.isfinite(out[0]).all())
