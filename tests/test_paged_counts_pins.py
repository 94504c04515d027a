"""The counting oracle of the decode over pages: against the plain one, and against mistakes planted in what it is given.  A row lost,
read twice or taken from elsewhere has to leave its bounds even among 70000 rows, where the plain oracle's bound is too wide for a
whole tile."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as P
from oracle.paged_counts import SCALE, Pages


@pytest.mark.parametrize("kw", [{}, dict(window=300), dict(softcap=50.0), dict(window=900, softcap=50.0)])
def test_counts_agree_with_the_plain_oracle(kw):
    pages = Pages(1, 30, 16, 64)
    rng = np.random.default_rng(2)
    rows = np.array([[0, 1, 37, 100], [160, 16, 3, 5]])
    table = torch.from_numpy(rng.integers(0, 30, (2, 4, 11)))
    q, q_pos = pages.queries(2, 12, 3), torch.tensor([700, 1200])
    out, lse, tol, tol_lse = pages.attend(table, rows, 3, q_pos=q_pos, **kw)
    want, want_lse, _, _ = P.paged_decode(q.numpy(), pages.k.numpy(), pages.v.numpy(), table.numpy(), rows, SCALE, kw.get("softcap", 0.0),
                                          kw.get("window", 0), None, pages.pos.numpy(), q_pos.numpy())
    assert (np.abs(out.numpy() - want) <= tol.numpy() + 1e-12).all()
    some = np.isfinite(want_lse)
    assert np.array_equal(some, np.isfinite(lse.numpy()))
    assert (np.abs(lse.numpy()[some] - want_lse[some]) <= tol_lse.numpy()[some] + 1e-12).all()


def moved(pages, good, table, rows, **kw):
    """How far a mistake moves the two results, in multiples of what is allowed."""
    out, lse, tol, tol_lse = good
    bad = pages.attend(table, rows, 8, **kw)
    return float(((bad[0] - out).abs() / tol).max()), float(((bad[1] - lse).abs() / tol_lse).max())


@pytest.mark.parametrize("rows,page,kw", [(70000, 128, {}), (33000, 16, {}), (33000, 16, dict(window=400)), (131072, 64, dict(softcap=50.0)), (300, 32, {})])
def test_a_planted_mistake_is_seen(rows, page, kw):
    n_pages, d = 300, 64
    blocks = -(-rows // page)
    pages = Pages(3, n_pages, page, d)
    rng = np.random.default_rng(rows)
    kw = dict(kw, q_pos=torch.tensor([990]))
    table = torch.from_numpy(rng.integers(0, n_pages, (1, 1, blocks)))
    good = pages.attend(table, [[rows]], 8, **kw)
    block = blocks // 3
    without = lambda n: (torch.cat([table[..., :block], table[..., block + n:]], -1), [[rows - n * page]])
    tile = max(1, 32 // page)
    mistakes = {"a page lost": without(1), "a tile's pages lost": without(tile),
                "a page twice": (torch.cat([table[..., : block + 1], table[..., block:]], -1), [[rows + page]]),
                "another head's page": (torch.where(torch.arange(blocks) == block, (table + 1) % n_pages, table), [[rows]]),
                "its last row lost": (table, [[rows - 1]])}
    if not kw.get("window"):                                         # the last row may be out of the window
        mistakes["two rows lost"] = (table, [[rows - 2]])
    else:
        mistakes.pop("its last row lost")
    for name, (t, r) in mistakes.items():
        by = moved(pages, good, t, r, **kw)
        print(name, by)
        assert by[0] > 2.0, (name, by)
    # values paired with the next row's probability, in one page; the probabilities of another query head
    used = int(table[0, 0, block])
    pages.v[used] = pages.v[used].roll(1, 0)
    assert moved(pages, good, table, [[rows]], **kw)[0] > 2.0
    pages.v[used] = pages.v[used].roll(-1, 0)
    assert moved(pages, good, table, [[rows]], **kw)[0] == 0.0
    pages.on[:2, used] = pages.on[:2, used].flip(0)
    assert moved(pages, good, table, [[rows]], **kw)[0] > 2.0
