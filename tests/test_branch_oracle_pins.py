"""The oracle of sequences that share pages against what its definitions imply: pages are held or free and never both, rows read through the
tables are the rows asked for, a beam step over all of a small tree finds its best paths."""
import itertools
import math

import numpy as np
import pytest

from oracle import branch_oracle as B
from oracle import paged_oracle as P
from test_paged_oracle_pins import random_state


def content(table, rows, page, cells):
    """Rows of every head, read through its table; cells [pages * page]."""
    return [[[int(cells[int(table[b, g, r // page]) * page + r % page]) for r in range(int(rows[b, g]))] for g in range(rows.shape[1])]
            for b in range(rows.shape[0])]


def check_pages(table, rows, page, free, n_free, n_pages):
    """Every page is in some table or on the stack, a page that is not full in one table only."""
    seen, open_pages = set(), []
    for b in range(rows.shape[0]):
        for g in range(rows.shape[1]):
            nb = -(-int(rows[b, g]) // page)
            pages = [int(p) for p in table[b, g, :nb]]
            assert len(set(pages)) == nb
            seen |= set(pages)
            if rows[b, g] % page:
                open_pages.append(pages[-1])
    assert len(set(open_pages)) == len(open_pages)
    held = [int(p) for b in range(rows.shape[0]) for g in range(rows.shape[1]) for p in table[b, g, : -(-int(rows[b, g]) // page)]]
    assert all(held.count(p) == 1 for p in open_pages)
    assert sorted(int(x) for x in free[:n_free]) == sorted(set(range(n_pages)) - seen)


def random_lists(rng, rows, share):
    """(head_counts, kept_idx) of a selection: some heads keep all, some nothing, some a run from the front and others."""
    counts, lists = np.zeros_like(rows), []
    for b in range(rows.shape[0]):
        mine = []
        for g in range(rows.shape[1]):
            n, how = int(rows[b, g]), rng.integers(0, 5)
            front = int(rng.integers(0, n + 1)) if how in (2, 3) else 0
            rest = front + np.flatnonzero(rng.random(n - front) < (0 if how == 3 else share))
            kept = list(range(n)) if how == 0 else [] if how == 1 else list(range(front)) + rest.tolist()
            counts[b, g] = len(kept)
            mine += kept
        lists.append(mine)
    cap = max(len(x) for x in lists) + 2
    return counts, np.array([x + [-5] * (cap - len(x)) for x in lists], np.int32)


@pytest.mark.parametrize("batch,heads,page", [(1, 1, 16), (5, 3, 16), (9, 4, 32), (16, 2, 64)])
def test_changes_keep_rows_and_pages(batch, heads, page):
    rng = np.random.default_rng(batch)
    mb = 9
    n_pages = batch * heads * mb + 7
    table, rows, pos, free, n_free = random_state(rng, batch, heads, mb, page, n_pages, 0.5)
    cells = rng.integers(0, 1 << 30, n_pages * page)
    for step in range(25):
        was = content(table, rows, page, cells)
        kind = rng.integers(0, 3)
        if kind == 0:
            source = rng.integers(-1, batch, batch).astype(np.int32) if step % 2 else rng.permutation(batch).astype(np.int32)
            out = B.page_change(page, n_pages, table, rows, pos, free, n_free, source=source)
            want = [was[s] if s >= 0 else [[] for _ in range(heads)] for s in source]
        elif kind == 1:
            counts, kept = random_lists(rng, rows, 0.6)
            evict = (rng.random(batch) < 0.7).astype(np.int32)
            out = B.page_change(page, n_pages, table, rows, pos, free, n_free, head_counts=counts, kept_idx=kept, evict=evict)
            want = []
            for b in range(batch):
                ends = np.cumsum(counts[b])
                want.append([[was[b][g][r] for r in kept[b, ends[g] - counts[b, g]: ends[g]]] if evict[b] else was[b][g] for g in range(heads)])
        else:                                                         # new tokens, by the tables as they are
            room = mb * page - rows.max(1)
            new = np.minimum(rng.integers(0, 2 * page, batch), room)
            got = P.page_tables(page, n_pages, table, rows, pos, free, n_free, new, max_tokens=int(new.sum()) + 1)
            if got[7] == 0:
                table, rows, pos, free, n_free, slots = got[:6]
                cells[slots[slots >= 0]] = rng.integers(0, 1 << 30, int((slots >= 0).sum()))
                now = content(table, rows, page, cells)
                for b in range(batch):
                    for g in range(heads):
                        assert now[b][g][: len(was[b][g])] == was[b][g]
            check_pages(table, rows, page, free, n_free, n_pages)
            continue
        if out[6]:
            assert all(np.array_equal(a, b) for a, b in zip(out[:4], (table, rows, pos, free))) and out[4] == n_free
            continue
        table, rows, pos, free, n_free, moves, _ = out
        written = [m[0] for m in moves]
        assert len(set(written)) == len(written) and not set(written) & {m[1] for m in moves}
        for dst, src in moves:
            cells[dst] = cells[src]
        assert content(table, rows, page, cells) == want
        check_pages(table, rows, page, free, n_free, n_pages)


def test_changes_refuse():
    table, rows, pos, free = np.array([[[0, 1]], [[2, 9]]], np.int32), np.array([[20], [3]], np.int32), np.zeros(2, np.int32), np.array([3, 4, 5, 6, 7, 8, -1, -1, -1], np.int32)
    call = lambda **kw: B.page_change(16, 9, kw.pop("table", table), kw.pop("rows", rows), pos, kw.pop("free", free), kw.pop("n_free", 6), **kw)[6]
    i32 = lambda *x: np.array(x, np.int32)
    assert call(source=i32(0, 0)) == 0 and call(source=i32(1, -1)) == 0
    assert call(source=i32(2, 0)) == call(source=i32(0, -2)) == B.INVALID
    assert call(source=i32(0, 0), n_free=0) == B.EXHAUSTED and call(source=i32(0, 1), n_free=0) == 0
    assert call(source=i32(0, 1), n_free=10) == B.INVALID and call(source=i32(0, 1), rows=i32(33, 3).reshape(2, 1)) == B.INVALID
    assert call(source=i32(0, 1), rows=i32(20, 17).reshape(2, 1)) == B.INVALID            # page 9 is not in the pool
    assert call(source=i32(0, 0), free=i32(3, 4, 5, 6, 7, 9, 0, 0, 0)) == B.INVALID
    kept = np.zeros((2, 4), np.int32)
    assert call(head_counts=i32(1, 1).reshape(2, 1), kept_idx=kept) == 0
    for bad in ((-1, 1), (21, 1), (5, 1)):
        assert call(head_counts=i32(*bad).reshape(2, 1), kept_idx=kept) == B.INVALID
    assert call(head_counts=i32(-1, 1).reshape(2, 1), kept_idx=kept, evict=i32(0, 1)) == 0


def test_beams_as_wide_as_the_tree_find_its_best_paths():
    """With as many beams as there are paths nothing is pruned: the scores are those of all paths, by brute force."""
    rng = np.random.default_rng(3)
    V, steps = 3, 3
    tables = rng.normal(size=(steps, V ** (steps - 1), V))
    logp = tables - np.log(np.exp(tables).sum(-1, keepdims=True))
    beams = V ** steps
    scores = np.full((1, beams), -np.inf)
    scores[0, 0] = 0.0
    paths = [()] * beams
    for t in range(steps):
        logits = np.zeros((1, beams, V))
        for i, path in enumerate(paths):
            at = 0
            for x in path:
                at = at * V + x
            logits[0, i] = tables[t, at]
        parents, tokens, scores, over, _ = B.beam_step(logits, scores, beams)
        paths = [paths[p] + (int(v),) if p >= 0 else () for p, v in zip(parents[0], tokens[0])]
    brute = {}
    for path in itertools.product(range(V), repeat=steps):
        at, s = 0, 0.0
        for t, x in enumerate(path):
            s += logp[t, at, x]
            at = at * V + x
        brute[path] = s
    assert sorted(brute.values(), reverse=True) == pytest.approx(scores[0].tolist(), abs=1e-12)
    assert sorted(paths) == sorted(brute) and all(brute[p] == pytest.approx(s, abs=1e-12) for p, s in zip(paths, scores[0]))


def test_beam_order_of_equals():
    x = np.zeros((1, 2, 4))
    x[0, 1, 2] = -np.inf
    p, v, s, over, gap = B.beam_step(x, np.array([[0.0, 0.0]]), 8, end_token=1)
    assert p[0].tolist() == [1, 1, 1, 0, 0, 0, 0, -1] and v[0].tolist() == [0, 1, 3, 0, 1, 2, 3, -1]
    assert over[0].tolist() == [0, 1, 0, 0, 1, 0, 0, 1] and s[0, 0] == pytest.approx(-math.log(3)) and s[0, 7] == -np.inf
