"""The paged cache's oracle against what its definitions imply: conservation of pages, the relative-position property of a
rotation, agreement with the packed cache's oracle."""
import math

import numpy as np
import pytest

from oracle import lava_oracle as O
from oracle import paged_oracle as P


def random_state(rng, batch, heads, max_blocks, page, n_pages, fill=0.6):
    """A state in which every page is owned once or free."""
    rows = rng.integers(0, max_blocks * page + 1, (batch, heads)).astype(np.int32)
    rows = (rows * fill).astype(np.int32)
    while (-(-rows // page)).sum() > n_pages:
        rows = rows // 2
    order = rng.permutation(n_pages).astype(np.int32)
    table, used = np.full((batch, heads, max_blocks), -7, np.int32), 0
    for b in range(batch):
        for g in range(heads):
            nb = -(-int(rows[b, g]) // page)
            table[b, g, :nb] = order[used: used + nb]
            used += nb
    free = np.full(n_pages, -9, np.int32)
    free[: n_pages - used] = order[used:]
    return table, rows, rng.integers(0, 1000, batch).astype(np.int32), free, n_pages - used


def owned(table, rows, page):
    return [int(p) for b in range(rows.shape[0]) for g in range(rows.shape[1]) for p in table[b, g, : -(-int(rows[b, g]) // page)]]


def test_pages_are_conserved():
    rng = np.random.default_rng(1)
    for batch, heads, page in ((1, 1, 16), (5, 3, 16), (9, 8, 32)):
        n_pages, mb = 300, 12
        table, rows, pos, free, n_free = random_state(rng, batch, heads, mb, page, n_pages, 0.3)
        for step in range(12):
            new = rng.integers(0, 4 * page, batch)
            release = (rng.random(batch) < 0.3).astype(np.int32)
            out = P.page_tables(page, n_pages, table, rows, pos, free, n_free, new, release=release, max_tokens=int(new.sum()) + 2)
            if out[7]:
                assert all(np.array_equal(a, b) for a, b in zip(out[:4], (table, rows, pos, free))) and (out[5] == -1).all()
                release = np.ones(batch, np.int32)
                out = P.page_tables(page, n_pages, table, rows, pos, free, n_free, None, release=release)
                assert out[7] == 0 and out[4] == n_pages
            table, rows, pos, free, n_free, slots, positions, _ = out
            pages = owned(table, rows, page) + [int(x) for x in free[:n_free]]
            assert sorted(pages) == list(range(n_pages))
            live = slots[slots >= 0]
            assert len(set(live.tolist())) == live.size


def test_refusals_name_their_reason():
    table, rows, pos, free = np.zeros((1, 1, 2), np.int32), np.array([[16]], np.int32), np.zeros(1, np.int32), np.arange(4, dtype=np.int32)
    step = lambda **kw: P.page_tables(16, 4, table, rows, pos, free, kw.pop("n_free", 3), **kw)[7]
    assert step(n_new=[1], max_tokens=1) == 0
    assert step(n_new=[17], max_tokens=17) == P.BLOCKS
    assert step(n_new=[1], n_free=0) == P.EXHAUSTED
    assert step(n_new=[-1]) == P.INVALID and step(head_counts=[[-1]]) == P.INVALID
    assert step(n_new=[2], max_tokens=1) == P.TOKENS
    assert step(release=[1], n_free=4) == P.INVALID


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_keeps_relative_positions(interleaved):
    rng = np.random.default_rng(2)
    f = P.rotary_frequencies(64, 10000.0)
    x, y = rng.standard_normal((2, 1, 1, 64))
    dot = lambda p, q: float((P.rotary(x, [p], f, interleaved) * P.rotary(y, [q], f, interleaved)).sum())
    assert abs(dot(1000, 900) - dot(100100, 100000)) < 1e-9
    assert np.allclose(P.rotary(x, [0], f, interleaved), x)
    back = P.rotary(P.rotary(x, [777], f, interleaved, 1.5), [777], f, interleaved, 1.5, transpose=True)
    assert np.allclose(back, 1.5 ** 2 * x)


def test_rotation_by_difference_quotients():
    """The transposed rotation is the gradient of <g, rotary(x)>."""
    rng = np.random.default_rng(3)
    f = P.rotary_frequencies(6)
    x, g = rng.standard_normal((2, 2, 1, 8))
    grad = P.rotary(g, [3, 70], f, True, 1.2, transpose=True)
    for i in np.ndindex(x.shape):
        e = np.zeros_like(x)
        e[i] = 1e-5
        d = ((P.rotary(x + e, [3, 70], f, True, 1.2) - P.rotary(x - e, [3, 70], f, True, 1.2)) * g).sum() / 2e-5
        assert abs(d - grad[i]) < 1e-8


def test_frequencies_by_parts():
    f = P.rotary_frequencies(64, 500000.0)
    s = P.rotary_frequencies(64, 500000.0, 8.0, 8192, 1.0, 4.0)
    turns = 8192 * f / (2 * math.pi)
    assert np.allclose(s[turns > 4], f[turns > 4]) and np.allclose(s[turns < 1], f[turns < 1] / 8)
    assert ((s <= f) & (s >= f / 8)).all()


def test_decode_over_pages_is_decode_over_packed_rows():
    rng = np.random.default_rng(4)
    H, Hkv, d, page = 6, 2, 8, 16
    rows = np.array([[37, 5]], np.int32)
    table, n_pages = np.array([[[3, 0, 5], [1, -1, -1]]], np.int32), 6
    k, v = rng.standard_normal((2, n_pages, page, d))
    q = rng.standard_normal((1, H, d))
    out, lse, tol, _ = P.paged_decode(q, k, v, table, rows, 1 / math.sqrt(d))
    packed = [np.concatenate([x[[3, 0, 5]].reshape(-1, d)[:37], x[1][:5]]) for x in (k, v)]
    want, want_lse = O.decode_attention(q[0], packed[0], packed[1], np.array([0, 37, 42]))
    assert np.allclose(out[0], want) and np.allclose(lse[0], want_lse) and (tol > 0).all()
    # nothing seen; a bias alone keeps the order of distances
    pos = np.zeros((n_pages, page), np.int32)
    out, lse, _, _ = P.paged_decode(q, k, v, table, rows, 1.0, window=3, pos_pages=pos, q_pos=[100])
    assert (out == 0).all() and np.isneginf(lse).all()
    out, _, _, _ = P.paged_decode(q * 0, k, v, table, rows, 1.0, softcap=5.0)
    assert np.allclose(out[0, 0], packed[1][:37].mean(0))


def test_gather_is_the_packed_gather():
    rng = np.random.default_rng(5)
    offs, n = np.array([0, 20, 23]), 40
    idx = np.concatenate([np.sort(rng.permutation(n)[:20]), np.sort(rng.permutation(n)[:3])])
    moves = P.compact_paged(4, 16, 2, offs, idx, [(0, n), (n, n)], np.array([[2, 0], [3, -1]]))
    x = rng.standard_normal((2, n, 4))
    packed = O.compact(x, offs, idx)
    for t, (slot, src, i) in enumerate(moves):
        assert np.array_equal(x.reshape(-1, 4)[src], packed[t]) and i == idx[t]
    assert [m[0] for m in moves] == [2 * 16 + r for r in range(16)] + [r for r in range(4)] + [48, 49, 50]
