"""Forks and compaction of states whose tables have more entries than one workgroup marks (8192): refusals, lists, last pages and replays there, against
the oracle, bit for bit.  The tables are those of small states with room for more blocks."""
import numpy as np
import pytest

from oracle import branch_oracle as B
from test_branch_oracle_pins import check_pages, random_lists
from test_gpu_forks import Cache, dev, host, sources
from test_paged_oracle_pins import random_state

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
DEV = "cuda"


@pytest.fixture(scope="module")
def lava():
    from paper_2509_09754_amd import lava as L
    return L


def wide(table):
    batch, heads, blocks = table.shape
    return np.pad(table, ((0, 0), (0, 0), (0, max(0, 8192 // (batch * heads) + 1 - blocks))), constant_values=-1)


def make(lava, batch, heads, page, blocks, dtype="bf16", d=128, spare=0, with_pos=True, seed=1):
    rng = np.random.default_rng(seed)
    n_pages = max(2, int(batch * heads * blocks * 0.6)) + spare
    table, rows, pos, free, n_free = random_state(rng, batch, heads, blocks, page, n_pages, 0.5)
    return rng, Cache(lava, lava.LayerDesc.make(heads, heads, d, 1, dtype), page, wide(table), rows, pos, free, n_free, with_pos, seed)


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("batch,heads", [(6, 3), (90, 3)])            # one workgroup that sums, and many
def test_refused_on_the_device(lava, in_place, batch, heads):
    """Nothing changes, the reason is in the error word; a call after it goes on."""
    page = 16
    rng, c = make(lava, batch, heads, page, 4, spare=4 * batch * heads, seed=9)
    start = {n: x.copy() for n, x in c.now.items()}

    def refused(over={}, **kw):
        """One call from the start's state, with some of its values replaced; then the start's state again."""
        for name, (where, value) in over.items():
            c.now[name][where] = value
        for name in start:
            c.view(name).copy_(dev(c.now[name]))
        error = c.change(in_place, **kw)
        for name, x in start.items():
            c.now[name] = x.copy()
            c.view(name).copy_(dev(x))
        return error

    same = np.arange(batch)
    good, full_one = same.copy(), int(np.argmax((start["rows"] % page != 0).sum(1)))
    good[0] = 1
    all_of_one, last = np.full(batch, full_one), (batch - 1, heads - 1)
    room = c.blocks * page
    assert (start["rows"][full_one] % page).any()
    for b, value in ((batch - 1, batch), (1, -2)):
        source = good.copy()
        source[b] = value
        assert refused(source=source) == B.INVALID
    counts, kept = random_lists(rng, c.now["rows"], 0.5)
    for where, value in (((2, 1), -1), (last, room + 1), ((0, 0), int(start["rows"][0, 0]) + 1)):
        x = counts.copy()
        x[where] = value
        assert refused(counts=x, kept=kept) == B.INVALID
    assert refused(counts=counts, kept=kept[:, : int(counts.sum(1).max()) - 1]) == B.INVALID
    held = np.argwhere(start["rows"] > page)[-1]
    for name, where, value in (("rows", (3, 1), -1), ("rows", last, room + 1), ("n_free", (0,), -1), ("n_free", (0,), c.n_pages + 1),
                               ("table", (*held, 0), -1), ("table", (*held, 1), c.n_pages)):
        assert refused(source=good, over={name: (where, value)}) == B.INVALID, (name, value)
    assert refused(source=all_of_one, over={"n_free": (0, 0)}) == B.EXHAUSTED
    for value in (-1, c.n_pages):                                     # the stack's top is no page
        assert refused(source=all_of_one, over={"free": (int(start["n_free"][0]) - 1, value)}) == B.INVALID
    full = {"free": (slice(None), 0), "n_free": (0, c.n_pages)}       # nowhere to put what comes back
    assert refused(source=np.full(batch, -1), over=full) == B.INVALID
    assert refused(source=all_of_one) == 0


@pytest.mark.parametrize("in_place", [True, False])
def test_lists_that_name_rows_a_head_does_not_hold(lava, in_place):
    """Their places stay unwritten, the others are copied."""
    rng, c = make(lava, 3, 2, 16, 6, spare=40, seed=5)
    counts = (c.now["rows"] * 2) // 3
    kept = np.full((3, int(counts.sum(1).max())), -5, np.int32)
    for b in range(3):
        at = 0
        for g in range(2):
            n = int(counts[b, g])
            kept[b, at: at + n] = np.sort(rng.permutation(int(c.now["rows"][b, g]))[:n])
            if n > 2:
                kept[b, at + n - 1] = (1 << 30, int(c.now["rows"][b, g]), 97)[b]
                kept[b, at] = (-9, 0, -1 << 31)[b]
            at += n
    assert (counts > 2).sum() > 3
    assert c.change(in_place, counts=counts, kept=kept) == 0


@pytest.mark.parametrize("same", [0, 1, 63, 64, 65, 127, 128, 200, 4096, 4097, 5000])
def test_lists_that_begin_with_what_is_there(lava, same):
    """How many leading rows stay in place is searched for 64 ways at a time: every number of them is found."""
    page, rows = 16, 5000
    nb = -(-rows // page)
    rng = np.random.default_rng(same)
    table = wide(np.arange(2 * nb).reshape(1, 2, nb).astype(np.int32))
    free = np.concatenate([np.arange(2 * nb, 4 * nb), np.full(2 * nb, -1)]).astype(np.int32)
    c = Cache(lava, lava.LayerDesc.make(2, 2, 64, 1, "bf16"), page, table, np.full((1, 2), rows, np.int32), np.array([rows], np.int32), free, 2 * nb)
    tail = same + 1 + np.flatnonzero(rng.random(max(0, rows - same - 1)) < 0.3)
    kept = np.concatenate([np.arange(same), tail, np.arange(rows)])
    assert c.change(False, counts=np.array([[same + len(tail), rows]]), kept=kept[None]) == 0
    assert np.array_equal(c.now["table"][0, 0, : same // page], np.arange(same // page))


@pytest.mark.parametrize("with_pos", [True, False])
def test_last_pages_stay_with_their_keeper(lava, with_pos):
    """Who goes on with a page that is not full: the sequence itself, else its first copy, and a head that loses no row."""
    page = 16
    table = wide(np.array([[[0, 1, -1]], [[2, -1, -1]], [[3, 4, 5]], [[-1, -1, -1]]], np.int32))
    rows = np.array([[20], [16], [33], [0]], np.int32)
    free = np.array([9, 8, 7, 6, -1, -1, -1, -1, -1, -1], np.int32)
    desc = lava.LayerDesc.make(1, 1, 128, 1, "bf16")
    for source in ([0, 0, 0, 0], [2, 2, 0, 0], [3, 0, 1, 2], [1, 1, 1, 1], [-1, 0, 0, -1], [-1, -1, -1, -1], [2, 0, 2, 2], [3, 3, 3, 3]):
        for in_place in (True, False):
            c = Cache(lava, desc, page, table.copy(), rows.copy(), np.array([7, 8, 9, 3], np.int32), free.copy(), 4, with_pos)
            assert c.change(in_place, source=np.array(source)) == 0
            check_pages(c.now["table"], c.now["rows"], page, c.now["free"], int(c.now["n_free"][0]), 10)
    for counts, kept in (([20, 16, 33, 0], [range(20), range(16), range(33), []]), ([19, 3, 32, 0], [range(19), range(3), range(32), []]),
                         ([17, 16, 17, 0], [range(17), range(16), range(17), []]), ([1, 1, 1, 0], [[19], [0], [5], []]), ([0, 0, 0, 0], [[]] * 4)):
        c = Cache(lava, desc, page, table.copy(), rows.copy(), np.zeros(4, np.int32), free.copy(), 4, with_pos)
        lists = np.array([list(x) + [-1] * (33 - len(x)) for x in kept], np.int32)
        assert c.change(False, counts=np.array(counts).reshape(4, 1), kept=lists) == 0
        check_pages(c.now["table"], c.now["rows"], page, c.now["free"], int(c.now["n_free"][0]), 10)


def test_keepers_among_many_sequences(lava):
    """The first copy is looked for 512 sequences at a time."""
    batch, page = 1300, 16
    rows = np.full((batch, 1), page + 3, np.int32)
    table = wide(np.arange(2 * batch).reshape(batch, 1, 2).astype(np.int32))
    free = np.concatenate([np.arange(2 * batch, 4 * batch), np.full(2 * batch, -1)]).astype(np.int32)
    c = Cache(lava, lava.LayerDesc.make(1, 1, 64, 1, "bf16"), page, table, rows, np.arange(batch).astype(np.int32), free, 2 * batch)
    source = (np.arange(batch) + 1) % batch
    source[[511, 512, 513, 1023, 1024, 1299]] = 700                   # 700 is not its own source: 511 goes on with its last page
    assert c.change(True, source=source) == 0
    assert int(c.now["table"][511, 0, 1]) == 1401 and int(c.now["table"][699, 0, 1]) >= 2 * batch


@pytest.mark.parametrize("evict", [False, True])
def test_no_lists_at_all(lava, evict):
    """A capacity of zero: every head gives all of its rows back, or those of the sequences that are evicted."""
    rng, c = make(lava, 4, 2, 32, 3, spare=9)
    assert c.change(True, counts=np.zeros((4, 2), np.int32), kept=np.zeros((4, 0), np.int32), evict=np.array([1, 0, 5, 0]) if evict else None) == 0
    assert (int(c.now["n_free"][0]) == c.n_pages) == (not evict) and not c.now["rows"][[0, 2]].any()


@pytest.mark.parametrize("what", ["fork", "compact"])
def test_replays(lava, what):
    """Replayed over a workspace of any contents with eager work between: the same state every time."""
    rng, c = make(lava, 12, 4, 32, 5, spare=200, seed=21)
    source = dev(np.array([0, 0, 0, 3, 3, 5, 5, 7, -1, 2, 10, 1], np.int32))
    counts, kept = (dev(x.astype(np.int32)) for x in random_lists(rng, c.now["rows"], 0.6))
    for n in ("table", "rows", "pos", "free", "n_free"):
        c.bufs[n + "_out"] = c._guarded(np.full_like(c.now[n], 55))
    names = [n for n in c.bufs if n.endswith("_out")]
    state = c.state("_out")
    ws = torch.empty(lava.lava_page_fork_workspace_bytes(12, 4, c.blocks, c.n_pages), dtype=torch.uint8, device=DEV)
    outs = dict(block_table_out=c.view("table_out"), free_pages_out=c.view("free_out"))
    if what == "fork":
        call = lambda **kw: lava.lava_page_fork(c.desc, c.pool, state, source, **outs, **kw)
    else:
        call = lambda **kw: lava.lava_page_compact(c.desc, c.pool, state, counts, kept, **outs, **kw)
    call(workspace=ws)
    torch.cuda.synchronize()
    want, k = {n: c.view(n).clone() for n in names}, c.k.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(workspace=ws)
    for i in range(6):
        ws.fill_((255, 0, 1, 128, 77, 254)[i])
        for n in names:
            c.view(n).fill_(55)
        if i % 2:
            call()
            for n in names:
                c.view(n).fill_(56)
                c.view(n).fill_(55)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(c.view(n), want[n]) for n in names) and torch.equal(c.k, k)
        assert int(c.view("error")[0]) == 0


@pytest.mark.parametrize("batch,heads,page,dtype,d", [(24, 2, 16, "bf16", 64), (8, 3, 128, "f32", 128), (300, 1, 32, "bf16", 128)])
def test_histories(lava, batch, heads, page, dtype, d):
    """Forks and evictions one after another, in place and apart."""
    rng, c = make(lava, batch, heads, page, 6, dtype, d, spare=2 * batch * heads, with_pos=d == 64, seed=batch)
    for step in range(10):
        if step % 2 == 0:
            c.change(step % 4 == 0, source=sources(rng, batch, (0, 4, 1, 3, 0)[step // 2]))
        else:
            counts, kept = random_lists(rng, c.now["rows"], 0.8)
            c.change(step % 4 == 1, counts=counts, kept=kept, evict=None if step % 3 else (rng.random(batch) < 0.6).astype(np.int32))
        check_pages(c.now["table"], c.now["rows"], page, c.now["free"], int(c.now["n_free"][0]), c.n_pages)
