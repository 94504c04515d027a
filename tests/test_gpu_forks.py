"""Forks and compaction of pages on the GPU against their oracle: tables, counts, stack and copied rows are equal, bit for bit, and nothing else
is written."""
import numpy as np
import pytest

from oracle import branch_oracle as B
from oracle import paged_oracle as P
from test_branch_oracle_pins import check_pages, random_lists
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


def host(t):
    return t.cpu().numpy()


class Cache:
    """A state and its pool on the device, canaries behind every buffer, and what the oracle makes of them."""

    def __init__(self, lava, desc, page, table, rows, pos, free, n_free, with_pos=True, seed=0):
        self.lava, self.desc, self.page, self.n_pages = lava, desc, page, free.size
        self.batch, self.heads, self.blocks = table.shape
        self.bufs = {}
        self.now = dict(table=table, rows=rows, pos=pos, free=free, n_free=np.array([n_free], np.int32))
        for name, a in self.now.items():
            self.bufs[name] = self._guarded(a)
        self.bufs["error"] = self._guarded(np.zeros(1, np.int32))
        g = torch.Generator(device=DEV).manual_seed(seed)
        shape = (self.n_pages, page, desc.head_dim)
        self.k, self.v = (torch.randn(shape, generator=g, device=DEV).to(desc.torch_dtype) for _ in range(2))
        self.pos_pages = torch.randint(0, 1 << 20, shape[:2], generator=g, device=DEV).to(torch.int32) if with_pos else None
        self.pool = lava.PagePool(self.k, self.v, self.pos_pages, max_blocks=self.blocks)

    def _guarded(self, a):
        t = torch.full((a.size + 64,), -77, dtype=torch.int32, device=DEV)
        t[: a.size] = dev(a.reshape(-1))
        return t, a.shape

    def view(self, name):
        t, shape = self.bufs[name]
        return t[: int(np.prod(shape))].view(*shape)

    def state(self, out=""):
        v = self.view
        return self.lava.PageState(v("table"), v("rows"), v("pos"), v("free"), v("n_free"), self.page, *(v(x + out) for x in ("rows", "pos", "n_free")),
                                   error=v("error"))

    def change(self, in_place, source=None, counts=None, kept=None, evict=None, workspace=None, call=None):
        """One call, checked; the state goes on with its result.  Returns the error bits."""
        i32 = lambda x: None if x is None else dev(np.asarray(x, np.int32))
        out, outs = ("", {}) if in_place else ("_out", {})
        apart = {}
        if not in_place:
            for name in ("table", "rows", "pos", "free", "n_free"):
                apart[name] = np.full_like(self.now[name], 55)
                self.bufs[name + "_out"] = self._guarded(apart[name])
            outs = dict(block_table_out=self.view("table_out"), free_pages_out=self.view("free_out"))
        n = self.now
        want = B.page_change(self.page, self.n_pages, n["table"], n["rows"], n["pos"], n["free"], int(n["n_free"][0]), source, counts, kept, evict,
                             apart.get("table"), apart.get("free"))
        k, v, pp = self.k.clone(), self.v.clone(), None if self.pos_pages is None else self.pos_pages.clone()
        if want[5]:
            moves = dev(np.array(want[5], np.int64))
            d = self.desc.head_dim
            for t, cells in ((k, k.view(-1, d)), (v, v.view(-1, d))) + (((pp, pp.view(-1)),) if pp is not None else ()):
                cells[moves[:, 0]] = cells[moves[:, 1]].clone()
        self.view("error").zero_()
        state = self.state(out)
        if counts is not None:
            self.lava.lava_page_compact(self.desc, self.pool, state, i32(counts), i32(kept), i32(evict), workspace=workspace, **outs)
        else:
            self.lava.lava_page_fork(self.desc, self.pool, state, i32(source), workspace=workspace, **outs)
        torch.cuda.synchronize()
        assert int(self.view("error")[0]) == want[6]
        for name, x in zip(("table", "rows", "pos", "free", "n_free"), want[:5]):
            got = host(self.view(name + out))
            assert np.array_equal(got, np.asarray(x).reshape(got.shape)), name
        assert torch.equal(self.k, k) and torch.equal(self.v, v) and (pp is None or torch.equal(self.pos_pages, pp))
        for t, shape in self.bufs.values():
            assert bool((t[int(np.prod(shape)):] == -77).all())
        for name in ("table", "rows", "pos", "free", "n_free"):
            if not in_place:                                           # what was there is as it was; the new state takes over
                assert np.array_equal(host(self.view(name)), n[name]), name
                self.bufs[name] = self.bufs.pop(name + "_out")
            self.now[name] = host(self.view(name)).copy()
        return want[6]

    def append(self, new):
        """New tokens by lava_page_tables; returns whether they were taken."""
        n, m = self.now, int(new.sum()) + 2
        want = P.page_tables(self.page, self.n_pages, n["table"], n["rows"], n["pos"], n["free"], int(n["n_free"][0]), new, max_tokens=m)
        slots = torch.empty(m, self.heads, dtype=torch.int64, device=DEV)
        self.view("error").zero_()
        self.lava.lava_page_tables(self.state(), dev(new.astype(np.int32)), slots=slots)
        torch.cuda.synchronize()
        assert int(self.view("error")[0]) == want[7] and np.array_equal(host(slots), want[5])
        for name in ("table", "rows", "pos", "free", "n_free"):
            self.now[name] = host(self.view(name)).copy()
        return want[7] == 0


def make(lava, batch, heads, page, blocks, dtype="bf16", d=128, fill=0.5, spare=0, with_pos=True, seed=1):
    rng = np.random.default_rng(seed)
    n_pages = max(2, int(batch * heads * blocks * (fill + 0.1))) + spare
    table, rows, pos, free, n_free = random_state(rng, batch, heads, blocks, page, n_pages, fill)
    desc = lava.LayerDesc.make(heads, heads, d, 1, dtype)
    return rng, Cache(lava, desc, page, table, rows, pos, free, n_free, with_pos, seed)


def sources(rng, batch, how):
    if how == 0:
        return rng.integers(0, batch, batch)
    if how == 1:
        return rng.permutation(batch)
    if how == 2:
        return np.arange(batch)
    if how == 3:
        return np.full(batch, rng.integers(-1, batch))
    x = rng.integers(-1, batch, batch)
    return np.where(rng.random(batch) < 0.5, np.arange(batch), x)


# one head; beams of a layer; more than a thousand sequences; pages of every size, both types and head sizes
@pytest.mark.parametrize("batch,heads,page,blocks,dtype,d", [
    (1, 1, 16, 3, "bf16", 64), (8, 8, 64, 6, "bf16", 128), (5, 64, 16, 4, "f32", 64), (40, 3, 32, 7, "f32", 128), (16, 2, 256, 3, "bf16", 128),
    (1100, 1, 16, 4, "bf16", 64), (3, 2, 16, 300, "bf16", 64), (33, 7, 128, 2, "f32", 64)])
def test_histories(lava, batch, heads, page, blocks, dtype, d):
    """Forks, evictions and tokens one after another, in place and apart."""
    print(f"history {batch}x{heads} pages of {page} {dtype} d {d}", flush=True)
    rng, c = make(lava, batch, heads, page, blocks, dtype, d, spare=batch * heads, with_pos=d == 64, seed=batch + heads)
    refused = 0
    for step in range(12 if batch < 1000 else 6):
        kind = step % 3
        if kind == 0:
            refused += c.change(step % 2 == 0, source=sources(rng, batch, int(rng.integers(0, 5)))) != 0
        elif kind == 1:
            counts, kept = random_lists(rng, c.now["rows"], 0.7)
            evict = None if step % 2 else (rng.random(batch) < 0.6).astype(np.int32) * -3
            ws = torch.full((lava.lava_page_fork_workspace_bytes(batch, heads, blocks, c.n_pages),), 0xA5, dtype=torch.uint8, device=DEV)
            refused += c.change(step % 2 == 1, counts=counts, kept=kept, evict=evict, workspace=ws) != 0
        else:
            room = blocks * page - c.now["rows"].max(1)
            refused += not c.append(np.minimum(rng.integers(0, page + 3, batch), room))
        if batch < 100 and batch * heads * blocks < 3000:
            check_pages(c.now["table"], c.now["rows"], page, c.now["free"], int(c.now["n_free"][0]), c.n_pages)
    assert refused < 6


# tables that one workgroup marks (256 heads and 8192 entries at most), and the next larger ones
@pytest.mark.parametrize("batch,heads,blocks", [(64, 4, 32), (257, 1, 4), (1, 1, 8192), (1, 1, 8193), (256, 1, 32), (127, 2, 33)])
def test_small_changes_and_the_next_larger(lava, batch, heads, blocks):
    print(f"edges {batch}x{heads}x{blocks}", flush=True)
    rng, c = make(lava, batch, heads, 16, blocks, "bf16", 64, fill=0.4, spare=3 * batch * heads, seed=blocks)
    for in_place in (True, False):
        c.change(in_place, source=sources(rng, batch, 4))
        counts, kept = random_lists(rng, c.now["rows"], 0.8)
        c.change(in_place, counts=counts, kept=kept)


def test_pool_beyond_four_gib(lava):
    """Pages whose bytes lie beyond 2^32 of the pool's start: copied from, copied to."""
    page, d, n_pages = 256, 128, 100_000
    desc = lava.LayerDesc.make(2, 2, d, 1, "bf16")
    k, v = (torch.empty(n_pages, page, d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    pool = lava.PagePool(k, v, None, max_blocks=2)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)
    for x in (k, v):
        x[[99_999, 70_001, 3, 80_000]] = torch.randn(4, page, d, device=DEV).to(torch.bfloat16)
    free = torch.zeros(n_pages, dtype=torch.int32, device=DEV)
    free[:4] = i32(99_998, 5, 99_997, 90_000)
    state = lava.PageState(i32([[99_999, 70_001], [3, 80_000]], [[-1, -1], [-1, -1]]), i32([300, 511], [0, 0]), i32(600, 0), free, i32(4), page)
    lava.lava_page_fork(desc, pool, state, i32(0, 0))
    torch.cuda.synchronize()
    assert state.block_table.tolist() == [[[99_999, 70_001], [3, 80_000]], [[99_999, 90_000], [3, 99_997]]] and int(state.n_free[0]) == 2
    for x in (k, v):
        assert torch.equal(x[90_000, :44], x[70_001, :44]) and torch.equal(x[99_997, :255], x[80_000, :255])
    kept = torch.cat([torch.arange(1, 300, 2), torch.arange(511)]).to(DEV, torch.int32)[None].repeat(2, 1).contiguous()
    lava.lava_page_compact(desc, pool, state, i32([150, 511], [150, 511]), kept, evict=i32(0, 1))
    torch.cuda.synchronize()
    assert state.block_table[1].tolist() == [[5, 90_000], [3, 99_997]] and state.head_rows.tolist() == [[300, 511], [150, 511]]
    for x in (k, v):
        old = torch.cat([x[99_999], x[70_001]])
        assert torch.equal(x[5, :150], old[1:300:2])
    assert int(state.n_free[0]) == 2 and state.free_pages[:2].tolist() == [99_998, 90_000]


@pytest.mark.parametrize("in_place", [True, False])
def test_refused_on_the_device(lava, in_place):
    """Nothing changes, the reason is in the error word; a call after it goes on."""
    batch, heads, page, blocks = 6, 3, 16, 4
    rng, c = make(lava, batch, heads, page, blocks, spare=40, seed=9)
    start = {n: x.copy() for n, x in c.now.items()}

    def refused(**kw):
        """One call from the start's state, with some of its values replaced; then the start's state again."""
        over = kw.pop("over", {})
        for name, (where, value) in over.items():
            c.now[name][where] = value
        for name in start:
            c.view(name).copy_(dev(c.now[name]))
        error = c.change(in_place, **kw)
        for name, x in start.items():
            c.now[name] = x.copy()
            c.view(name).copy_(dev(x))
        return error

    good, all_of_one = np.array([1, 1, 2, 3, 4, 5]), np.array([4] * 6)
    assert start["table"][1, 0, 0] >= 0 and (start["rows"][4] % page).any()
    assert refused(source=np.array([0, 1, 2, 3, 4, 6])) == B.INVALID and refused(source=np.array([0, -2, 2, 3, 4, 5])) == B.INVALID
    counts, kept = random_lists(rng, c.now["rows"], 0.5)
    for where, value in (((2, 1), -1), ((5, 2), blocks * page + 1), ((0, 0), int(c.now["rows"][0, 0]) + 1)):
        x = counts.copy()
        x[where] = value
        assert refused(counts=x, kept=kept) == B.INVALID
    assert refused(counts=counts, kept=kept[:, : int(counts.sum(1).max()) - 1]) == B.INVALID
    for name, where, value in (("rows", (3, 1), -1), ("rows", (3, 1), blocks * page + 1), ("n_free", (0,), -1), ("n_free", (0,), c.n_pages + 1),
                               ("table", (1, 0, 0), -1), ("table", (1, 0, 0), c.n_pages)):
        assert refused(source=good, over={name: (where, value)}) == B.INVALID, (name, value)
    assert refused(source=all_of_one, over={"n_free": (0, 0)}) == B.EXHAUSTED
    for value in (-1, c.n_pages):                                     # the stack's top is no page
        assert refused(source=all_of_one, over={"free": (int(start["n_free"][0]) - 1, value)}) == B.INVALID
    full = {"free": (slice(None), 0), "n_free": (0, c.n_pages)}       # nowhere to put what comes back
    assert refused(source=np.full(6, -1), over=full) == B.INVALID
    assert refused(source=all_of_one) == 0


def test_lists_that_name_rows_a_head_does_not_hold(lava):
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
    assert c.change(False, counts=counts, kept=kept) == 0


@pytest.mark.parametrize("with_pos", [True, False])
def test_last_pages_stay_with_their_keeper(lava, with_pos):
    """Who goes on with a page that is not full: the sequence itself, else its first copy, and a head that loses no row."""
    page, blocks = 16, 3
    table = np.array([[[0, 1, -1]], [[2, -1, -1]], [[3, 4, 5]], [[-1, -1, -1]]], np.int32)
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


def test_no_lists_at_all(lava):
    """A capacity of zero: every head gives all of its rows back."""
    rng, c = make(lava, 4, 2, 32, 3, spare=9)
    assert c.change(True, counts=np.zeros((4, 2), np.int32), kept=np.zeros((4, 0), np.int32)) == 0
    assert int(c.now["n_free"][0]) == c.n_pages and not c.now["rows"].any()


def test_replays(lava):
    """Forks apart, replayed over a workspace of any contents with eager work between: the same state every time."""
    rng, c = make(lava, 12, 4, 32, 5, spare=60, seed=21)
    source = dev(np.array([0, 0, 0, 3, 3, 5, 5, 7, -1, 2, 10, 1], np.int32))
    outs = {n: c._guarded(np.full_like(c.now[n], 55)) for n in ("table", "rows", "pos", "free", "n_free")}
    for n, b in outs.items():
        c.bufs[n + "_out"] = b
    state = c.state("_out")
    ws = torch.empty(lava.lava_page_fork_workspace_bytes(12, 4, 5, c.n_pages), dtype=torch.uint8, device=DEV)
    call = lambda: lava.lava_page_fork(c.desc, c.pool, state, source, c.view("table_out"), c.view("free_out"), workspace=ws)
    call()
    torch.cuda.synchronize()
    want = {n: c.view(n + "_out").clone() for n in outs}
    k = c.k.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in range(5):
        ws.fill_(255 - i)
        for n in outs:
            c.view(n + "_out").fill_(55)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(c.view(n + "_out"), want[n]) for n in outs) and torch.equal(c.k, k)


def test_large_state(lava):
    """65536 heads, a wavefront has several; most sequences change places."""
    batch, heads, page, blocks = 16384, 4, 16, 2
    rng = np.random.default_rng(2)
    rows = rng.integers(0, 33, (batch, heads)).astype(np.int32)
    nb = -(-rows // page)
    n_pages = int(nb.sum()) + 70000
    order = rng.permutation(n_pages).astype(np.int32)
    table = np.full((batch, heads, blocks), -1, np.int32)
    table[np.arange(blocks) < nb[..., None]] = order[: int(nb.sum())]
    free = np.full(n_pages, -1, np.int32)
    n_free = n_pages - int(nb.sum())
    free[:n_free] = order[int(nb.sum()):]
    desc = lava.LayerDesc.make(4, 4, 64, 1, "bf16")
    c = Cache(lava, desc, page, table, rows, rng.integers(0, 99, batch).astype(np.int32), free, n_free)
    source = np.where(rng.random(batch) < 0.5, np.arange(batch), rng.integers(-1, batch, batch))
    i32 = lambda x: dev(np.asarray(x, np.int32))
    state = c.state()
    old_t, old_r = table.copy(), rows.copy()
    lava.lava_page_fork(c.desc, c.pool, state, i32(source))
    torch.cuda.synchronize()
    assert int(c.view("error")[0]) == 0
    got_r, got_t, got_f = host(c.view("rows")), host(c.view("table")), host(c.view("free"))
    src = np.clip(source, 0, None)
    assert np.array_equal(got_r, np.where(source[:, None] >= 0, old_r[src], 0))
    full = np.arange(blocks) < (got_r // page)[..., None]
    assert np.array_equal(got_t[full], old_t[src][full])
    used = got_t[np.arange(blocks) < (-(-got_r // page))[..., None]]
    left = int(c.view("n_free")[0])
    both = np.concatenate([np.unique(used), got_f[:left]])
    assert both.size == n_pages and np.array_equal(np.sort(both), np.arange(n_pages))
    last = got_t[np.arange(blocks) == (got_r // page)[..., None]]
    open_pages = last[(got_r % page != 0)[(got_r // page) < blocks]]
    assert np.unique(open_pages).size == open_pages.size


def test_binding_refuses(lava):
    rng, c = make(lava, 4, 2, 32, 3, spare=9)
    state, i32 = c.state(), lambda *s: torch.zeros(*s, dtype=torch.int32, device=DEV)
    fork = lambda **kw: lava.lava_page_fork(**{**dict(desc=c.desc, pool=c.pool, state=state, source=i32(4)), **kw})
    compact = lambda **kw: lava.lava_page_compact(**{**dict(desc=c.desc, pool=c.pool, state=state, head_counts=i32(4, 2), kept_idx=i32(4, 5)), **kw})
    for kw in (dict(source=i32(3)), dict(source=i32(4).long()), dict(block_table_out=i32(4, 2, 2)), dict(free_pages_out=i32(3)),
               dict(desc=lava.LayerDesc.make(4, 4, 128, 1, "bf16")), dict(desc=lava.LayerDesc.make(2, 2, 64, 1, "bf16")),
               dict(pool=lava.PagePool(c.k, c.v, c.pos_pages, max_blocks=4)), dict(pool=lava.PagePool(c.k[:-1], c.v[:-1], None, max_blocks=3))):
        with pytest.raises(ValueError):
            fork(**kw)
    for kw in (dict(head_counts=i32(4)), dict(kept_idx=i32(20)), dict(kept_idx=i32(3, 5)), dict(evict=i32(5)), dict(kept_idx=i32(4, 5).float())):
        with pytest.raises(ValueError):
            compact(**kw)
    with pytest.raises(lava.LavaError):
        fork(workspace=torch.zeros(256, dtype=torch.uint8, device=DEV))
