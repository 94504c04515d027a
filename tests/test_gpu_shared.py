"""Decode over shared pages on the GPU: what decode over pages gives, by that one's oracle (roundings bounded beside it) and by pages whose
answer is a count; groups of every size, pages in common or not; and beams through forks, tables, rotary and eviction as a program runs them."""
import math

import numpy as np
import pytest

from oracle import branch_oracle as B
from oracle import paged_oracle as P
from oracle.paged_counts import MOST, SCALE, Pages

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
DEV = "cuda"


@pytest.fixture(scope="module")
def lava():
    from paper_2509_09754_amd import lava as L
    return L


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


ROOM = 410_000_000                                                   # bytes that tables must have room for to be looked at for common pages


def widened(table, page, row_bytes):
    """The same tables with room for more blocks."""
    batch, heads, blocks = table.shape
    wide = max(blocks, -(-ROOM // (batch * heads * page * row_bytes)))
    return np.pad(table, ((0, 0), (0, 0), (0, wide - blocks)), constant_values=-1)


def shared_tables(rng, sizes, Hkv, page, front, own_lo, own_hi, idle=()):
    """(table, rows, pages) of groups of those sizes; front(group, head): pages in common."""
    batch = sum(sizes)
    fronts = np.array([[front(i, g) for g in range(Hkv)] for i in range(len(sizes))])
    group = np.repeat(np.arange(len(sizes)), sizes)
    rows = fronts[group] * page + rng.integers(own_lo, own_hi + 1, (batch, Hkv))
    for b in idle:
        rows[b] = 0
    nb = -(-rows // page)
    table = np.full((batch, Hkv, max(1, nb.max())), -1, np.int64)
    n = 0
    first = {}
    for b in range(batch):
        for g in range(Hkv):
            for j in range(nb[b, g]):
                key = (group[b], g, j)
                if j < fronts[group[b], g]:
                    if key not in first:
                        first[key] = n
                        n += 1
                    table[b, g, j] = first[key]
                else:
                    table[b, g, j] = n
                    n += 1
    order = rng.permutation(n + 3)
    table = np.where(table >= 0, order[np.maximum(table, 0)], -1)
    return table.astype(np.int32), rows.astype(np.int32), n + 3


def own_weight(lse):
    """How far the weight of a sequence's own rows may be off, relative: their log-sum-exp is stored in 32 bits (a logarithm within 2^-22, a sum
    and two products within half a step each), and an exponential of it."""
    return lse.abs() * 2.0 ** -21 + 2.0 ** -21


class Case:
    def __init__(self, lava, rng, H, Hkv, d, dtype, page, sizes, table, rows, n_pages, softcap=0.0, window=0, bias=False, span=None, narrow=False):
        self.lava, self.batch = lava, len(rows)
        if not narrow:
            table = widened(table, page, 2 * d * (2 if dtype == "bf16" else 4))
        dt = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.desc = lava.LayerDesc.make(H, Hkv, d, 1, dtype)
        val = lambda *s: dev(rng.normal(size=s).astype(np.float32)).to(dt)
        self.q, self.k, self.v = val(self.batch, H, d), val(n_pages, page, d), val(n_pages, page, d)
        self.table, self.rows = dev(table), dev(rows)
        self.start = dev(np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32))
        span = span or 4 * max(1, int(rows.max()))
        self.pos = dev(rng.integers(0, span, (n_pages, page)).astype(np.int32))
        self.q_pos = dev(rng.integers(span // 2, span, self.batch).astype(np.int32))
        self.slopes = dev((2.0 ** (-8.0 * (1 + np.arange(H)) / H)).astype(np.float32)) if bias else None
        self.kw = dict(softcap=softcap, window=window, slopes=self.slopes)
        self.options = lava.DecodeOptions.make(**self.kw) if softcap or window or bias else None
        self.pool = lava.PagePool(self.k, self.v, self.pos, max_blocks=table.shape[2])

    def run(self, start=None, workspace=None, **kw):
        out, lse = self.lava.lava_shared_decode(self.desc, self.q, self.pool, self.table, self.rows, self.start if start is None else start,
                                                self.options, self.q_pos, workspace=workspace, **kw)
        torch.cuda.synchronize()
        return out, lse

    def want(self):
        f = lambda t: t.double().cpu().numpy()
        out, lse, tol, tol_lse = P.paged_decode(f(self.q), f(self.k), f(self.v), self.table.cpu().numpy(), self.rows.cpu().numpy(),
                                                self.desc.head_dim ** -0.5, self.kw["softcap"], self.kw["window"],
                                                None if self.slopes is None else f(self.slopes), self.pos.cpu().numpy(), self.q_pos.cpu().numpy())
        return [torch.from_numpy(x) for x in (out, lse, tol, tol_lse)]

    def check(self, out, lse):
        want, want_lse, tol, tol_lse = self.want()
        out, lse = out.double().cpu(), lse.double().cpu()
        assert torch.equal(torch.isnan(lse), torch.isnan(want_lse)) and torch.equal(torch.isnan(out), torch.isnan(want))
        some = torch.isfinite(want_lse)
        assert torch.equal(torch.isfinite(lse), some)
        # the weight of the own rows: both parts are averages of values (at most `top` of them), and a (1 - a) <= 1 / 4.  What is in common is summed as
        # products of exact parts of the probabilities, which leaves out less than 2^-24 of each
        top = float(self.v.double().abs().max())
        weight = own_weight(want_lse.where(some, torch.zeros(())).abs() + 20.0)
        tol = tol + 0.25 * weight[..., None] * 2.0 * top + 2.0 ** -22 * top
        bad = (out - want).abs() > tol
        assert not bool(bad[some].any()), float(((out - want).abs() / tol)[some].max())
        assert not bool(((lse - want_lse).abs() > tol_lse + weight)[some].any())


SHAPES = [(32, 8, 128, "bf16", 16), (14, 2, 128, "bf16", 64), (4, 4, 64, "bf16", 32), (16, 2, 64, "f32", 16), (8, 2, 128, "f32", 32), (3, 1, 64, "bf16", 256)]
OPTIONS = [{}, dict(softcap=20.0), dict(bias=True), dict(window=60), dict(softcap=30.0, window=200, bias=True)]


# groups of one, of a few, of more queries than an item has (256), of 33 and 65 query rows; commons of no page, of part of a stage, of several
@pytest.mark.parametrize("H,Hkv,d,dtype,page", SHAPES)
@pytest.mark.parametrize("kw", OPTIONS, ids=["plain", "cap", "bias", "window", "all"])
def test_shared(lava, H, Hkv, d, dtype, page, kw):
    print(f"shared {H}/{Hkv} d {d} {dtype} pages of {page} {kw}", flush=True)
    rng = np.random.default_rng(H * 7 + d + page + len(kw))
    for sizes, blocks in (([1, 5, 2], 3), ([9], 16), ([2, 1, 1, 4], 0), ([11, 3], 9)):
        front = lambda i, g: (blocks * 16 // page + (i + g) % 3) if blocks else 0
        table, rows, n_pages = shared_tables(rng, sizes, Hkv, page, front, 0, 40, idle=[0] if len(sizes) == 3 else [])
        c = Case(lava, rng, H, Hkv, d, dtype, page, sizes, table, rows, n_pages, **kw)
        ws = torch.full((lava.lava_shared_decode_workspace_bytes(c.desc, c.batch, c.table.shape[2]),), 0xFF, dtype=torch.uint8, device=DEV)
        c.check(*c.run(workspace=ws))


@pytest.mark.parametrize("H,Hkv,d,dtype,n", [(8, 1, 128, "bf16", 70), (4, 1, 64, "f32", 130), (1, 1, 64, "bf16", 300), (7, 1, 128, "bf16", 37)])
def test_groups_wider_than_an_item(lava, H, Hkv, d, dtype, n):
    rng = np.random.default_rng(n)
    table, rows, n_pages = shared_tables(rng, [n, 2], Hkv, 16, lambda i, g: 7, 0, 20, idle=[3])
    c = Case(lava, rng, H, Hkv, d, dtype, 16, [n, 2], table, rows, n_pages)
    c.check(*c.run())


COUNTS = {                                                           # group sizes, pages in common, own rows
    "one group of four, long": ([4], lambda i, g: 700 + 31 * g, 30),
    "sixty-four queries": ([16], lambda i, g: 300, 100),
    "groups of all sizes": ([1, 2, 3, 9, 17, 30], lambda i, g: 5 + 40 * i + 7 * g, 300),
    "many small groups": ([2] * 150, lambda i, g: 1 + (i + g) % 20, 60),
}


@pytest.mark.parametrize("G,d,dtype,page", [(4, 128, "bf16", 16), (7, 128, "bf16", 32), (8, 64, "bf16", 16), (1, 64, "bf16", 32), (4, 128, "f32", 16),
                                            (5, 64, "f32", 32)])
@pytest.mark.parametrize("load", COUNTS)
@pytest.mark.parametrize("kw", [{}, dict(window=300)], ids=["plain", "window"])
def test_every_row_counts_once(lava, G, d, dtype, page, load, kw):
    print(f"counts: {load}, {G} heads a group, d {d} {dtype}, pages of {page} {kw}", flush=True)
    sizes, front, own = COUNTS[load]
    Hkv, rng = 3, np.random.default_rng(len(load) + G)
    table, rows, n_pages = shared_tables(rng, sizes, Hkv, page, front, 1, own)
    batch, window = len(rows), kw.get("window", 0)
    table = widened(table, page, 2 * d * (2 if dtype == "bf16" else 4))
    pages = Pages(G + page, n_pages, page, d, device=DEV)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    desc = lava.LayerDesc.make(G * Hkv, Hkv, d, 1, dtype, softmax_scale=SCALE)
    pool = lava.PagePool(pages.k.to(dt), pages.v.to(dt), pages.pos, max_blocks=table.shape[2])
    q_pos = torch.where(torch.arange(batch, device=DEV) % 2 == 0, 999, 700).to(torch.int32)
    options = lava.DecodeOptions.make(**kw) if kw else None
    start = dev(np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32))
    out, lse = lava.lava_shared_decode(desc, pages.queries(batch, G * Hkv, G).to(dt), pool, dev(table), dev(rows), start, options, q_pos)
    want, want_lse, tol, tol_lse = pages.attend(dev(table), rows, G, window, q_pos if window else None)
    torch.cuda.synchronize()
    some = torch.isfinite(want_lse)
    assert bool((torch.isfinite(lse) == some).all())
    # rows that are off weigh 2^-1477 of those that are on; where all of either part are off, it weighs nothing
    weight = own_weight(want_lse.where(some, torch.zeros((), device=DEV, dtype=torch.float64)))
    tol = tol + 0.25 * weight[..., None] * MOST
    print(f"   worst {float(((out.double() - want).abs() / tol).max()):.3f} of the bound", flush=True)
    assert bool(((out.double() - want).abs() <= tol).all())
    assert bool(((lse.double() - want_lse).abs() <= tol_lse + weight)[some].all())


IDLE = pytest.mark.parametrize("idle", [0, 260], ids=["few", "many"])   # sequences that hold nothing: own rows of 512 heads and more are decoded apart


@IDLE
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64)])
def test_masked_values_may_be_anything(lava, dtype, d, idle):
    """Infinities and NaN in rows that a window leaves out, for all of a group or for some of its sequences only, and behind last rows."""
    rng = np.random.default_rng(3)
    H, Hkv, page = 8, 2, 16
    sizes = [4, 3, idle]
    table, rows, n_pages = shared_tables(rng, sizes, Hkv, page, lambda i, g: 12 + g, 1, 30, idle=range(7, 7 + idle))
    c = Case(lava, rng, H, Hkv, d, dtype, page, sizes, table, rows, n_pages, window=100, span=400)
    c.q_pos[:7] = dev(np.array([399, 399, 350, 310, 300, 300, 300], np.int32))
    inf = float("inf")
    low, high = c.pos < 200, c.pos >= 399                              # nobody sees the first; the last one some
    for t in (c.k, c.v):
        t[(c.pos < 200)] = inf
        t[(c.pos % 7 == 0) & (c.pos < 200)] = float("nan")
        t[(c.pos % 5 == 0) & (c.pos < 200)] = -inf
    assert bool(low.any())
    ends = c.rows.cpu().numpy()
    for b in range(c.batch):
        for g in range(Hkv):
            r = int(ends[b, g])
            if r % page:
                c.k[int(table[b, g, r // page]), r % page:] = float("nan")
                c.v[int(table[b, g, r // page]), r % page:] = inf
    c.check(*c.run())
    # rows that the first group's later sequences no longer see, its first ones do: those get NaN or infinities, these do not
    mixed = (c.pos >= 320) & (c.pos < 330)
    c.v[mixed] = float("nan")
    out, lse = c.run()
    f = lambda t: t.double().cpu().numpy()
    seen = np.zeros((c.batch, Hkv), bool)
    for b in range(c.batch):
        for g in range(Hkv):
            p = [int(c.pos[int(table[b, g, r // page]), r % page]) for r in range(int(ends[b, g]))]
            seen[b, g] = any(320 <= x < 330 and 0 <= int(c.q_pos[b]) - x < 100 for x in p)
    assert seen.any() and not seen.all()
    nan = torch.isnan(out).view(c.batch, Hkv, -1).all(2).cpu().numpy()
    assert np.array_equal(nan, seen)
    c.v[mixed] = 0.0
    want, want_lse, tol, tol_lse = c.want()
    clear = torch.from_numpy(~seen).repeat_interleave(H // Hkv, dim=1)
    assert bool(((out.double().cpu() - want).abs() <= tol + 1e-5)[clear].all())


def test_nothing_seen_and_nothing_held(lava):
    rng = np.random.default_rng(8)
    table, rows, n_pages = shared_tables(rng, [3, 4], 2, 16, lambda i, g: 6, 0, 9, idle=[1, 3, 4, 5, 6])
    c = Case(lava, rng, 4, 2, 64, "bf16", 16, [3, 4], table, rows, n_pages, window=5, span=100)
    c.q_pos[0] = 100000                                                # every row is too far back
    out, lse = c.run()
    c.check(out, lse)
    assert not bool(out[0].any()) and bool((lse[0] == -math.inf).all()) and not bool(out[3:].any())


def test_groups_that_are_none(lava):
    """Bounds that decrease, begin late or end early: nothing is shared, the result stands."""
    rng = np.random.default_rng(9)
    table, rows, n_pages = shared_tables(rng, [4, 5], 2, 16, lambda i, g: 8, 1, 20)
    c = Case(lava, rng, 8, 2, 128, "bf16", 16, [4, 5], table, rows, n_pages)
    plain = lava.lava_paged_decode(c.desc, c.q, c.pool, c.table, c.rows)
    for start in ([0, 4, 9], [0, 9], [0, 0, 9], [0, 9, 9], [1, 4, 9], [0, 4, 8], [0, 5, 4, 9], [0, 4, 10], [-1, 4, 9], [9, 4, 0], [0, 1 << 30, 9],
                  list(range(10)), [0, 2, 4, 6, 9]):
        out, lse = c.run(start=dev(np.array(start, np.int32)))
        c.check(out, lse)
    out, lse = c.run(start=dev(np.arange(10, dtype=np.int32)))
    assert torch.equal(out, plain[0]) and torch.equal(lse, plain[1])   # alone, every sequence is decoded as it is


@IDLE
def test_wrong_counts_and_pages(lava, idle):
    rng = np.random.default_rng(10)
    table, rows, n_pages = shared_tables(rng, [4, 5, idle], 2, 16, lambda i, g: 8, 1, 20, idle=range(9, 9 + idle))
    for what, value in (("rows", -1), ("rows", widened(table, 16, 512).shape[2] * 16 + 1), ("common", -1), ("common", n_pages), ("own", n_pages)):
        t, r = table.copy(), rows.copy()
        if what == "rows":
            r[2, 1] = value
        elif what == "common":
            t[:4, 0, 5] = value
        else:
            t[6, 1, rows[6, 1] // 16 if rows[6, 1] % 16 else rows[6, 1] // 16 - 1] = value
        c = Case(lava, np.random.default_rng(11), 8, 2, 128, "bf16", 16, [4, 5, idle], t, r, n_pages)
        out, lse = c.run()
        bad = torch.isnan(lse).view(9 + idle, 2, 4).all(2).cpu().numpy()
        want = np.zeros((9 + idle, 2), bool)
        want[(2, 1) if what == "rows" else (slice(0, 4), 0) if what == "common" else (6, 1)] = True
        assert np.array_equal(bad, want), what
        c.check(out, lse)


@pytest.mark.parametrize("page,d,dtype", [(16, 128, "bf16"), (64, 64, "f32")])
def test_little_room_is_decoded_apart(lava, launches, page, d, dtype):
    """Which launches a step takes follows from the room its tables have, from the number of heads and of groups, never from what they hold."""
    rng = np.random.default_rng(15)
    for narrow, idle in ((True, 0), (False, 0), (False, 248), (False, 250)):
        sizes = [3, 4, 1 + idle]
        table, rows, n_pages = shared_tables(rng, sizes, 2, page, lambda i, g: 5, 1, 20, idle=range(8, 8 + idle))
        c = Case(lava, rng, 8, 2, d, dtype, page, sizes, table, rows, n_pages, narrow=narrow)
        (out, lse), n = launches(c.run)
        c.check(out, lse)
        assert n["shared_plan"] == n["shared_decode"] == n["shared_merge"] == (0 if narrow else 1)
        assert n["paged_decode"] == (1 if narrow or 2 * (8 + idle) > 512 else 0)
    (out, lse), n = launches(lambda: c.run(start=dev(np.arange(c.batch + 1, dtype=np.int32))))
    c.check(out, lse)
    assert n["paged_decode"] == 1 and n["shared_plan"] == 0


def test_without_lse_and_replayed(lava):
    rng = np.random.default_rng(12)
    table, rows, n_pages = shared_tables(rng, [6, 1, 5], 4, 32, lambda i, g: 9 + g, 1, 70)
    c = Case(lava, rng, 16, 4, 128, "bf16", 32, [6, 1, 5], table, rows, n_pages, softcap=25.0, bias=True)
    want, want_lse = c.run()
    ws = torch.empty(lava.lava_shared_decode_workspace_bytes(c.desc, c.batch, c.table.shape[2]), dtype=torch.uint8, device=DEV)
    out, lse = torch.empty_like(want), torch.empty_like(want_lse)
    import ctypes
    status = lava.lib.lava_shared_decode(ctypes.byref(c.desc), c.batch, c.q.data_ptr(), c.pool._ref, c.table.data_ptr(), c.rows.data_ptr(), 3,
                                         c.start.data_ptr(), ctypes.byref(c.options), c.q_pos.data_ptr(), out.data_ptr(), None, ws.data_ptr(), ws.numel(),
                                         torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert status == lava.LAVA_OK and torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lava.lava_shared_decode(c.desc, c.q, c.pool, c.table, c.rows, c.start, c.options, c.q_pos, out=out, lse=lse, workspace=ws)
    for i in range(5):
        out.fill_(3), lse.fill_(3), ws.fill_(255 - i)
        graph.replay()
        eager = c.run()
        assert torch.equal(out, want) and torch.equal(lse, want_lse) and torch.equal(eager[0], want)


def test_pool_beyond_four_gib(lava):
    """Common and own pages whose bytes lie beyond 2^32 of the pool's start."""
    page, d, H, Hkv, n_pages = 256, 128, 8, 2, 100_000
    desc = lava.LayerDesc.make(H, Hkv, d, 1, "bf16")
    rng = np.random.default_rng(21)
    table, rows, few = shared_tables(rng, [3, 2], Hkv, page, lambda i, g: 3, 1, 300)
    high = n_pages - 1 - 37 * np.arange(few)
    k, v = (torch.empty(n_pages, page, d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    c = Case(lava, rng, H, Hkv, d, "bf16", page, [3, 2], table, rows, few)
    k[dev(high)], v[dev(high)] = c.k, c.v
    wide = dev(np.where(c.table.cpu().numpy() >= 0, high[np.maximum(c.table.cpu().numpy(), 0)], -1).astype(np.int32))
    pool = lava.PagePool(k, v, None, max_blocks=wide.shape[2])
    out, lse = lava.lava_shared_decode(desc, c.q, pool, wide, c.rows, c.start)
    torch.cuda.synchronize()
    c.check(out, lse)


def test_first_call_of_a_kernel_inside_a_capture(lava):
    """A step whose kernels are first launched while they are recorded."""
    rng = np.random.default_rng(22)
    table, rows, n_pages = shared_tables(rng, [5, 3], 1, 128, lambda i, g: 2, 1, 300)
    c = Case(lava, rng, 3, 1, 128, "f32", 128, [5, 3], table, rows, n_pages, softcap=9.0)
    ws = torch.full((lava.lava_shared_decode_workspace_bytes(c.desc, c.batch, c.table.shape[2]),), 0xFF, dtype=torch.uint8, device=DEV)
    out, lse = torch.empty(8, 3, 128, device=DEV), torch.empty(8, 3, device=DEV)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        lava.lava_shared_decode(c.desc, c.q, c.pool, c.table, c.rows, c.start, c.options, out=out, lse=lse, workspace=ws)
    for _ in range(3):
        out.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        c.check(out, lse)


def test_two_calls_at_once(lava):
    rng = np.random.default_rng(13)
    cases = []
    for i in range(2):
        table, rows, n_pages = shared_tables(rng, [20, 12], 4, 16, lambda a, g: 100 + 9 * g, 1, 70)
        cases.append(Case(lava, rng, 16, 4, 128, "bf16", 16, [20, 12], table, rows, n_pages))
    want = [c.run() for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    for _ in range(5):
        got = [lava.lava_shared_decode(c.desc, c.q, c.pool, c.table, c.rows, c.start, stream=s) for c, s in zip(cases, streams)]
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_binding_refuses(lava):
    rng = np.random.default_rng(14)
    table, rows, n_pages = shared_tables(rng, [2, 2], 2, 16, lambda i, g: 2, 1, 9)
    c = Case(lava, rng, 4, 2, 64, "bf16", 16, [2, 2], table, rows, n_pages)
    for start in (c.start[:1], c.start.long(), c.start.cpu()):
        with pytest.raises(ValueError):
            c.run(start=start)
    for start, status in ((torch.zeros(6, dtype=torch.int32, device=DEV), lava.LAVA_ERR_INVALID_ARG),):
        with pytest.raises(lava.LavaError) as e:
            c.run(start=start)
        assert e.value.status == status
    with pytest.raises(lava.LavaError) as e:
        c.run(workspace=torch.zeros(256, dtype=torch.uint8, device=DEV))
    assert e.value.status == lava.LAVA_ERR_WORKSPACE


# ------------------------------------------------------------------------------------------- all of them together
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("room", ["narrow", "wide"])
def test_beam_search(lava, dtype, room):
    """Two prompts of a small model of one layer: their evicted caches go to pages, become four beams each, and every step picks continuations,
    reorders, appends and attends; halfway the caches are evicted again, at the end one search is over.  Every beam's own history, kept as
    plain lists on the host, gives what it should see."""
    H, Hkv, d, page, beams, prompts, V = 8, 2, 64, 16, 4, 2, 97
    blocks = 12 if room == "narrow" else -(-ROOM // (8 * 2 * 16 * 2 * 64 * (2 if dtype == "bf16" else 4)))
    batch, heads = prompts * beams, Hkv
    rng = np.random.default_rng(31 if dtype == "bf16" else 32)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    desc = lava.LayerDesc.make(H, Hkv, d, 1, dtype)
    n_pages = batch * heads * 12
    k, v = (torch.full((n_pages, page, d), float("nan"), dtype=dt, device=DEV) for _ in range(2))
    pos = torch.full((n_pages, page), -1, dtype=torch.int32, device=DEV)
    pool = lava.PagePool(k, v, pos, max_blocks=blocks)
    state = lava.PageState.empty(batch, heads, blocks, n_pages, page)
    i32 = lambda x: dev(np.asarray(x, np.int32))
    embed = dev(rng.normal(size=(V, (H + 2 * Hkv) * d)).astype(np.float32)).to(dt)
    head = dev(rng.normal(size=(H * d, V)).astype(np.float32))
    rot = lava.RotaryDesc.make(d)
    turns = lava.lava_rotary_turns(rot, DEV)
    freqs = P.rotary_frequencies(d)
    start = i32(np.arange(prompts + 1) * beams)
    ws = torch.full((lava.lava_shared_decode_workspace_bytes(desc, batch, blocks),), 0xFF, dtype=torch.uint8, device=DEV)
    # prompts: rows of the heads of each group's first sequence, as an eviction leaves them
    counts = np.zeros((batch, heads), np.int32)
    history = [[[] for _ in range(heads)] for _ in range(batch)]      # (key, value, position) of every row a head holds, 64 bits
    seen = np.zeros(batch, np.int32)
    for i in range(prompts):
        counts[i * beams] = [37 + 20 * i, 48 - 5 * i]
        seen[i * beams] = 200
    lava.lava_page_tables(state, i32(seen), head_counts=i32(counts))
    for i in range(prompts):
        b = i * beams
        n = 200
        dense = [dev(rng.normal(size=(heads, n, d)).astype(np.float32)).to(dt) for _ in range(2)]
        kept = [np.sort(rng.permutation(n)[: counts[b, g]]) for g in range(heads)]
        offs = dev(np.concatenate([[0], np.cumsum(counts[b])]).astype(np.int64))
        lava.lava_compact_paged(desc, [lava.paged_compact_problem(desc, n, *dense, offs, i32(np.concatenate(kept)), int(counts[b].sum()),
                                                                  state.block_table[b])], pool)
        for g in range(heads):
            history[b][g] = [(dense[0][g, r].double().cpu().numpy(), dense[1][g, r].double().cpu().numpy(), int(r)) for r in kept[g]]
    source = np.repeat(np.arange(prompts) * beams, beams)
    lava.lava_page_fork(desc, pool, state, i32(source))
    history = [[list(x) for x in history[s]] for s in source]
    scores = torch.full((prompts, beams), -math.inf, device=DEV)
    scores[:, 0] = 0.0                                                 # the beams are still alike: one of each group counts
    done = torch.zeros(prompts, beams, dtype=torch.int32, device=DEV)
    logits = dev(rng.normal(size=(prompts, beams, V)).astype(np.float32) * 2.0)
    logits[:] = logits[:, :1]
    where = np.full(batch, 200)
    used_before = None
    for step in range(9):
        want = B.beam_step(logits.double().cpu().numpy(), scores.cpu().numpy(), beams, done.cpu().numpy(), end_token=3)
        sources = torch.empty(1, batch, dtype=torch.int32, device=DEV)
        parents, tokens, scores, done = lava.lava_beam_step(logits, scores, done=done, end_token=3, sources=sources)
        torch.cuda.synchronize()
        assert want[4].min() > 1e-9
        assert np.array_equal(parents.cpu().numpy(), want[0]) and np.array_equal(tokens.cpu().numpy(), want[1])
        lava.lava_page_fork(desc, pool, state, sources.view(-1))
        src = want[0].reshape(-1)
        history = [[list(x) for x in history[s]] for s in src]
        where = where[src]
        if step == 5:                                                  # memory is short: heads keep two thirds of what they hold
            rows = state.head_rows.cpu().numpy()
            keep = [[np.sort(rng.permutation(rows[b, g])[: rows[b, g] * 2 // 3]) for g in range(heads)] for b in range(batch)]
            cap = max(sum(len(x) for x in y) for y in keep)
            lists = np.array([np.pad(np.concatenate(y), (0, cap - sum(len(x) for x in y)), constant_values=-1) for y in keep])
            lava.lava_page_compact(desc, pool, state, i32([[len(x) for x in y] for y in keep]), i32(lists))
            history = [[[history[b][g][r] for r in keep[b][g]] for g in range(heads)] for b in range(batch)]
        new = np.ones(batch, np.int32)
        slots = torch.empty(batch, heads, dtype=torch.int64, device=DEV)
        positions = torch.empty(batch, dtype=torch.int32, device=DEV)
        lava.lava_page_tables(state, i32(new), slots=slots, positions=positions)
        x = embed[tokens.view(-1).long()].view(batch, H + 2 * Hkv, d)
        q, kk, vv = x[:, :H], x[:, H: H + Hkv], x[:, H + Hkv:]
        q_rot = lava.lava_rotary_append(desc, rot, turns, positions, q, kk, vv, pool, slots)
        out, lse = lava.lava_shared_decode(desc, q_rot, pool, state.block_table, state.head_rows, start, workspace=ws)
        plain, plain_lse = lava.lava_paged_decode(desc, q_rot, pool, state.block_table, state.head_rows)
        torch.cuda.synchronize()
        assert int(state.error[0]) == 0 and np.array_equal(positions.cpu().numpy(), where)
        turned = P.rotary(kk.double().cpu().numpy(), where, freqs)
        stored_k = k.view(-1, d)[slots.view(-1)].double().cpu().numpy().reshape(batch, heads, d)
        for b in range(batch):
            for g in range(heads):
                # one rounding to the storage type, the 32-bit arithmetic before it far below
                assert np.abs(stored_k[b, g] - turned[b, g]).max() <= np.abs(turned[b, g]).max() * (2.0 ** -8 if dtype == "bf16" else 2.0 ** -20)
                history[b][g].append((stored_k[b, g], vv[b, g].double().cpu().numpy(), int(where[b])))
        where = where + 1
        assert torch.allclose(lse, plain_lse, rtol=0, atol=2e-5) and float((out - plain).abs().max()) < 1e-4
        # what every beam should see, from its history, as pages of one row each
        rows = np.array([[len(history[b][g]) for g in range(heads)] for b in range(batch)], np.int32)
        assert np.array_equal(rows, state.head_rows.cpu().numpy())
        flat_k = np.array([r[0] for b in range(batch) for g in range(heads) for r in history[b][g]])
        flat_v = np.array([r[1] for b in range(batch) for g in range(heads) for r in history[b][g]])
        t = np.zeros((batch, heads, rows.max()), np.int32)
        at = 0
        for b in range(batch):
            for g in range(heads):
                t[b, g, : rows[b, g]] = np.arange(at, at + rows[b, g])
                at += rows[b, g]
        ref, ref_lse, tol, tol_lse = P.paged_decode(q_rot.double().cpu().numpy(), flat_k[:, None], flat_v[:, None], t, rows, d ** -0.5)
        weight = np.abs(ref_lse) * 2.0 ** -21 + 2.0 ** -17
        assert (np.abs(out.double().cpu().numpy() - ref) <= tol + (weight[..., None] + 2.0 ** -22) * np.abs(flat_v).max()).all()
        logits = (out.view(batch, H * d) @ head / 4.0).view(prompts, beams, V)
        held = set(int(p) for b in range(batch) for g in range(heads) for p in state.block_table[b, g, : -(-int(rows[b, g]) // page)])
        assert len(held) + int(state.n_free[0]) == n_pages
        used_before = len(held)
    assert used_before < batch * heads * -(-int(rows.max()) // page)   # pages are shared
    lava.lava_page_fork(desc, pool, state, i32([-1] * beams + list(range(beams, batch))))
    lava.lava_page_fork(desc, pool, state, i32([-1] * batch))
    torch.cuda.synchronize()
    assert int(state.n_free[0]) == n_pages and sorted(state.free_pages.tolist()) == list(range(n_pages)) and int(state.error[0]) == 0
