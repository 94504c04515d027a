"""The paged cache on the GPU against its oracle: block tables and slots (equal integers), rotary positions and decode over pages
(within the roundings of 32-bit arithmetic, bounded beside each), the gather into pages (equal bits), and all of them together
as a serving loop uses them."""
import math

import numpy as np
import pytest

from oracle import lava_oracle as O
from oracle import paged_oracle as P
from paper_2509_09754_amd import synth
from test_paged_oracle_pins import owned, random_state

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
DEV = "cuda"


@pytest.fixture(scope="module")
def lava():
    from paper_2509_09754_amd import lava as L
    return L


def say(*a):
    print(*a, flush=True)


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def host(t):
    return t.cpu().numpy()


# ------------------------------------------------------------------------------------------- block tables
class Tables:
    """A state on the device with canaries behind every buffer."""

    def __init__(self, lava, page, table, rows, pos, free, n_free, in_place=False):
        self.lava, self.page, self.table_in = lava, page, table
        self.bufs = {}
        for name, a in (("table", table), ("rows", rows), ("pos", pos), ("free", free), ("n_free", np.array([n_free], np.int32))):
            self.bufs[name] = self._guarded(a)
        for name in ("rows", "pos", "n_free"):
            self.bufs[name + "_out"] = self.bufs[name] if in_place else self._guarded(np.full_like(host(self.view(name)), 99))
        self.bufs["error"] = self._guarded(np.zeros(1, np.int32))
        v = self.view
        self.state = lava.PageState(v("table"), v("rows"), v("pos"), v("free"), v("n_free"), page, v("rows_out"), v("pos_out"),
                                    v("n_free_out"), v("error"))

    def _guarded(self, a):
        t = torch.full((a.size + 64,), -77, dtype=torch.int32, device=DEV)
        t[: a.size] = dev(a.reshape(-1))
        return t, a.shape

    def view(self, name):
        t, shape = self.bufs[name]
        return t[: int(np.prod(shape))].view(*shape)

    def step(self, n_new=None, head_counts=None, release=None, max_tokens=0, workspace=None):
        i32 = lambda x: None if x is None else dev(np.asarray(x, np.int32))
        heads = self.table_in.shape[1]
        slots = torch.full((max_tokens + 3, heads), 55, dtype=torch.int64, device=DEV)
        positions = torch.full((max_tokens + 3,), 55, dtype=torch.int32, device=DEV)
        self.lava.lava_page_tables(self.state, i32(n_new), i32(head_counts), i32(release), slots[:max_tokens] if max_tokens else None,
                                   positions[:max_tokens] if max_tokens else None, workspace=workspace)
        torch.cuda.synchronize()
        assert bool((slots[max_tokens:] == 55).all()) and bool((positions[max_tokens:] == 55).all())
        for t, shape in self.bufs.values():
            assert bool((t[int(np.prod(shape)):] == -77).all())
        return [host(self.view(x)) for x in ("table", "rows_out", "pos_out", "free")] + [
            int(self.view("n_free_out")[0]), host(slots[:max_tokens]), host(positions[:max_tokens]), int(self.view("error")[0])]


def check_step(got, want):
    for name, a, b in zip(("table", "rows", "pos", "free", "n_free", "slots", "positions", "error"), got, want):
        assert np.array_equal(a, b), name


# one head; a few; more than a thousand heads and than a thousand sequences; long prompts; pages of every size
@pytest.mark.parametrize("batch,heads,page,max_blocks,new_hi", [
    (1, 1, 16, 4, 3), (1, 1, 256, 2, 300), (3, 2, 16, 9, 60), (64, 8, 64, 6, 1), (7, 64, 32, 5, 50), (130, 8, 32, 6, 40),
    (1025, 1, 16, 3, 9), (700, 5, 128, 3, 2), (2, 3, 16, 500, 4000), (300, 32, 16, 6, 20)])
@pytest.mark.parametrize("mode", ["tokens", "counts", "turnover"])
def test_tables(lava, batch, heads, page, max_blocks, new_hi, mode):
    say(f"tables {batch}x{heads} page {page} {mode}")
    rng = np.random.default_rng(batch * 1000 + heads + new_hi)
    n_pages = batch * heads * max_blocks
    for trial in range(3):
        table, rows, pos, free, n_free = random_state(rng, batch, heads, max_blocks, page, n_pages, 0.5)
        room = max_blocks * page - rows.max(1)
        new = np.minimum(rng.integers(0, new_hi + 1, batch), room)
        if trial == 2:
            new[:] = 0                                             # a step without tokens
        release = counts = None
        tokens = int(new.sum()) + int(rng.integers(0, 4))
        if mode != "tokens":
            release = (rng.random(batch) < 0.3).astype(np.int32) * -5 if mode == "turnover" else None
        if mode == "counts":
            counts, tokens = np.minimum(rng.integers(0, new_hi + 1, (batch, heads)), room[:, None]), 0
        t = Tables(lava, page, table, rows, pos, free, n_free, in_place=trial == 1)
        check_step(t.step(new, counts, release, tokens),
                   P.page_tables(page, n_pages, table, rows, pos, free, n_free, new, counts, release, tokens))


def test_tables_of_nothing_new(lava):
    rng = np.random.default_rng(3)
    table, rows, pos, free, n_free = random_state(rng, 4, 2, 5, 16, 40, 0.5)
    t = Tables(lava, 16, table, rows, pos, free, n_free)
    check_step(t.step(), P.page_tables(16, 40, table, rows, pos, free, n_free))
    check_step(t.step(None, None, [1, 0, 0, 1]), P.page_tables(16, 40, table, rows, pos, free, n_free, release=[1, 0, 0, 1]))


@pytest.mark.parametrize("heads,batch", [(2, 3), (8, 400)])
def test_tables_refuse_on_the_device(lava, heads, batch):
    """A step that cannot be carried out changes nothing and says why."""
    say(f"tables refused {batch}x{heads}")
    rng = np.random.default_rng(4)
    page, mb = 16, 4
    n_pages = batch * heads * mb
    table, rows, pos, free, n_free = random_state(rng, batch, heads, mb, page, n_pages, 0.4)
    one = np.ones(batch, np.int32)
    last = np.where(np.arange(batch) == batch - 1, 1, 0)
    big = lambda x: one + last * x
    cases = [(dict(n_new=big(10 * page)), P.BLOCKS, {}), (dict(n_new=one, max_tokens=batch - 1), P.TOKENS, {}),
             (dict(n_new=one - 2 * last, max_tokens=batch), P.INVALID, {}), (dict(n_new=one, max_tokens=batch), P.EXHAUSTED, dict(n_free=0)),
             (dict(head_counts=np.where(np.arange(heads) == heads - 1, -1, 1) * np.ones((batch, 1), int)), P.INVALID, {}),
             (dict(n_new=one), P.INVALID, dict(n_free=-1)), (dict(n_new=one), P.INVALID, dict(n_free=n_pages + 1)),
             (dict(release=one), P.INVALID, dict(n_free=n_pages)), (dict(n_new=one), P.INVALID, dict(rows=mb * page + 1)),
             (dict(n_new=one), P.INVALID, dict(rows=-3)), (dict(n_new=one), P.INVALID, dict(pos=-1)),
             (dict(n_new=one), P.INVALID, dict(pos=2 ** 31 - 1))]
    full = rows.copy()
    full[:, :] = page * 2                                          # the next row of every head needs a page
    for kw, reason, over in cases:
        r, p, f = (full if reason == P.EXHAUSTED else rows).copy(), pos.copy(), n_free
        if "rows" in over:
            r[-1, -1] = over["rows"]
        if "pos" in over:
            p[-1] = over["pos"]
        f = over.get("n_free", f)
        t = Tables(lava, page, table, r, p, free, f)
        got = t.step(**kw)
        want = P.page_tables(page, n_pages, table, r, p, free, f, **kw)
        assert want[7] & reason
        check_step(got, want)
        good = P.page_tables(page, n_pages, table, rows, pos, free, n_free, one * 0)
        assert good[7] == 0
        t.view("rows").copy_(dev(rows)), t.view("pos").copy_(dev(pos)), t.view("n_free").fill_(n_free)
        assert t.step(one * 0)[7] == want[7]                       # the word collects; a good step clears nothing


def test_tables_replay(lava):
    """A captured decode step in place, replayed while eager steps and other work run in between."""
    say("tables: graph replays")
    rng = np.random.default_rng(6)
    batch, heads, page, mb = 5, 4, 16, 8
    n_pages = 200
    table, rows, pos, free, n_free = random_state(rng, batch, heads, mb, page, n_pages, 0.3)
    t = Tables(lava, page, table, rows, pos, free, n_free, in_place=True)
    new, release = dev(np.ones(batch, np.int32)), dev(np.zeros(batch, np.int32))
    slots = torch.zeros(batch + 1, heads, dtype=torch.int64, device=DEV)
    positions = torch.zeros(batch + 1, dtype=torch.int32, device=DEV)
    ws = torch.full((lava.lava_page_tables_workspace_bytes(batch, heads),), 0xAB, dtype=torch.uint8, device=DEV)
    call = lambda: lava.lava_page_tables(t.state, new, release=release, slots=slots, positions=positions, workspace=ws)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    cur = (table, rows, pos, free, n_free)
    for i in range(40):
        rel = (rng.random(batch) < 0.1).astype(np.int32)
        n = rng.integers(0, 2, batch).astype(np.int32)
        new.copy_(dev(n)), release.copy_(dev(rel))
        want = P.page_tables(page, n_pages, *cur, n, None, rel, batch + 1)
        graph.replay() if i % 3 else call()
        torch.cuda.synchronize()
        got = [host(t.view(x)) for x in ("table", "rows", "pos", "free")] + [int(t.view("n_free")[0]), host(slots), host(positions),
                                                                            int(t.view("error")[0])]
        check_step(got, want)
        cur = want[:5]
        assert sorted(owned(cur[0], cur[1], page) + [int(x) for x in cur[3][: cur[4]]]) == list(range(n_pages))


# ------------------------------------------------------------------------------------------- rotary
def stored(rng, shape, dtype):
    return synth.store(rng.standard_normal(shape, dtype=np.float32), dtype)


def rotary_tolerance(x, magnitude, freqs, positions, interleaved, dtype, want):
    """Sine and cosine are within 2^-22 (the angle to 24 bits, its factor, the polynomial), their product with the magnitude,
    two products and a sum round once each: 2^-21 of |a| + |b|; then the rounding to the storage type, half a step.  The
    frequencies here are doubles: 2^-50 of the angle."""
    half = len(freqs)
    a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    tol = np.zeros_like(want)
    angle = np.abs(np.asarray(positions, np.float64))[:, None, None] * freqs * 2.0 ** -50
    size = (np.abs(x[..., a]) + np.abs(x[..., b])) * magnitude
    tol[..., a] = tol[..., b] = size * (2.0 ** -21 + angle)
    if dtype == "bf16":
        tol[..., : 2 * half] += 2.0 ** -8 * (np.abs(want[..., : 2 * half]) + tol[..., : 2 * half])
    return tol


LAYOUTS = [(128, 128, False), (128, 128, True), (128, 64, False), (128, 96, True), (128, 38, False), (128, 38, True), (128, 2, False),
           (128, 2, True), (64, 64, False), (64, 64, True), (64, 48, False), (64, 18, True), (64, 30, False), (64, 16, False)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,rot,interleaved", LAYOUTS)
def test_rotary(lava, d, rot, interleaved, dtype):
    say(f"rotary d{d} rot {rot} interleaved {interleaved} {dtype}")
    rng = np.random.default_rng(d + rot)
    for tokens, heads, transpose, magnitude in ((1, 1, False, 0.0), (5, 3, True, 1.25), (67, 7, False, 1.0)):
        x = stored(rng, (tokens, heads, d), dtype)
        pos = rng.integers(0, 1 << 20, tokens).astype(np.int32)
        pos[0] = (2 ** 31 - 1, 0, 131071)[heads % 3]
        if tokens > 2:
            pos[tokens // 2] = -1                                  # left out
        kw = dict(base=500000.0, factor=4.0)
        desc = lava.RotaryDesc.make(rot, interleaved, magnitude, **kw)
        turns = lava.lava_rotary_turns(desc, DEV)
        xd = lava.to_device(x, dtype)
        outs = {"rows": torch.full_like(xd, 7.0), "in place": xd.clone()}
        heads_first = torch.full((heads, tokens, d), 7.0, dtype=xd.dtype, device=DEV)
        outs["heads first"] = heads_first.transpose(0, 1)
        wide = torch.full((tokens, 3 * heads, d), 7.0, dtype=xd.dtype, device=DEV)
        outs["part"] = wide[:, heads: 2 * heads]
        for name, out in outs.items():
            lava.lava_rotary(desc, turns, dev(pos), out if name == "in place" else xd, out=out, transpose=transpose)
        torch.cuda.synchronize()
        f = P.rotary_frequencies(rot, **kw)
        x64 = synth.load_f64(x, dtype)
        want = P.rotary(x64, pos, f, interleaved, magnitude or 1.0, transpose)
        tol = rotary_tolerance(x64, magnitude or 1.0, f, pos, interleaved, dtype, want)
        first = outs["rows"]
        got = host(first.double())
        skip = pos < 0
        assert (got[skip] == 7.0).all()
        assert (np.abs(got - want)[~skip] <= tol[~skip]).all()
        assert np.array_equal(lava.to_host_bits(first)[~skip][..., rot:], x[~skip][..., rot:])   # the rest passes bit for bit
        for name, out in outs.items():
            keep = torch.from_numpy(~skip).to(DEV)
            assert torch.equal(out[keep], first[keep]), name
            if skip.any():
                assert bool((out[~keep] == (xd[~keep] if name == "in place" else 7.0)).all()), name
        assert bool((wide[:, :heads] == 7.0).all()) and bool((wide[:, 2 * heads:] == 7.0).all())


def test_rotary_broadcast_and_special_values(lava):
    """One row for all heads; infinities and NaN stay in their pair."""
    d, rot = 64, 32
    desc = lava.RotaryDesc.make(rot)
    turns = lava.lava_rotary_turns(desc, DEV)
    x = torch.randn(6, 1, d, device=DEV)
    x[2, 0, 5], x[3, 0, 40] = math.inf, math.nan
    pos = torch.arange(6, dtype=torch.int32, device=DEV)
    one = lava.lava_rotary(desc, turns, pos, x)
    many = lava.lava_rotary(desc, turns, pos, x.expand(6, 5, d))
    torch.cuda.synchronize()
    assert torch.equal(many.nan_to_num(9.0, 8.0, 7.0), one.expand(6, 5, d).nan_to_num(9.0, 8.0, 7.0))
    bad = ~torch.isfinite(one)
    assert bad[2, 0].nonzero().view(-1).tolist() == [5, 5 + rot // 2] and bad[3, 0].nonzero().view(-1).tolist() == [40]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rotary_gradient(lava, dtype):
    """The transposed rotation of a cotangent against differences of <cotangent, rotary(x)> and against the formula."""
    rng = np.random.default_rng(8)
    d, rot, tokens = 64, 48, 3
    desc = lava.RotaryDesc.make(rot, True, 1.125)
    turns = lava.lava_rotary_turns(desc, DEV)
    pos = np.array([3, 99, 12345], np.int32)
    g = stored(rng, (tokens, 2, d), dtype)
    grad = lava.lava_rotary(desc, turns, dev(pos), lava.to_device(g, dtype), transpose=True)
    f = P.rotary_frequencies(rot)
    g64 = synth.load_f64(g, dtype)
    want = P.rotary(g64, pos, f, True, 1.125, transpose=True)
    assert (np.abs(host(grad.double()) - want) <= rotary_tolerance(g64, 1.125, f, pos, True, dtype, want)).all()
    if dtype == "f32":                                             # the map is linear: a difference quotient of step 1 is exact but
        x = torch.randn(tokens, 2, d, device=DEV)                  # for roundings of products of size up to |g| |x|
        for e in (0, 1, 30, 50):
            step = torch.zeros_like(x)
            step[:, :, e] = 1.0
            hi, lo = (lava.lava_rotary(desc, turns, dev(pos), y).double() for y in (x + step, x))
            dq = ((hi - lo) * torch.from_numpy(g64).to(DEV)).sum(-1)
            assert float((dq - grad[:, :, e].double()).abs().max()) <= 2.0 ** -18 * float(np.abs(g64).max() * x.abs().max() + 4)


@pytest.mark.parametrize("H,Hkv,d,dtype,page,rot,interleaved,fused", [
    (32, 8, 128, "bf16", 64, 128, False, True), (4, 4, 64, "bf16", 16, 38, False, False), (8, 2, 64, "f32", 32, 32, True, True),
    (7, 1, 128, "f32", 128, 128, True, False), (28, 4, 128, "bf16", 256, 96, True, True)])
@pytest.mark.parametrize("tokens", [1, 3, 130])
def test_append(lava, H, Hkv, d, dtype, page, rot, interleaved, fused, tokens):
    say(f"append H{H}/{Hkv} d{d} {dtype} page {page} rot {rot} tokens {tokens}")
    rng = np.random.default_rng(tokens + H)
    desc = lava.LayerDesc.make(H, Hkv, d, 1, dtype)
    n_pages = tokens * Hkv // page + Hkv + 2
    slots = rng.permutation(n_pages * page)[: tokens * Hkv].reshape(tokens, Hkv).astype(np.int64)
    pos = rng.integers(0, 100000, tokens).astype(np.int32)
    if tokens > 2:
        slots[1, 0], pos[2] = -1, -1                               # one row and one token left out
        slots[0, Hkv - 1] = n_pages * page                         # not in the pool
    x = stored(rng, (tokens, H + 2 * Hkv, d), dtype)
    xd = lava.to_device(x, dtype)
    q, k, v = (t if fused else t.contiguous() for t in (xd[:, :H], xd[:, H: H + Hkv], xd[:, H + Hkv:]))
    dt = desc.torch_dtype
    kp, vp = (torch.full((n_pages, page, d), 3.0, dtype=dt, device=DEV) for _ in range(2))
    pp = torch.full((n_pages, page), -3, dtype=torch.int32, device=DEV)
    rot_desc = lava.RotaryDesc.make(rot, interleaved)
    q_out = torch.full((tokens, H, d), 3.0, dtype=dt, device=DEV)
    turns = lava.lava_rotary_turns(rot_desc, DEV)
    lava.lava_rotary_append(desc, rot_desc, turns, dev(pos), q, k, v, lava.PagePool(kp, vp, pp), dev(slots), q_out=q_out)
    f = P.rotary_frequencies(rot)
    x64 = synth.load_f64(x, dtype)
    want = P.rotary(x64, pos, f, interleaved)
    tol = rotary_tolerance(x64, 1.0, f, pos, interleaved, dtype, want)
    got_q, got_k, got_v, got_p = host(q_out.double()), host(kp.double()).reshape(-1, d), host(vp.double()).reshape(-1, d), host(pp).reshape(-1)
    seen = np.zeros(n_pages * page, bool)
    for t in range(tokens):
        if pos[t] < 0:
            assert (got_q[t] == 3.0).all()
            continue
        assert (np.abs(got_q[t] - want[t, :H]) <= tol[t, :H]).all()
        for g in range(Hkv):
            s = slots[t, g]
            if s < 0 or s >= n_pages * page:
                continue
            seen[s] = True
            assert (np.abs(got_k[s] - want[t, H + g]) <= tol[t, H + g]).all()
            assert np.array_equal(got_v[s], x64[t, H + Hkv + g]) and got_p[s] == pos[t]
    assert (got_k[~seen] == 3.0).all() and (got_v[~seen] == 3.0).all() and (got_p[~seen] == -3).all()
    # the cache alone, without positions; queries in place
    kp2, vp2 = torch.full_like(kp, 3.0), torch.full_like(vp, 3.0)
    lava.lava_rotary_append(desc, rot_desc, turns, dev(pos), None, k, v, lava.PagePool(kp2, vp2), dev(slots))
    q2 = q.contiguous().clone()
    lava.lava_rotary_append(desc, rot_desc, turns, dev(pos), q2, k, v, lava.PagePool(kp2, vp2), dev(slots), q_out=q2)
    torch.cuda.synchronize()
    assert torch.equal(kp2, kp) and torch.equal(vp2, vp)
    real = torch.from_numpy(pos >= 0).to(DEV)
    assert torch.equal(q2[real], q_out[real]) and torch.equal(q2[~real], q[~real])


# ------------------------------------------------------------------------------------------- gather into pages
@pytest.mark.parametrize("Hkv,d,dtype,page,packed", [(8, 128, "bf16", 64, False), (2, 64, "f32", 16, False), (3, 128, "f32", 32, True),
                                                     (1, 64, "bf16", 256, True), (64, 64, "bf16", 16, False)])
def test_compact_paged(lava, Hkv, d, dtype, page, packed):
    say(f"compact into pages Hkv{Hkv} d{d} {dtype} page {page} packed {packed}")
    rng = np.random.default_rng(Hkv + page)
    desc = lava.LayerDesc.make(Hkv, Hkv, d, 1, dtype)
    batch, mb = 3, 6
    n_pages = batch * Hkv * mb
    kp, vp = (torch.full((n_pages, page, d), 3.0, dtype=desc.torch_dtype, device=DEV) for _ in range(2))
    pp = torch.full((n_pages, page), -3, dtype=torch.int32, device=DEV)
    order = rng.permutation(n_pages).astype(np.int32)
    pool = lava.PagePool(kp, vp, pp, max_blocks=mb)
    problems, keep, expect = [], [], []
    for b in range(batch):
        lens = rng.integers(1, 3 * page, Hkv) if packed else np.full(Hkv, 2 * page + 5 + b)
        start = np.concatenate([[0], np.cumsum(lens)])
        k, v = stored(rng, (int(start[-1]), d), dtype), stored(rng, (int(start[-1]), d), dtype)
        counts = [0 if b == 2 else int(rng.integers(0, n + 1)) for n in lens]     # the last one keeps nothing
        offs = np.concatenate([[0], np.cumsum(counts)]).astype(np.int64)
        idx = np.concatenate([np.sort(rng.permutation(n)[:c]) for n, c in zip(lens, counts)] + [[]]).astype(np.int32)
        idx = np.concatenate([idx, np.full(4, 1 << 20)]).astype(np.int32)
        table = order[b * Hkv * mb: (b + 1) * Hkv * mb].reshape(Hkv, mb).copy()
        first = rng.integers(0, page + 2, Hkv).astype(np.int32) if b else None
        if b == 1:
            table[0, 0], table[-1, -1] = -1, n_pages                # pages that are none
            if idx.size > 6:
                idx[1] = 1 << 24                                    # a source row that is none
        pos = rng.integers(0, 9999, int(start[-1])).astype(np.int32) if packed else None
        t = [lava.to_device(k, dtype), lava.to_device(v, dtype), dev(offs), dev(idx), dev(table)]
        src = dict(src_offsets=dev(start.astype(np.int64)), pos_src=dev(pos)) if packed else {}
        t += list(src.values())
        if first is not None:
            t.append(dev(first))
            src["first_rows"] = t[-1]
        keep.append(t)
        cap = max(int(offs[-1]) - (3 if b == 1 else 0), 0)          # survivors beyond the capacity are not written
        problems.append(lava.paged_compact_problem(desc, int(start[-1]) if packed else int(lens[0]), t[0], t[1], t[2], t[3], cap, t[4], **src))
        segs = [(int(s), int(n)) for s, n in zip(start[:-1], lens)]
        offs_cap = np.minimum(offs, cap)
        for slot, row, i in P.compact_paged(n_pages, page, mb, offs_cap, idx, segs, table, first):
            expect.append((slot, k[row], v[row], int(pos[row]) if packed else i))
    lava.lava_compact_paged(desc, problems, pool)
    torch.cuda.synchronize()
    got_k, got_v, got_p = lava.to_host_bits(kp).reshape(-1, d), lava.to_host_bits(vp).reshape(-1, d), host(pp).reshape(-1)
    blank = lava.to_host_bits(torch.full((1,), 3.0, dtype=desc.torch_dtype, device=DEV))[0]
    seen = np.zeros(n_pages * page, bool)
    for slot, krow, vrow, p in expect:
        seen[slot] = True
        assert np.array_equal(got_k[slot], krow) and np.array_equal(got_v[slot], vrow) and got_p[slot] == p
    assert (got_k[~seen] == blank).all() and (got_v[~seen] == blank).all() and (got_p[~seen] == -3).all()


def test_compact_paged_many_problems(lava):
    """More problems than one launch takes; one selection that gave up."""
    say("compact into pages: 40 problems")
    rng = np.random.default_rng(11)
    desc = lava.LayerDesc.make(2, 2, 64, 1, "bf16")
    page, mb, n = 16, 2, 50
    kp, vp = (torch.zeros(160, page, 64, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    k, v = (torch.randn(40, 2, n, 64, device=DEV).bfloat16() for _ in range(2))
    table = torch.arange(160, dtype=torch.int32, device=DEV).view(40, 2, mb)
    offs = torch.tensor([0, 20, 32], device=DEV).repeat(40, 1)
    offs[7] = 0
    idx = dev(np.stack([np.concatenate([np.sort(rng.permutation(n)[:20]), np.sort(rng.permutation(n)[:12])]) for _ in range(40)]).astype(np.int32))
    lava.lava_compact_paged(desc, [lava.paged_compact_problem(desc, n, k[i], v[i], offs[i], idx[i], 32, table[i]) for i in range(40)],
                            lava.PagePool(kp, vp, max_blocks=mb))
    torch.cuda.synchronize()
    kp, vp = kp.view(40, 2, mb * page, 64), vp.view(40, 2, mb * page, 64)
    assert not bool(kp[7].any())
    for i in range(40):
        if i == 7:
            continue
        for g, (a, c) in enumerate(((0, 20), (20, 12))):
            rows = idx[i, a: a + c].long()
            assert torch.equal(kp[i, g, :c], k[i, g, rows]) and torch.equal(vp[i, g, :c], v[i, g, rows]) and not bool(kp[i, g, c:].any())


# ------------------------------------------------------------------------------------------- decode over pages
class Decode:
    """Pages, tables and queries of one case; what lies behind the last row of a head is NaN, unused table entries are wild."""

    def __init__(self, lava, H, Hkv, d, dtype, page, rows, seed, spare=2, scale=0.0):
        rng = np.random.default_rng(seed)
        self.lava, self.rows, self.page, self.dtype = lava, np.asarray(rows, np.int32), page, dtype
        batch = self.rows.shape[0]
        nb = -(-self.rows // page)
        mb = max(1, int(nb.max())) + 1
        n_pages = int(nb.sum()) + spare
        order = rng.permutation(n_pages).astype(np.int32)
        self.table, at = np.full((batch, Hkv, mb), 1 << 30, np.int32), 0
        self.k, self.v = (synth.store(rng.standard_normal((n_pages, page, d), dtype=np.float32), dtype) for _ in range(2))
        nan = synth.store(np.full(1, np.nan, np.float32), dtype)[0] if dtype == "f32" else np.uint16(0x7FC0)
        used = np.zeros((n_pages, page), bool)
        self.pos = np.full((n_pages, page), 1 << 29, np.int32)
        newest = np.zeros(batch, np.int32)                         # position of a sequence's newest row
        for b in range(batch):
            for g in range(Hkv):
                n = int(self.rows[b, g])
                self.table[b, g, : nb[b, g]] = order[at: at + nb[b, g]]
                at += nb[b, g]
                p = np.sort(rng.permutation(4 * n + 8)[:n]).astype(np.int32)
                newest[b] = max(newest[b], p.max(initial=0))
                for j in range(nb[b, g]):
                    c = min(page, n - j * page)
                    used[self.table[b, g, j], :c] = True
                    self.pos[self.table[b, g, j], :c] = p[j * page: j * page + c]
        self.k[~used], self.v[~used] = nan, nan
        self.q = synth.store(rng.standard_normal((batch, H, d), dtype=np.float32), dtype)
        self.desc = lava.LayerDesc.make(H, Hkv, d, 1, dtype, softmax_scale=scale)
        self.scale = scale or 1.0 / math.sqrt(d)
        self.slopes = (2.0 ** (-8.0 * (1 + np.arange(H)) / H)).astype(np.float32)
        self.q_pos = newest
        self.need = lava.lava_paged_decode_workspace_bytes(self.desc)
        self.ws = torch.full((self.need + 4096,), 0xFF, dtype=torch.uint8, device=DEV)
        self.ws[self.need:] = 0x5A
        self.dev = dict(q=lava.to_device(self.q, dtype), k=lava.to_device(self.k, dtype), v=lava.to_device(self.v, dtype), pos=dev(self.pos),
                        table=dev(self.table), rows=dev(self.rows), slopes=dev(self.slopes), q_pos=dev(self.q_pos))
        self.pool = lava.PagePool(self.dev["k"], self.dev["v"], self.dev["pos"], max_blocks=mb)
        self.out = torch.full((batch, H, d), 777.0, device=DEV)
        self.lse = torch.full((batch, H), 777.0, device=DEV)

    def run(self, softcap=0.0, window=0, bias=False):
        o = self.lava.DecodeOptions.make(softcap, window, self.dev["slopes"] if bias else None)
        self.lava.lava_paged_decode(self.desc, self.dev["q"], self.pool, self.dev["table"], self.dev["rows"], o if softcap or window or bias else None,
                                    self.dev["q_pos"] if window or bias else None, self.out, self.lse, self.ws[: self.need])
        torch.cuda.synchronize()
        assert bool((self.ws[self.need:] == 0x5A).all())
        return host(self.out.double()), host(self.lse.double())

    def check(self, softcap=0.0, window=0, bias=False):
        out, lse = self.run(softcap, window, bias)
        f = lambda x: synth.load_f64(x, self.dtype)
        want, want_lse, tol, tol_lse = P.paged_decode(f(self.q), f(self.k), f(self.v), self.table, self.rows, self.scale, softcap, window,
                                                      self.slopes if bias else None, self.pos, self.q_pos)
        assert np.array_equal(np.isnan(out), np.isnan(want)) and np.array_equal(np.isfinite(lse), np.isfinite(want_lse))
        ok, okl = ~np.isnan(want), np.isfinite(want_lse)
        worst = np.abs(out - want)[ok] / np.maximum(tol[ok], 1e-30) if ok.any() else np.zeros(1)
        say(f"   worst {worst.max():.3f} of the bound")
        assert (np.abs(out - want)[ok] <= tol[ok]).all()
        assert (np.abs(lse[okl] - want_lse[okl]) <= tol_lse[okl]).all()
        return out


# groups of every padded size, both types and head sizes, pages of every size; heads with nothing, one row, a tile and one
# more, many pages
ROWS = [[0, 1], [31, 32], [33, 200]]
SHAPES = [(2, 2, 128, "bf16", 16), (4, 2, 64, "bf16", 32), (6, 2, 128, "bf16", 64), (14, 2, 128, "bf16", 16), (16, 2, 64, "f32", 128),
          (8, 2, 128, "f32", 16), (2, 2, 64, "f32", 256), (10, 2, 64, "bf16", 16), (12, 2, 128, "f32", 64)]


@pytest.mark.parametrize("H,Hkv,d,dtype,page", SHAPES)
def test_decode(lava, H, Hkv, d, dtype, page):
    say(f"paged decode H{H}/{Hkv} d{d} {dtype} page {page}")
    c = Decode(lava, H, Hkv, d, dtype, page, ROWS, H + page)
    first = c.check()
    c.ws.fill_(0x00), c.ws[c.need:].fill_(0x5A)
    for _ in range(3):                                             # the same bits over any workspace, as the call before left it too
        assert np.array_equal(c.run()[0], first)


@pytest.mark.parametrize("H,Hkv,d,dtype,page", SHAPES)
@pytest.mark.parametrize("softcap,window,bias", [(20.0, 0, False), (0.0, 40, False), (0.0, 0, True), (5.0, 100, True), (0.0, 1, True)])
def test_decode_options(lava, H, Hkv, d, dtype, page, softcap, window, bias):
    say(f"paged decode options H{H}/{Hkv} d{d} {dtype} page {page} cap {softcap} window {window} bias {bias}")
    Decode(lava, H, Hkv, d, dtype, page, ROWS, H + page + 1).check(softcap, window, bias)


@pytest.mark.parametrize("rows,page,Hkv", [
    ([[5000, 3, 129, 0]], 16, 4), ([[20000]], 64, 1), ([[700]] * 37, 32, 1), ([[17, 400, 63, 64, 65, 0, 1, 3000]] * 9, 16, 8),
    ([[0]] * 5 + [[9000]], 128, 1), ([[1] * 8] * 70, 16, 8), ([[33, 2]] * 150, 16, 2)])
def test_decode_splits(lava, rows, page, Hkv):
    """Heads split over many workgroups and workgroups that hold many heads."""
    say(f"paged decode splits {len(rows)} sequences, page {page}")
    c = Decode(lava, 4 * Hkv, Hkv, 128, "bf16", page, rows, 7 + len(rows))
    first = c.check()
    assert np.array_equal(c.run()[0], first)
    c.check(softcap=30.0, window=300, bias=True)


def test_decode_masked_values(lava):
    """Rows outside the window hold infinities and NaN; so does a whole head."""
    say("paged decode: masked infinities")
    for dtype, page in (("bf16", 32), ("f32", 16)):
        c = Decode(lava, 4, 2, 128, dtype, page, [[300, 40], [200, 10]], 5)
        window = 150
        for b in range(2):
            for g in range(2):
                for r in range(int(c.rows[b, g])):
                    at = c.table[b, g, r // page], r % page
                    if not 0 <= c.q_pos[b] - c.pos[at] < window or (b, g) == (1, 1):
                        c.pos[at] = -(1 << 20) if (b, g) == (1, 1) else c.pos[at]
                        c.k[at], c.v[at] = (np.float32(np.inf), np.float32(np.nan)) if dtype == "f32" else (np.uint16(0x7F80), np.uint16(0x7FC0))
        for name in ("k", "v"):
            c.dev[name].copy_(lava.to_device(getattr(c, name), dtype))
        c.dev["pos"].copy_(dev(c.pos))
        out = c.check(window=window)
        assert (out[1, 2:] == 0).all()


def test_decode_refuses_on_the_device(lava):
    """A row count out of range or a page that is not in the pool: NaN for that head, the others as they are."""
    say("paged decode: bad tables")
    for window in (0, 50):
        for what in ("rows", "huge", "page", "negative"):
            c = Decode(lava, 8, 2, 128, "bf16", 32, [[100, 700], [60, 40]], 9)
            if what == "rows":
                c.rows[0, 1] = -1
            elif what == "huge":
                c.rows[0, 1] = c.table.shape[2] * 32 + 1
            else:
                c.table[0, 1, 11] = c.k.shape[0] if what == "page" else -1
            c.dev["rows"].copy_(dev(c.rows)), c.dev["table"].copy_(dev(c.table))
            out = c.check(window=window)
            assert np.isnan(out[0, 4:]).all() and np.isfinite(out[0, :4]).all() and np.isfinite(out[1]).all()


def test_decode_replay(lava):
    """A captured step on changing row counts, two graphs over one workspace, eager calls in between."""
    say("paged decode: graph replays")
    c = Decode(lava, 8, 2, 128, "bf16", 16, [[900, 3000], [10, 2000]], 12)
    full = c.rows.copy()
    call = lambda: lava.lava_paged_decode(c.desc, c.dev["q"], c.pool, c.dev["table"], c.dev["rows"], out=c.out, lse=c.lse, workspace=c.ws[: c.need])
    call()
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for g in graphs:
        with torch.cuda.graph(g):
            call()
    f = lambda x: synth.load_f64(x, "bf16")
    rng = np.random.default_rng(1)
    for i in range(8):
        c.rows = (full * rng.random(full.shape)).astype(np.int32) if i else full
        c.dev["rows"].copy_(dev(c.rows))
        want, want_lse, tol, _ = P.paged_decode(f(c.q), np.nan_to_num(f(c.k)), np.nan_to_num(f(c.v)), c.table, c.rows, c.scale)
        for run in (graphs[i % 2].replay, call, graphs[1 - i % 2].replay):
            c.out.fill_(777.0)
            run()
            torch.cuda.synchronize()
            assert (np.abs(host(c.out.double()) - want) <= tol).all()


def test_decode_on_another_stream(lava):
    say("paged decode: side stream")
    c = Decode(lava, 8, 2, 64, "bf16", 16, [[900, 300]], 13)
    first = c.check()
    side = torch.cuda.Stream()
    c.out.fill_(777.0)
    torch.cuda.synchronize()
    lava.lava_paged_decode(c.desc, c.dev["q"], c.pool, c.dev["table"], c.dev["rows"], out=c.out, lse=c.lse, workspace=c.ws[: c.need], stream=side)
    side.synchronize()
    assert np.array_equal(host(c.out.double()), first)


# ------------------------------------------------------------------------------------------- all of it
@pytest.mark.parametrize("dtype,page", [("bf16", 16), ("f32", 32)])
def test_serving_loop(lava, dtype, page):
    """Two prompts are evicted into pages; six decode steps; one sequence leaves and another prompt takes its place; more steps.
    Every step's attention against the oracle over the rows that each head should hold."""
    say(f"serving loop {dtype} page {page}")
    H, Hkv, d, w, budget = 8, 2, 64, 8, 120
    desc = lava.LayerDesc.make(H, Hkv, d, w, dtype)
    n_pages, mb, batch = 64, 12, 2
    st = lava.PageState.empty(batch, Hkv, mb, n_pages, page)
    dt = desc.torch_dtype
    pool = lava.PagePool(torch.full((n_pages, page, d), math.nan, dtype=dt, device=DEV), torch.full((n_pages, page, d), math.nan, dtype=dt, device=DEV),
                         torch.full((n_pages, page), 1 << 29, dtype=torch.int32, device=DEV), max_blocks=mb)
    rot = lava.RotaryDesc.make(d, base=500000.0, factor=8.0, original_context=8192)
    f = P.rotary_frequencies(d, 500000.0, 8.0, 8192)
    turns = lava.lava_rotary_turns(rot, DEV)
    rng = np.random.default_rng(21)
    holds = [[None] * Hkv for _ in range(batch)]                     # (k, v, pos) of every head as stored
    seen = [0] * batch
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)

    def admit(prompts, release):
        outs, counts, new = {}, torch.zeros(batch, Hkv, dtype=torch.int32, device=DEV), [0] * batch
        for b, n in prompts.items():
            sh = synth.config(1, n=n, budget=budget, n_q_heads=H, n_kv_heads=Hkv, head_dim=d, window=w, dtype=dtype)
            inp = synth.gen_layer(sh, 100 + n)
            kd, vd = lava.to_device(inp.k, dtype), lava.to_device(inp.v, dtype)
            outs[b] = (lava.evict_layer(desc, n, lava.to_device(inp.q_win, dtype), kd, vd, budget), kd, vd, inp, n)
            counts[b], new[b] = outs[b][0]["head_counts"], n
        lava.lava_page_tables(st, i32(*new), head_counts=counts, release=i32(*release))
        lava.lava_compact_paged(desc, [lava.paged_compact_problem(desc, n, kd, vd, o["head_offsets"], o["kept_idx"], budget, st.block_table[b])
                                       for b, (o, kd, vd, inp, n) in outs.items()], pool)
        torch.cuda.synchronize()
        for b, (o, kd, vd, inp, n) in outs.items():
            offs, idx = host(o["head_offsets"]), host(o["kept_idx"])
            seen[b] = n
            for g in range(Hkv):
                rows = idx[offs[g]: offs[g + 1]]
                holds[b][g] = [inp.k[g][rows], inp.v[g][rows], rows.astype(np.int64)]
        # what was just packed, read by both decode steps
        q = lava.to_device(stored(rng, (1, H, d), dtype), dtype)
        for b, (o, *_rest) in outs.items():
            a, _ = lava.lava_decode_attention(desc, 1, q, o["k_hat"], o["v_hat"], o["head_offsets"].view(1, -1).contiguous(), budget)
            p, _ = lava.lava_paged_decode(desc, q, lava.PagePool(pool.k, pool.v, pool.pos, max_blocks=mb), st.block_table[b: b + 1],
                                          st.head_rows[b: b + 1])
            torch.cuda.synchronize()
            scale = float(a.abs().max())
            assert float((a - p).abs().max()) <= 1e-5 * scale        # two orders of summation in 32 bits

    slots, positions = torch.zeros(batch + 1, Hkv, dtype=torch.int64, device=DEV), torch.zeros(batch + 1, dtype=torch.int32, device=DEV)
    x = torch.zeros(batch + 1, H + 2 * Hkv, d, dtype=dt, device=DEV)
    ws = torch.empty(lava.lava_paged_decode_workspace_bytes(desc), dtype=torch.uint8, device=DEV)
    q_out = torch.zeros(batch + 1, H, d, dtype=dt, device=DEV)
    out, lse = torch.zeros(batch, H, d, device=DEV), torch.zeros(batch, H, device=DEV)
    new, release = i32(1, 1), i32(0, 0)
    tws = torch.empty(lava.lava_page_tables_workspace_bytes(batch, Hkv), dtype=torch.uint8, device=DEV)

    def step():
        lava.lava_page_tables(st, new, release=release, slots=slots, positions=positions, workspace=tws)
        lava.lava_rotary_append(desc, rot, turns, positions, x[:, :H], x[:, H: H + Hkv], x[:, H + Hkv:], pool, slots, q_out=q_out)
        lava.lava_paged_decode(desc, q_out[:batch], pool, st.block_table, st.head_rows, out=out, lse=lse, workspace=ws)

    def decode(steps, run):
        for _ in range(steps):
            xs = stored(rng, (batch + 1, H + 2 * Hkv, d), dtype)
            x.copy_(lava.to_device(xs, dtype))
            run()
            torch.cuda.synchronize()
            assert int(st.error[0]) == 0
            got_k, got_q = lava.to_host_bits(pool.k).reshape(-1, d), lava.to_host_bits(q_out)
            table = host(slots)
            kp, vp = np.zeros((batch * Hkv, 512, d)), np.zeros((batch * Hkv, 512, d))
            for b in range(batch):
                x64 = synth.load_f64(xs[b: b + 1], dtype)
                want = P.rotary(x64, [seen[b]], f)
                tol = rotary_tolerance(x64, 1.0, f, [seen[b]], False, dtype, want)[0]
                assert (np.abs(synth.load_f64(got_q[b], dtype) - want[0, :H]) <= tol[:H]).all()
                for g in range(Hkv):
                    row = got_k[table[b, g]]                         # the key as it was stored: what later steps attend to
                    assert (np.abs(synth.load_f64(row, dtype) - want[0, H + g]) <= tol[H + g]).all()
                    h = holds[b][g]
                    h[0], h[1] = np.concatenate([h[0], row[None]]), np.concatenate([h[1], xs[b, H + Hkv + g][None]])
                    h[2] = np.append(h[2], seen[b])
                    n = len(h[2])
                    assert int(st.head_rows[b, g]) == n
                    kp[b * Hkv + g, :n], vp[b * Hkv + g, :n] = synth.load_f64(h[0], dtype), synth.load_f64(h[1], dtype)
                seen[b] += 1
            rows = np.array([[len(h[2]) for h in hb] for hb in holds], np.int32)
            ref, _, tol, _ = P.paged_decode(synth.load_f64(got_q[:batch], dtype), kp, vp, np.arange(batch * Hkv).reshape(batch, Hkv, 1), rows,
                                            1 / math.sqrt(d))
            assert (np.abs(host(out.double()) - ref) <= tol).all()

    admit({0: 300, 1: 411}, (0, 0))
    decode(3, step)
    graph = torch.cuda.CUDAGraph()
    snapshot = [t.clone() for t in (st.block_table, st.head_rows, st.seq_pos, st.free_pages, st.n_free)]
    with torch.cuda.graph(graph):
        step()
    for t, s in zip((st.block_table, st.head_rows, st.seq_pos, st.free_pages, st.n_free), snapshot):
        assert torch.equal(t, s)                                     # recording runs nothing
    decode(3, graph.replay)
    admit({1: 200}, (0, 1))                                          # sequence 1 is over, a new one takes its place
    decode(2, graph.replay)
    decode(2, step)
    pages = owned(host(st.block_table), host(st.head_rows), page) + [int(p) for p in host(st.free_pages)[: int(st.n_free[0])]]
    assert sorted(pages) == list(range(n_pages))


@pytest.mark.parametrize("H,Hkv,d,dtype,page", [(32, 8, 128, "bf16", 16), (8, 8, 64, "bf16", 32), (40, 8, 128, "f32", 16)])
@pytest.mark.parametrize("kw", [{}, dict(softcap=20.0, window=60, bias=True)])
def test_decode_many_short_heads(lava, H, Hkv, d, dtype, page, kw):
    """More short heads than the device holds wavefronts, some of them empty, a few of many tiles."""
    say(f"paged decode: short heads H{H}/{Hkv} d{d} {dtype} {kw}")
    rng = np.random.default_rng(H)
    rows = rng.integers(0, 70, (430, Hkv))
    rows[rng.random(rows.shape) < 0.03] = 0
    rows[rng.random(rows.shape) < 0.01] = 500
    c = Decode(lava, H, Hkv, d, dtype, page, rows, H + 3)
    first = c.check(**kw)
    assert np.array_equal(c.run(**kw)[0], first)


def test_decode_split_over_every_workgroup(lava):
    """One head alone: as many parts as its length allows, merged in order."""
    for H, rows, page in ((8, 70000, 128), (1, 33000, 16), (3, 5, 16)):
        say(f"paged decode: one head of {rows} rows, {H} query heads")
        c = Decode(lava, H, 1, 128, "bf16", page, [[rows]], H)
        first = c.check()
        assert np.array_equal(c.run()[0], first)


# ------------------------------------------------------------------------------------------- the ends of the ranges
def test_tables_of_many_heads(lava):
    """More heads than one chunk of sums per thread covers, one of them the last to change."""
    say("tables: 320 thousand heads")
    rng = np.random.default_rng(31)
    batch, heads, page, mb = 40000, 8, 16, 2
    n_pages = batch * heads + 100
    rows = rng.integers(0, 17, (batch, heads)).astype(np.int32)
    nb = -(-rows // page)
    order = rng.permutation(n_pages).astype(np.int32)
    table = np.full((batch, heads, mb), -7, np.int32)
    table[..., 0][nb > 0] = order[: int(nb.sum())]
    free = np.full(n_pages, -9, np.int32)
    n_free = n_pages - int(nb.sum())
    free[:n_free] = order[n_pages - n_free:]
    pos = rng.integers(0, 50, batch).astype(np.int32)
    new = (rng.random(batch) < 0.02).astype(np.int32)
    new[-1] = 3
    release = (rng.random(batch) < 0.3).astype(np.int32)
    tokens = int(new.sum()) + 1
    t = Tables(lava, page, table, rows, pos, free, n_free)
    check_step(t.step(new, None, release, tokens), P.page_tables(page, n_pages, table, rows, pos, free, n_free, new, None, release, tokens))


@pytest.mark.parametrize("batch,heads,per", [(6, 4, 3), (3, 8, 9000)])
def test_tables_one_map_alone(lava, batch, heads, per):
    """Slots without positions, positions without slots."""
    say(f"tables: one map alone, {per} tokens")
    rng = np.random.default_rng(32)
    page, mb = 64, 200
    n_pages = batch * heads * mb
    table, rows, pos, free, n_free = random_state(rng, batch, heads, mb, page, n_pages, 0.1)
    new = np.full(batch, per)
    tokens = int(new.sum()) + 2
    want = P.page_tables(page, n_pages, table, rows, pos, free, n_free, new, None, None, tokens)
    for which in ("slots", "positions"):
        t = Tables(lava, page, table, rows, pos, free, n_free)
        out = torch.full((tokens, heads), 7, dtype=torch.int64, device=DEV) if which == "slots" else torch.full((tokens,), 7, dtype=torch.int32, device=DEV)
        lava.lava_page_tables(t.state, dev(new.astype(np.int32)), **{which: out})
        torch.cuda.synchronize()
        assert np.array_equal(host(out), want[5 if which == "slots" else 6])
        assert np.array_equal(host(t.view("rows_out")), want[1]) and int(t.view("n_free_out")[0]) == want[4]


def test_pool_beyond_four_gib(lava):
    """Pages whose bytes lie beyond 2^32 of the pool's start: appended to, gathered into, attended to."""
    say("a pool of 2 x 6.5 GB")
    H, Hkv, d, page = 8, 2, 128, 256
    n_pages = 100_000
    desc = lava.LayerDesc.make(H, Hkv, d, 1, "bf16")
    k, v = (torch.empty(n_pages, page, d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    pos = torch.empty(n_pages, page, dtype=torch.int32, device=DEV)
    pool = lava.PagePool(k, v, pos, max_blocks=3)
    table = torch.tensor([[[99_999, 70_001, 5], [99_998, 80_000, 3]]], dtype=torch.int32, device=DEV)
    rng = np.random.default_rng(41)
    n, kept = 700, 520                                               # per head: two pages and eight rows
    src = [stored(rng, (Hkv, n, d), "bf16") for _ in range(2)]
    idx = np.concatenate([np.sort(rng.permutation(n)[:kept]) for _ in range(Hkv)]).astype(np.int32)
    offs = dev(np.arange(Hkv + 1, dtype=np.int64) * kept)
    sd = [lava.to_device(x, "bf16") for x in src]
    lava.lava_compact_paged(desc, [lava.paged_compact_problem(desc, n, sd[0], sd[1], offs, dev(idx), kept * Hkv, table[0])], pool)
    slots = torch.tensor([[5 * page + 8, 3 * page + 8], [99_999 * page + 7, 99_998 * page + 9]], device=DEV)
    x = stored(rng, (2, H + 2 * Hkv, d), "bf16")
    xd = lava.to_device(x, "bf16")
    rot = lava.RotaryDesc.make(d)
    lava.lava_rotary_append(desc, rot, lava.lava_rotary_turns(rot, DEV), torch.zeros(2, dtype=torch.int32, device=DEV), xd[:, :H],
                            xd[:, H: H + Hkv], xd[:, H + Hkv:], pool, slots)             # position 0: unturned
    torch.cuda.synchronize()
    rows = [[synth.load_f64(s[g][idx[g * kept: (g + 1) * kept]], "bf16") for g in range(Hkv)] for s in src]
    x64 = synth.load_f64(x, "bf16")
    for g in range(Hkv):
        for which, part in ((0, H + g), (1, H + Hkv + g)):
            r = rows[which][g]
            r[7 if g == 0 else 9] = x64[1, part]
            rows[which][g] = np.concatenate([r, x64[:1, part]])
    q = stored(rng, (1, H, d), "bf16")
    out, _ = lava.lava_paged_decode(desc, lava.to_device(q, "bf16"), pool, table, torch.full((1, Hkv), kept + 1, dtype=torch.int32, device=DEV))
    kp, vp = (np.zeros((Hkv, 768, d)) for _ in range(2))
    for g in range(Hkv):
        kp[g, : kept + 1], vp[g, : kept + 1] = rows[0][g], rows[1][g]
    want, _, tol, _ = P.paged_decode(synth.load_f64(q, "bf16"), kp, vp, np.arange(Hkv).reshape(1, Hkv, 1), np.full((1, Hkv), kept + 1), 1 / math.sqrt(d))
    torch.cuda.synchronize()
    assert (np.abs(host(out.double()) - want) <= tol).all()


def test_first_call_of_a_kernel_inside_a_capture(lava):
    """A kernel whose first launch of the process is recorded: its grid is found without disturbing the capture."""
    say("paged decode: first use inside a capture")
    c = Decode(lava, 2, 2, 128, "f32", 16, [[70, 5]], 51)
    options = lava.DecodeOptions.make(softcap=7.0)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        lava.lava_paged_decode(c.desc, c.dev["q"], c.pool, c.dev["table"], c.dev["rows"], options, out=c.out, lse=c.lse, workspace=c.ws[: c.need])
    for _ in range(3):
        c.out.fill_(777.0)
        graph.replay()
        torch.cuda.synchronize()
        got = host(c.out.double())
    assert np.array_equal(got, c.check(softcap=7.0))


def test_two_calls_at_once(lava):
    """Two streams, each with its own workspace, over one pool."""
    say("paged decode: two streams")
    cs = [Decode(lava, 8, 2, 128, "bf16", 32, [[3000, 200], [40, 900]], 60 + i) for i in range(2)]
    want = [c.check() for c in cs]
    streams = [torch.cuda.Stream() for _ in cs]
    for _ in range(5):
        for c in cs:
            c.out.fill_(777.0)
        torch.cuda.synchronize()
        for c, s in zip(cs, streams):
            lava.lava_paged_decode(c.desc, c.dev["q"], c.pool, c.dev["table"], c.dev["rows"], out=c.out, lse=c.lse, workspace=c.ws[: c.need], stream=s)
        torch.cuda.synchronize()
        for c, w in zip(cs, want):
            assert np.array_equal(host(c.out.double()), w)


def test_tensors_on_another_device(lava, monkeypatch):
    """The binding launches on the current device only."""
    c = Decode(lava, 2, 2, 64, "bf16", 16, [[5, 5]], 70)
    monkeypatch.setattr(lava, "_device_index", lambda: 1)
    with pytest.raises(ValueError):
        lava.lava_paged_decode(c.desc, c.dev["q"], c.pool, c.dev["table"], c.dev["rows"])
    with pytest.raises(ValueError):
        lava.lava_rotary(lava.RotaryDesc.make(64), torch.zeros(32, dtype=torch.int64, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV),
                         torch.zeros(1, 2, 64, device=DEV))
    with pytest.raises(ValueError):
        lava.lava_page_tables(lava.PageState.empty(1, 1, 1, 1, 16))


def test_binding_refuses_shapes(lava):
    z = lambda *s, dt=torch.float32: torch.zeros(*s, dtype=dt, device=DEV)
    i32 = torch.int32
    desc = lava.LayerDesc.make(4, 2, 64, 1, "f32")
    pool = lava.PagePool(z(4, 16, 64), z(4, 16, 64), max_blocks=2)
    bad = [lambda: lava.PagePool(z(4, 16, 64), z(4, 16, 32)), lambda: lava.PagePool(z(4, 16, 64), z(4, 16, 64), z(4, 15, dt=i32)),
           lambda: lava.lava_paged_decode(desc, z(1, 4, 64), pool, z(1, 2, 3, dt=i32), z(1, 2, dt=i32)),
           lambda: lava.lava_paged_decode(desc, z(1, 4, 64), pool, z(1, 2, 2, dt=i32), z(1, 3, dt=i32)),
           lambda: lava.lava_paged_decode(desc, z(1, 4, 64), pool, z(1, 2, 2, dt=i32), z(1, 2, dt=i32), q_pos=z(2, dt=i32)),
           lambda: lava.lava_paged_decode(desc, z(1, 4, 64), pool, z(1, 2, 2, dt=i32), z(1, 2, dt=i32), lava.DecodeOptions.make(slopes=z(3))),
           lambda: lava.lava_paged_decode(desc, z(1, 4, 64), pool, z(1, 2, 2, dt=i32), z(1, 2, dt=i32), out=z(1, 4, 32)),
           lambda: lava.lava_paged_decode(lava.LayerDesc.make(4, 2, 64, 1, "bf16"), z(1, 4, 64).bfloat16(), pool, z(1, 2, 2, dt=i32), z(1, 2, dt=i32)),
           lambda: lava.lava_rotary(lava.RotaryDesc.make(64), z(32, dt=torch.int64), z(3, dt=i32), z(2, 2, 64)),
           lambda: lava.lava_rotary(lava.RotaryDesc.make(64), z(31, dt=torch.int64), z(2, dt=i32), z(2, 2, 64)),
           lambda: lava.lava_rotary(lava.RotaryDesc.make(64), z(32, dt=torch.int64), z(2, dt=i32), z(2, 2, 64), out=z(2, 3, 64)),
           lambda: lava.lava_rotary(lava.RotaryDesc.make(64), z(32, dt=torch.int64), z(2, dt=i32), z(2, 2, 128)[..., ::2]),
           lambda: lava.lava_rotary(lava.RotaryDesc.make(64), z(32, dt=torch.int64), z(2, dt=i32), z(2, 2, 64).half()),
           lambda: lava.lava_rotary_append(desc, lava.RotaryDesc.make(64), z(32, dt=torch.int64), z(1, dt=i32), z(1, 4, 64), z(1, 3, 64), z(1, 2, 64), pool, z(1, 2, dt=torch.int64)),
           lambda: lava.lava_rotary_append(desc, lava.RotaryDesc.make(64), z(32, dt=torch.int64), z(1, dt=i32), z(1, 4, 64), z(1, 2, 64), z(1, 2, 64), pool, z(1, 3, dt=torch.int64)),
           lambda: lava.lava_page_tables(lava.PageState.empty(2, 2, 1, 4, 16), z(3, dt=i32)),
           lambda: lava.lava_page_tables(lava.PageState.empty(2, 2, 1, 4, 16), z(2, dt=i32), slots=z(3, dt=torch.int64)),
           lambda: lava.lava_page_tables(lava.PageState.empty(2, 2, 1, 4, 16), z(2, dt=i32), slots=z(2, 2, dt=torch.int64), positions=z(3, dt=i32)),
           lambda: lava.paged_compact_problem(desc, 10, z(2, 10, 64), z(2, 10, 64), z(3, dt=torch.int64), z(4, dt=i32), 5, z(2, 2, dt=i32)),
           lambda: lava.paged_compact_problem(desc, 11, z(2, 10, 64), z(2, 10, 64), z(3, dt=torch.int64), z(4, dt=i32), 4, z(2, 2, dt=i32))]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            say("not refused:", i)


def test_decode_without_rows_and_without_lse(lava):
    """Nothing held at all; a softmax scale of the caller's; no log-sum-exp asked for."""
    say("paged decode: empty batch, scale, no lse")
    import ctypes
    c = Decode(lava, 4, 2, 64, "bf16", 16, [[0, 0], [0, 0]], 80)
    out = c.check()
    assert (out == 0).all()
    c = Decode(lava, 4, 2, 128, "f32", 16, [[50, 3], [0, 900]], 81, scale=0.031)
    first = c.check()
    c.out.fill_(777.0)
    assert lava.lib.lava_paged_decode(ctypes.byref(c.desc), 2, c.dev["q"].data_ptr(), ctypes.byref(c.pool.c), c.dev["table"].data_ptr(),
                                      c.dev["rows"].data_ptr(), None, None, c.out.data_ptr(), None, c.ws.data_ptr(), c.need, None) == lava.LAVA_OK
    torch.cuda.synchronize()
    assert np.array_equal(host(c.out.double()), first)


@pytest.mark.parametrize("window", [0, 40])
def test_bad_tables_among_many_short_heads(lava, window):
    """Heads that wavefronts handle alone: impossible row counts and pages that are none give NaN for those heads only."""
    say(f"paged decode: bad tables among short heads, window {window}")
    rng = np.random.default_rng(82)
    rows = rng.integers(1, 60, (400, 8))
    c = Decode(lava, 8, 8, 64, "bf16", 16, rows, 82)
    c.rows[7, 3], c.rows[399, 7] = -4, c.table.shape[2] * 16 + 1
    c.table[100, 0, 0], c.table[0, 0, 0], c.table[200, 5, (c.rows[200, 5] - 1) // 16] = -1, c.k.shape[0], 1 << 30
    c.dev["rows"].copy_(dev(c.rows)), c.dev["table"].copy_(dev(c.table))
    out = c.check(window=window)
    bad = np.zeros((400, 8), bool)
    for at in ((7, 3), (399, 7), (100, 0), (0, 0), (200, 5)):
        bad[at] = True
    assert np.array_equal(np.isnan(out).all(-1), bad)


def test_rotary_of_more_tokens_than_a_launch_counts(lava):
    """Eight million tokens and five."""
    say("rotary: 2^23 + 5 tokens")
    tokens, d = (1 << 23) + 5, 64
    desc = lava.RotaryDesc.make(d)
    turns = lava.lava_rotary_turns(desc, DEV)
    x = torch.randn(tokens, 1, d, device=DEV).bfloat16()
    pos = torch.randint(0, 1 << 20, (tokens,), dtype=torch.int32, device=DEV)
    out = lava.lava_rotary(desc, turns, pos, x)
    at = torch.cat([torch.arange(3), torch.arange((1 << 23) - 3, tokens)]).to(DEV)
    few = lava.lava_rotary(desc, turns, pos[at].contiguous(), x[at].contiguous())
    torch.cuda.synchronize()
    assert torch.equal(out[at], few)
    assert not bool((out == 0).all(-1).any())


def test_buffers_off_their_lines(lava):
    """The same step through tables whose buffers start four bytes off a line: nothing assumes more than its type's alignment."""
    say("tables and decode: buffers off their lines")
    off = lambda t: torch.cat([torch.zeros(1, dtype=t.dtype, device=DEV), t.reshape(-1)])[1:].view(t.shape)
    rng = np.random.default_rng(83)
    page, batch, heads, mb, n_pages = 16, 6, 3, 7, 200
    table, rows, pos, free, n_free = random_state(rng, batch, heads, mb, page, n_pages, 0.4)
    st = lava.PageState(*(off(dev(a)) for a in (table, rows, pos, free, np.array([n_free], np.int32))), page)
    new = np.minimum(rng.integers(0, 4, batch), mb * page - rows.max(1)).astype(np.int32)
    tokens = int(new.sum()) + 1
    slots, positions = off(torch.zeros(tokens, heads, dtype=torch.int64, device=DEV)), off(torch.zeros(tokens, dtype=torch.int32, device=DEV))
    lava.lava_page_tables(st, off(dev(new)), slots=slots, positions=positions)
    torch.cuda.synchronize()
    want = P.page_tables(page, n_pages, table, rows, pos, free, n_free, new, max_tokens=tokens)
    assert np.array_equal(host(st.block_table), want[0]) and np.array_equal(host(slots), want[5]) and np.array_equal(host(positions), want[6])
    c = Decode(lava, 6, 2, 64, "f32", 16, [[90, 30], [5, 700]], 84)
    first = c.check(window=50, bias=True)
    for name in ("table", "rows", "slopes", "q_pos"):
        c.dev[name] = off(c.dev[name])
    c.out, c.lse = off(c.out), off(c.lse)
    assert np.array_equal(c.run(window=50, bias=True)[0], first)
