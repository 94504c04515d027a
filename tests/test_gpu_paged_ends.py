"""The paged cache at the ends of what its documentation allows."""
import math

import numpy as np
import pytest

from oracle import paged_oracle as P
from paper_2509_09754_amd import synth

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


@pytest.mark.parametrize("page,rows", [(16, 2 ** 31 - 16), (64, 2 ** 31 - 64 - 129)])
def test_window_over_the_longest_head(lava, page, rows):
    """A head of as many rows as a block table can name, on pages that repeat; the few pages inside the window lie at its ends and
    anywhere between."""
    say(f"paged decode: window over {rows} rows, pages of {page}")
    rng = np.random.default_rng(page)
    H, d, n_pages, window, q_pos = 4, 64, 40, 500, 100000
    blocks = -(-rows // page)
    last = rows - (blocks - 1) * page                                  # rows of the last page
    desc = lava.LayerDesc.make(H, 1, d, 1, "bf16")
    k, v, q = (synth.store(rng.standard_normal(s, dtype=np.float32), "bf16") for s in ((n_pages, page, d), (n_pages, page, d), (1, H, d)))
    pos = np.zeros((n_pages, page), np.int32)                          # page 0, which repeats, is out of the window
    pos[1:] = rng.integers(q_pos - 2 * window, q_pos + 20, (n_pages - 1, page))
    at = np.concatenate([[0, 1, blocks - 1, blocks - 2], rng.integers(2, blocks - 2, n_pages - 5)])
    assert len(set(at.tolist())) == n_pages - 1
    table = torch.zeros(1, 1, blocks, dtype=torch.int32, device=DEV)
    table[0, 0, torch.from_numpy(at).to(DEV)] = torch.arange(1, n_pages, dtype=torch.int32, device=DEV)
    pool = lava.PagePool(lava.to_device(k, "bf16"), lava.to_device(v, "bf16"), dev(pos), max_blocks=blocks)
    out, lse = lava.lava_paged_decode(desc, lava.to_device(q, "bf16"), pool, table, dev(np.array([[rows]], np.int32)),
                                      lava.DecodeOptions.make(window=window), dev(np.array([q_pos], np.int32)))
    torch.cuda.synchronize()
    # the same rows as a short head: the special pages one after another, the last one, which may be in part, at the end
    order = [p for p in range(1, n_pages) if p != 3] + [3]
    f = lambda x: synth.load_f64(x, "bf16")
    want, want_lse, tol, tol_lse = P.paged_decode(f(q), f(k), f(v), np.array(order).reshape(1, 1, -1), np.array([[(n_pages - 2) * page + last]]),
                                                  1 / math.sqrt(d), window=window, pos_pages=pos, q_pos=[q_pos])
    assert (np.abs(out.cpu().double().numpy() - want) <= tol).all()
    assert (np.abs(lse.cpu().double().numpy() - want_lse) <= tol_lse).all()


def test_gather_refuses_tables_and_lists_of_other_sizes(lava):
    """A pool made for appending knows no table width; a problem whose table, row counts, offsets or positions have another length than
    the heads and the source is refused before anything is read."""
    say("compact into pages: sizes that do not belong together")
    z = lambda *s, dt=torch.int32: torch.zeros(*s, dtype=dt, device=DEV)
    desc = lava.LayerDesc.make(4, 2, 64, 1, "f32")
    kp = [z(8, 16, 64, dt=torch.float32) for _ in range(2)]
    kv = [torch.ones(2, 10, 64, device=DEV) for _ in range(2)]
    offs, idx = torch.tensor([0, 2, 4], device=DEV), z(4)
    make = lambda table, **kw: lava.paged_compact_problem(desc, kw.pop("n", 10), *kv, offs, idx, 4, table, **kw)
    table = torch.arange(8, dtype=torch.int32, device=DEV).view(2, 4)
    for pool in (lava.PagePool(*kp), lava.PagePool(*kp, max_blocks=3), lava.PagePool(*kp, max_blocks=5)):
        for problems in ([make(table)], (lava.PagedCompactProblem * 1)(make(table)), [make(z(2, pool.max_blocks)), make(table)]):
            with pytest.raises(lava.LavaError):
                lava.lava_compact_paged(desc, problems, pool)
    for call in (lambda: make(z(2, 4)[:, :0]), lambda: make(z(7)), lambda: make(table, first_rows=z(1)), lambda: make(table, first_rows=z(4)),
                 lambda: make(table, n=20, src_offsets=z(2, dt=torch.int64)), lambda: make(table, pos_src=z(10)),
                 lambda: make(table, n=20, src_offsets=z(3, dt=torch.int64), pos_src=z(19))):
        with pytest.raises(ValueError):
            call()
    torch.cuda.synchronize()
    assert not bool(kp[0].any()) and not bool(kp[1].any())
    lava.lava_compact_paged(desc, [make(table, first_rows=z(2), pos_src=z(20))], lava.PagePool(*kp, max_blocks=4))
    torch.cuda.synchronize()
    assert bool((kp[0].view(8, 16, 64)[[0, 4], :2] == 1).all()) and int(kp[0].sum()) == 4 * 64


def test_steps_of_nothing(lava):
    """No tokens, no survivors: tensors of no elements are accepted, nothing is written."""
    say("paged cache: empty tensors")
    desc, rot = lava.LayerDesc.make(4, 2, 64, 1, "bf16"), lava.RotaryDesc.make(64)
    turns = lava.lava_rotary_turns(rot, DEV)
    kp, vp = (torch.full((8, 16, 64), 3.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    none = lambda *s, dt=torch.bfloat16: torch.empty(*s, dtype=dt, device=DEV)
    pos, slots = none(0, dt=torch.int32), none(0, 2, dt=torch.int64)
    x = none(0, 8, 64)
    assert lava.lava_rotary(rot, turns, pos, x).shape == (0, 8, 64)
    q_out = lava.lava_rotary_append(desc, rot, turns, pos, x[:, :4], x[:, 4:6], x[:, 6:], lava.PagePool(kp, vp), slots)
    assert q_out.shape == (0, 4, 64)
    assert lava.lava_rotary_append(desc, rot, turns, pos, None, x[:, 4:6], x[:, 6:], lava.PagePool(kp, vp), slots) is None
    st = lava.PageState.empty(2, 2, 4, 8, 16)
    lava.lava_page_tables(st, torch.zeros(2, dtype=torch.int32, device=DEV), slots=slots, positions=pos)
    k = torch.ones(2, 10, 64, dtype=torch.bfloat16, device=DEV)
    table = torch.arange(8, dtype=torch.int32, device=DEV).view(2, 4)
    offs = torch.tensor([0, 1, 2], device=DEV)                         # the capacity rules
    lava.lava_compact_paged(desc, [lava.paged_compact_problem(desc, 10, k, k, offs, pos, 0, table)], lava.PagePool(kp, vp, max_blocks=4))
    torch.cuda.synchronize()
    assert bool((kp == 3.0).all()) and bool((vp == 3.0).all()) and int(st.n_free[0]) == 8 and int(st.error[0]) == 0


def test_idle_sequences_between_others(lava):
    """A captured step in which any of the sequences may see no token: slots number the tokens without gaps, and the queries are moved to
    their sequences' rows as the documentation says.  Every replay against the oracle."""
    say("paged cache: idle sequences")
    H, Hkv, d, page, batch, mb = 4, 2, 64, 16, 4, 3
    desc, rot = lava.LayerDesc.make(H, Hkv, d, 1, "f32"), lava.RotaryDesc.make(d)
    turns = lava.lava_rotary_turns(rot, DEV)
    st = lava.PageState.empty(batch, Hkv, mb, batch * Hkv * mb, page)
    kp, vp = (torch.zeros(batch * Hkv * mb, page, d, device=DEV) for _ in range(2))
    pool = lava.PagePool(kp, vp, max_blocks=mb)
    new = torch.zeros(batch, dtype=torch.int32, device=DEV)
    x = torch.zeros(batch, H + 2 * Hkv, d, device=DEV)
    slots, pos = torch.zeros(batch, Hkv, dtype=torch.int64, device=DEV), torch.zeros(batch, dtype=torch.int32, device=DEV)
    q_out, out, lse = torch.zeros(batch, H, d, device=DEV), torch.zeros(batch, H, d, device=DEV), torch.zeros(batch, H, device=DEV)
    tws, dws = (torch.zeros(n, dtype=torch.uint8, device=DEV) for n in (lava.lava_page_tables_workspace_bytes(batch, Hkv),
                                                                        lava.lava_paged_decode_workspace_bytes(desc)))

    def step():
        lava.lava_page_tables(st, new, slots=slots, positions=pos, workspace=tws)
        lava.lava_rotary_append(desc, rot, turns, pos, x[:, :H], x[:, H: H + Hkv], x[:, H + Hkv:], pool, slots, q_out=q_out)
        q = q_out.index_select(0, (new.cumsum(0) - 1).clamp(min=0))
        lava.lava_paged_decode(desc, q, pool, st.block_table, st.head_rows, out=out, lse=lse, workspace=dws)

    snapshot = [t.clone() for t in (st.block_table, st.head_rows, st.seq_pos, st.free_pages, st.n_free)]
    step()                                                           # no tokens: warms up torch's own calls
    torch.cuda.synchronize()
    for t, s in zip((st.block_table, st.head_rows, st.seq_pos, st.free_pages, st.n_free), snapshot):
        assert torch.equal(t, s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    rng = np.random.default_rng(3)
    f = P.rotary_frequencies(d)
    held = [[[] for _ in range(Hkv)] for _ in range(batch)]            # (key, value) of every head, as turned in 64 bits
    seen = [0] * batch
    patterns = [[1, 0, 1, 1], [0, 1, 0, 0], [0, 0, 0, 0], [0, 0, 0, 1], [1, 1, 1, 1], [1, 0, 0, 1], [0, 1, 1, 0]] * 3
    for i, n in enumerate(patterns):
        xs = rng.standard_normal((batch, H + 2 * Hkv, d)).astype(np.float32)
        x.copy_(dev(xs)), new.copy_(dev(np.array(n, np.int32)))
        graph.replay() if i % 4 else step()
        torch.cuda.synchronize()
        assert int(st.error[0]) == 0
        row = 0
        q64 = np.zeros((batch, H, d))
        for b in range(batch):
            if not n[b]:
                continue
            turned = P.rotary(xs[row: row + 1].astype(np.float64), [seen[b]], f)[0]
            q64[b] = turned[:H]
            for g in range(Hkv):
                held[b][g].append((turned[H + g], xs[row, H + Hkv + g].astype(np.float64)))
            seen[b] += 1
            row += 1
        rows = np.array([[len(h) for h in hb] for hb in held], np.int32)
        assert np.array_equal(st.head_rows.cpu().numpy(), rows) and st.seq_pos.cpu().tolist() == seen
        k64, v64 = (np.array([np.pad(np.array([r[j] for r in h]).reshape(len(h), d), ((0, 64 - len(h)), (0, 0))) for hb in held for h in hb])
                    for j in range(2))
        want, _, tol, _ = P.paged_decode(q64, k64, v64, np.arange(batch * Hkv).reshape(batch, Hkv, 1), rows, 1 / math.sqrt(d))
        # queries and keys are within 2^-20 of the turned values here (two products of values below 6 with 2^-22 sines, rounded): a
        # logit, of 64 products of size up to 6, over 8, within 2 * 64 * 6 * 2^-20 / 8 = 2^-13.4; twice that in a weight, times |v| < 6
        tol = tol + 2.0 ** -12.4 * 6
        busy = np.array(n, bool)
        assert (np.abs(out.cpu().double().numpy() - want)[busy] <= tol[busy]).all()
        wrong = P.paged_decode(q64[::-1], k64, v64, np.arange(batch * Hkv).reshape(batch, Hkv, 1), rows, 1 / math.sqrt(d))[0]
        assert i < 5 or not busy.any() or (np.abs(wrong - want)[busy].max() > tol[busy].max())   # another row's query would be seen


@pytest.mark.parametrize("cap", [1e-30, 1e-6, 1e30])
def test_caps_at_the_ends(lava, cap):
    """The smallest cap makes every row weigh the same, zeros among the logits included; the largest changes nothing."""
    say(f"paged decode: cap {cap}")
    rng = np.random.default_rng(4)
    desc = lava.LayerDesc.make(4, 2, 64, 1, "f32")
    k, v, q = (rng.standard_normal(s).astype(np.float32) for s in ((6, 16, 64), (6, 16, 64), (1, 4, 64)))
    q[0, 1] = 0.0
    table, rows = np.arange(6, dtype=np.int32).reshape(1, 2, 3), np.array([[40, 17]], np.int32)
    pool = lava.PagePool(dev(k), dev(v), max_blocks=3)
    out, lse = lava.lava_paged_decode(desc, dev(q), pool, dev(table), dev(rows), lava.DecodeOptions.make(softcap=cap))
    want, want_lse, tol, tol_lse = P.paged_decode(*(x.astype(np.float64) for x in (q, k, v)), table, rows, 0.125, softcap=0.0 if cap > 1 else cap)
    # near zero the cap's series is relative: z (1 + 2^-20); the oracle counts 2^-20 of the cap, which says nothing for a large one
    slack = 2.0 ** -19 * 8 * 6 if cap > 1 else 0.0                     # logits below 8, values below 6
    assert (np.abs(out.cpu().double().numpy() - want) <= tol + slack).all()
    assert (np.abs(lse.cpu().double().numpy() - want_lse) <= tol_lse + slack).all()


def test_tables_of_as_many_heads_as_there_may_be(lava):
    """2^20 heads: every chunk of the sums is full.  One token for a few sequences, a few that leave."""
    say("tables: 2^20 heads")
    rng = np.random.default_rng(61)
    batch, heads, page, mb = 16384, 64, 16, 1
    n_pages = batch * heads
    rows = rng.integers(0, 2, (batch, heads)).astype(np.int32) * rng.integers(1, 15, (batch, 1)).astype(np.int32)
    order = rng.permutation(n_pages).astype(np.int32)
    held = int((rows > 0).sum())
    table = np.full((batch, heads, mb), -7, np.int32)
    table[..., 0][rows > 0] = order[:held]
    free = np.full(n_pages, -9, np.int32)
    free[: n_pages - held] = order[held:]
    pos = rng.integers(0, 50, batch).astype(np.int32)
    new, release = (rng.random(batch) < 0.01).astype(np.int32), (rng.random(batch) < 0.02).astype(np.int32)
    new[-1] = release[-1] = 1
    tokens = int(new.sum()) + 1
    want = P.page_tables(page, n_pages, table, rows, pos, free, n_pages - held, new, None, release, tokens)
    assert want[7] == 0
    st = lava.PageState(*(dev(a) for a in (table, rows, pos, free, np.array([n_pages - held], np.int32))), page)
    slots, positions = torch.zeros(tokens, heads, dtype=torch.int64, device=DEV), torch.zeros(tokens, dtype=torch.int32, device=DEV)
    lava.lava_page_tables(st, dev(new), release=dev(release), slots=slots, positions=positions)
    torch.cuda.synchronize()
    for got, a in zip((st.block_table, st.head_rows, st.seq_pos, st.free_pages, st.n_free, slots, positions), want[:4] + (want[4:5],) + want[5:7]):
        assert np.array_equal(got.cpu().numpy(), np.asarray(a))


def test_decode_of_as_many_heads_as_there_may_be(lava):
    """65536 heads, most of them of a row or two, one long."""
    from oracle.paged_counts import SCALE, Pages
    say("paged decode: 65536 heads")
    batch, Hkv, page, d = 8192, 8, 16, 64
    rng = np.random.default_rng(62)
    rows = rng.integers(0, 40, (batch, Hkv)).astype(np.int32)
    for longest in (40, 3000):
        rows[batch // 2, 3] = rows[-1, -1] = longest
        blocks = -(-int(rows.max()) // page)
        pages = Pages(longest, 300, page, d, device=DEV)
        table = torch.randint(0, 300, (batch, Hkv, blocks), device=DEV, dtype=torch.int32)
        desc = lava.LayerDesc.make(2 * Hkv, Hkv, d, 1, "bf16", softmax_scale=SCALE)
        pool = lava.PagePool(pages.k.bfloat16(), pages.v.bfloat16(), max_blocks=blocks)
        out, lse = lava.lava_paged_decode(desc, pages.queries(batch, 2 * Hkv, 2).bfloat16(), pool, table, dev(rows))
        want, want_lse, tol, tol_lse = pages.attend(table, rows, 2)
        torch.cuda.synchronize()
        some = torch.isfinite(want_lse)
        assert bool((torch.isfinite(lse) == some).all())
        assert bool(((out.double() - want).abs() <= tol).all()) and bool(((lse.double() - want_lse).abs() <= tol_lse)[some].all())
