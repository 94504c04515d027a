"""Calls of different kinds on one cache of sequences that share pages, as a program chains them: scores and selections before a compaction of pages, beams
that become fewer before a fork."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
DEV = "cuda"


@pytest.fixture(scope="module")
def lava():
    from paper_2509_09754_amd import lava as L
    return L


def i32(x):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(x, np.int32))).to(DEV)


def best(scores, lengths, budget):
    """Of the heads' scores, one head after another, the `budget` largest (of equals the first): rows of every head, ascending."""
    order = np.sort(np.argsort(-scores, kind="stable")[:budget])
    first = np.concatenate([[0], np.cumsum(lengths)])
    return [order[(order >= first[g]) & (order < first[g + 1])] - first[g] for g in range(len(lengths))]


def read(pool_rows, table, rows, page):
    """What the heads of one sequence hold, from a pool [pages * page, ..]."""
    return [pool_rows[(table[g, np.arange(n) // page].astype(np.int64) * page + np.arange(n) % page)] for g, n in enumerate(rows)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("blocks", [9, 700], ids=["small", "wide"])   # marked by one workgroup, and by launches of their own
def test_evicted_again_by_the_scores_that_were_kept(lava, dtype, blocks):
    """Dense caches are scored, selected and go to pages; sequences are forked and grow; then the scores that the selection kept, carried along
    with the forks, select again: lava_select_topk's counts and lists are what lava_page_compact takes.  New tokens are scored with +inf: they
    stay."""
    H, Hkv, d, w, page, lens = 8, 2, 64, 8, 16, [150, 97, 230]
    batch, heads, n_pages = 6, Hkv, 200
    rng = np.random.default_rng(71)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    desc = lava.LayerDesc.make(H, Hkv, d, w, dtype)
    val = lambda *s: torch.from_numpy(rng.normal(size=s).astype(np.float32)).to(DEV).to(dt)
    k, v = (torch.zeros(n_pages, page, d, dtype=dt, device=DEV) for _ in range(2))
    pos = torch.full((n_pages, page), -1, dtype=torch.int32, device=DEV)
    pool = lava.PagePool(k, v, pos, max_blocks=blocks)
    state = lava.PageState.empty(batch, heads, blocks, n_pages, page)
    # the prompts: sequences 0, 1, 2
    first, counts, seen = [], np.zeros((batch, heads), np.int32), np.zeros(batch, np.int32)
    for b, n in enumerate(lens):
        kd, vd = val(Hkv, n, d), val(Hkv, n, d)
        scores = lava.lava_window_scores(desc, [n], val(1, H, w, d), kd, vd)[0]
        cnt, off, idx, sc = lava.lava_select_topk(Hkv, scores, n // 2 + 30)
        first.append((n, kd, vd, off, idx, sc))
        counts[b], seen[b] = cnt.cpu().numpy(), n
    lava.lava_page_tables(state, i32(seen), head_counts=i32(counts))
    for b, (n, kd, vd, off, idx, sc) in enumerate(first):
        lava.lava_compact_paged(desc, [lava.paged_compact_problem(desc, n, kd, vd, off, idx, n // 2 + 30, state.block_table[b])], pool)
    held = [[[(int(b), int(r)) for r in np.split(first[b][4].cpu().numpy(), [counts[b, 0]])[g]] for g in range(heads)] if b < 3 else [[], []]
            for b in range(batch)]                                     # (prompt, row) of every row that a head holds
    scores = [first[b][5].clone() if b < 3 else torch.zeros(0, device=DEV) for b in range(batch)]
    # forked: the scores go with their sequences
    source = [2, 0, 2, 1, 2, 0]
    lava.lava_page_fork(desc, pool, state, i32(source))
    held, scores = [[list(x) for x in held[s]] for s in source], [scores[s].clone() for s in source]
    # and grown by a few tokens each
    new = np.array([3, 0, 17, 5, 1, 20])
    slots = torch.empty(int(new.sum()), heads, dtype=torch.int64, device=DEV)
    lava.lava_page_tables(state, i32(new), slots=slots)
    tokens = val(2, int(new.sum()), heads, d)
    for x, t in ((k, tokens[0]), (v, tokens[1])):
        x.view(-1, d)[slots.view(-1)] = t.view(-1, d)
    at = 0
    for b in range(batch):
        parts = torch.split(scores[b], [len(x) for x in held[b]])
        scores[b] = torch.cat([torch.cat([x, torch.full((int(new[b]),), float("inf"), device=DEV)]) for x in parts])
        for g in range(heads):
            held[b][g] += [(-1, at + i) for i in range(new[b])]
        at += int(new[b])
    # evicted again: every sequence but one, to budgets of their own, into rows of one list
    budgets = [60, 40, 77, 50, 61, 0]
    capacity = max(budgets) + 3
    kept, cnt = torch.full((batch, capacity), -7, dtype=torch.int32, device=DEV), torch.zeros(batch, heads, dtype=torch.int32, device=DEV)
    for b in range(batch):
        lengths = [len(x) for x in held[b]]
        offsets = torch.tensor([0, lengths[0], sum(lengths)], dtype=torch.int64, device=DEV)
        want = best(scores[b].cpu().numpy(), lengths, budgets[b])
        lava.lava_select_topk(heads, scores[b], budgets[b], offsets, head_counts=cnt[b], kept_idx=kept[b])
        held[b] = [[held[b][g][r] for r in want[g]] for g in range(heads)] if b != 1 else held[b]
    lava.lava_page_compact(desc, pool, state, cnt, kept, evict=i32([1, 0, 1, 1, 1, 1]))
    torch.cuda.synchronize()
    assert int(state.error[0]) == 0
    rows, table = state.head_rows.cpu().numpy(), state.block_table.cpu().numpy()
    assert [[len(x) for x in y] for y in held] == rows.tolist()
    for b in range(batch):
        for cells, dense, t in ((k, 1, 0), (v, 2, 1)):
            got = read(cells.view(-1, d).float().cpu().numpy(), table[b], rows[b], page)
            for g in range(heads):
                for r, (prompt, row) in enumerate(held[b][g]):
                    want = tokens[t][row, g] if prompt < 0 else first[prompt][dense].view(Hkv, -1, d)[g, row]
                    assert np.array_equal(got[g][r], want.float().cpu().numpy())
    used = {int(p) for b in range(batch) for g in range(heads) for p in table[b, g, : -(-int(rows[b, g]) // page)]}
    assert len(used) + int(state.n_free[0]) == n_pages


def test_fewer_beams_go_on(lava):
    """n_out below the number of beams: parents name rows of `beams` a group, so that their places in a state that keeps `beams` a group are the
    caller's to choose."""
    batch, beams, n_out, V, page = 2, 4, 2, 50, 16
    rng = np.random.default_rng(72)
    logits = torch.from_numpy(rng.normal(size=(batch, beams, V)).astype(np.float32)).to(DEV)
    scores = torch.from_numpy(rng.normal(size=(batch, beams)).astype(np.float32)).to(DEV)
    parents, tokens, out, done = lava.lava_beam_step(logits, scores, n_out)
    desc = lava.LayerDesc.make(1, 1, 64, 1, "bf16")
    state = lava.PageState.empty(batch * beams, 1, 3, 40, page)
    k, v = (torch.zeros(40, page, 64, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    pool = lava.PagePool(k, v, None, max_blocks=3)
    rows = i32([20 + b for b in range(batch * beams)])
    lava.lava_page_tables(state, rows)
    source = torch.full((batch, beams), -1, dtype=torch.int32, device=DEV)
    source[:, :n_out] = parents
    lava.lava_page_fork(desc, pool, state, source.view(-1))
    torch.cuda.synchronize()
    want = np.full((batch, beams), 0)
    p = parents.cpu().numpy()
    assert (p // beams == np.arange(batch)[:, None]).all()
    want[:, :n_out] = 20 + p
    assert state.head_rows.view(batch, beams).cpu().numpy().tolist() == want.tolist() and int(state.error[0]) == 0


def test_one_token(lava):
    """A vocabulary of one, whose only column may have any stride: every beam goes on at its score."""
    logits = torch.randn(2, 7, 3, device=DEV).transpose(1, 2)[:, :, :1]
    assert logits.stride(2) != 1
    logits = torch.as_strided(logits, (2, 3, 1), (3, 1, logits.stride(2)))
    scores = torch.tensor([[-1.0, -3.0, -2.0], [-5.0, -4.0, -6.0]], device=DEV)
    parents, tokens, out, done = lava.lava_beam_step(logits, scores)
    assert parents.tolist() == [[0, 2, 1], [4, 3, 5]] and not tokens.any() and out.tolist() == [[-1.0, -2.0, -3.0], [-4.0, -5.0, -6.0]]
