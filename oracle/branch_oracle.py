"""CPU oracle of what many continuations of one prompt need over the paged cache: a beam step, sequences that become copies of others or
lose rows, written from their definitions in plain loops and 64 bits.  (Attention over shared pages is attention over pages:
paged_oracle.paged_decode.)  Shares no code with the library."""
from __future__ import annotations

import math

import numpy as np

EXHAUSTED, INVALID = 1, 4


def beam_step(logits, scores, n_out, done=None, end_token=-1, pad_token=0):
    """logits [batch, beams, V], scores [batch, beams].  Returns (parents, tokens, scores, done, gap): gap [batch], the least distance between two
    of the best n_out + 1 candidates that are not of one beam with equal logits (nearer than rounding: their order says nothing)."""
    batch, beams, V = logits.shape
    parents, tokens = np.full((batch, n_out), -1, np.int32), np.full((batch, n_out), -1, np.int32)
    out, over = np.full((batch, n_out), -np.inf), np.ones((batch, n_out), np.int32)
    gap = np.full(batch, np.inf)
    for b in range(batch):
        found = []                                                    # (score, beam, logit, token)
        for i in range(beams):
            s = float(scores[b, i])
            if not math.isfinite(s):
                continue
            if done is not None and done[b, i] != 0:
                found.append((s, i, 0.0, pad_token))
                continue
            x = logits[b, i].astype(np.float64)
            m = x.max() if not np.isnan(x).any() else np.nan
            if not math.isfinite(m):
                continue
            lse = m + math.log(np.exp(x - m).sum())
            best = np.argsort(-x, kind="stable")[: n_out + 1]
            found += [(s + (x[v] - lse), i, x[v], int(v)) for v in best if x[v] > -np.inf]
        found.sort(key=lambda f: (-f[0], f[1], -f[2], f[3]))
        for j, (c, i, x, v) in enumerate(found[:n_out]):
            parents[b, j], tokens[b, j], out[b, j] = b * beams + i, v, c
            over[b, j] = 1 if v == end_token or (done is not None and done[b, i] != 0) else 0
        for f, g in zip(found, found[1: n_out + 1]):
            if (f[1], f[2]) != (g[1], g[2]):
                gap[b] = min(gap[b], f[0] - g[0])
    return parents, tokens, out, over, gap


def page_change(page_rows, n_pages, block_table, head_rows, seq_pos, free_pages, n_free, source=None, head_counts=None, kept_idx=None, evict=None,
                block_table_out=None, free_pages_out=None):
    """Sequence b becomes sequence source[b] (None: itself), or what head_counts and kept_idx [batch, capacity] keep of it.  Returns (block_table,
    head_rows, seq_pos, free_pages, n_free, moves, error): moves are (slot written, slot read)."""
    batch, heads, width = block_table.shape
    P = page_rows
    blocks = lambda r: -(-r // P)
    in_place_table = block_table if block_table_out is None else block_table_out
    in_place_free = free_pages if free_pages_out is None else free_pages_out
    table, free = in_place_table.copy(), in_place_free.copy()
    src = list(range(batch)) if source is None else [int(x) for x in source]
    error, top = 0, int(n_free)
    if top < 0 or top > n_pages:
        error |= INVALID
    for b in range(batch):
        if src[b] < -1 or src[b] >= batch:
            error |= INVALID
        for g in range(heads):
            n = int(head_rows[b, g])
            if n < 0 or n > width * P:
                error |= INVALID
            elif any(p < 0 or p >= n_pages for p in block_table[b, g, : blocks(n)]):
                error |= INVALID
        if head_counts is not None and (evict is None or evict[b] != 0):
            counts = [int(x) for x in head_counts[b]]
            if any(c < 0 or c > int(head_rows[b, g]) for g, c in enumerate(counts)) or sum(counts) > kept_idx.shape[1]:
                error |= INVALID
    fresh, plan = 0, []
    for b in range(batch if not error else 0):
        s = src[b]
        first = s >= 0 and (b == s if src[s] == s else b == src.index(s))
        begin = 0
        for g in range(heads):
            old = int(head_rows[s, g]) if s >= 0 else 0
            rows = list(range(old))
            if head_counts is not None and (evict is None or evict[b] != 0):
                n = int(head_counts[b, g])
                rows = [int(x) for x in kept_idx[b, begin: begin + n]]
                begin += n
            n, same = len(rows), 0
            while same < n and rows[same] == same:
                same += 1
            stay = same // P
            if n % P and same == n and old % P and n // P == old // P and first:
                stay += 1                                             # the last page, by whom it is held alone
            plan.append((b, g, s, n, stay, rows))
            fresh += blocks(n) - stay
    if not error and fresh > top:
        error |= EXHAUSTED
    if not error and any(p < 0 or p >= n_pages for p in free_pages[top - fresh: top]):
        error |= INVALID
    back = []
    if not error:
        alive = {int(block_table[s, g, j]) for b, g, s, n, stay, rows in plan for j in range(stay)}
        for b in range(batch):
            for g in range(heads):
                for j in range(blocks(int(head_rows[b, g]))):
                    p = int(block_table[b, g, j])
                    if p not in alive and p not in back:
                        back.append(p)
        if top - fresh + len(back) > n_pages:
            error |= INVALID
    if error:
        for b in range(batch):
            for g in range(heads):
                nb = blocks(int(head_rows[b, g])) if 0 <= head_rows[b, g] <= width * P else 0
                table[b, g, :nb] = block_table[b, g, :nb]
        n = min(max(top, 0), n_pages)
        free[:n] = free_pages[:n]
        return table, head_rows.copy(), seq_pos.copy(), free, int(n_free), [], error
    rows_out, pos_out, moves = np.zeros_like(head_rows), np.zeros_like(seq_pos), []
    taken = 0
    for b, g, s, n, stay, rows in plan:
        for j in range(blocks(n)):
            if j < stay:
                table[b, g, j] = block_table[s, g, j]
            else:
                table[b, g, j] = free_pages[top - 1 - taken]
                taken += 1
        for t in range(stay * P, n):
            if 0 <= rows[t] < int(head_rows[s, g]):
                moves.append((int(table[b, g, t // P]) * P + t % P, int(block_table[s, g, rows[t] // P]) * P + rows[t] % P))
        rows_out[b, g] = n
        pos_out[b] = seq_pos[s] if s >= 0 else 0
    left = top - taken
    free[:left] = free_pages[:left]
    free[left: left + len(back)] = back
    return table, rows_out, pos_out, free, left + len(back), moves, 0
