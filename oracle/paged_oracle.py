"""CPU oracle of the paged cache: block tables, rotary positions, gather into pages and decode over pages, written from their
definitions in plain loops and 64 bits.  Shares no code with the library."""
from __future__ import annotations

import math

import numpy as np

EXHAUSTED, BLOCKS, INVALID, TOKENS = 1, 2, 4, 8


def page_tables(page_rows, n_pages, block_table, head_rows, seq_pos, free_pages, n_free, n_new=None, head_counts=None,
                release=None, max_tokens=0):
    """One step.  Returns (block_table, head_rows, seq_pos, free_pages, n_free, slots, positions, error), all new arrays."""
    table, free = block_table.copy(), list(int(x) for x in free_pages)
    batch, heads, max_blocks = table.shape
    new = [0] * batch if n_new is None else [int(x) for x in n_new]
    add = [[new[b]] * heads if head_counts is None else [int(x) for x in head_counts[b]] for b in range(batch)]
    over = [False] * batch if release is None else [int(x) != 0 for x in release]
    blocks = lambda r: -(-r // page_rows)
    error, back, need = 0, 0, 0
    for b in range(batch):
        pos = 0 if over[b] else int(seq_pos[b])
        if new[b] < 0 or pos < 0 or pos + new[b] >= 1 << 31:
            error |= INVALID
        for g in range(heads):
            rows = int(head_rows[b, g])
            if rows < 0 or rows > max_blocks * page_rows or add[b][g] < 0:
                error |= INVALID
                continue
            back += blocks(rows) if over[b] else 0
            old = 0 if over[b] else rows
            if old + add[b][g] > max_blocks * page_rows:
                error |= BLOCKS
                continue
            need += blocks(old + add[b][g]) - blocks(old)
    top = int(n_free)
    if top < 0 or top + back > n_pages:
        error |= INVALID
    elif need > top + back:
        error |= EXHAUSTED
    if max_tokens and sum(x for x in new if x > 0) > max_tokens:
        error |= TOKENS
    slots = np.full((max_tokens, heads), -1, np.int64)
    positions = np.full(max_tokens, -1, np.int32)
    if error:
        return table, head_rows.copy(), seq_pos.copy(), np.array(free, np.int32), int(n_free), slots, positions, error
    for b in range(batch):                                            # pages go back first
        for g in range(heads):
            for j in range(blocks(int(head_rows[b, g])) if over[b] else 0):
                free[top] = int(table[b, g, j])
                top += 1
    rows_out, pos_out = head_rows.copy(), seq_pos.copy()
    for b in range(batch):
        pos_out[b] = (0 if over[b] else int(seq_pos[b])) + new[b]
        for g in range(heads):
            old = 0 if over[b] else int(head_rows[b, g])
            for j in range(blocks(old), blocks(old + add[b][g])):
                top -= 1
                table[b, g, j] = free[top]
            rows_out[b, g] = old + add[b][g]
    if max_tokens:
        t = 0
        for b in range(batch):
            for i in range(new[b]):
                positions[t] = pos_out[b] - new[b] + i
                for g in range(heads):
                    r = rows_out[b, g] - new[b] + i
                    slots[t, g] = int(table[b, g, r // page_rows]) * page_rows + r % page_rows
                t += 1
    return table, rows_out, pos_out, np.array(free, np.int32), top, slots, positions, 0


def rotary_frequencies(rotary_dim, base=10000.0, factor=1.0, original_context=0, low_turns=1.0, high_turns=4.0):
    """Radians a token of every pair."""
    out = []
    for i in range(rotary_dim // 2):
        f = float(base) ** (-2.0 * i / rotary_dim)
        if original_context:
            c = (original_context * f / (2.0 * math.pi) - low_turns) / (high_turns - low_turns)
            c = min(1.0, max(0.0, c))
            f = c * f + (1.0 - c) * f / factor
        else:
            f /= factor
        out.append(f)
    return np.array(out)


def rotary(x, positions, freqs, interleaved=False, magnitude=1.0, transpose=False):
    """x [tokens, heads, d] in 64 bits; every pair times magnitude * e^(+-i angle)."""
    y = np.array(x, np.float64)
    half = len(freqs)
    angle = np.asarray(positions, np.float64)[:, None, None] * freqs
    w = magnitude * np.exp((-1j if transpose else 1j) * angle)
    a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    z = (y[..., a] + 1j * y[..., b]) * w
    y[..., a], y[..., b] = z.real, z.imag
    return y


def compact_paged(pages, page_rows, max_blocks, head_offsets, kept_idx, segments, block_table, first_rows=None):
    """[(slot, source row, index)] of the survivors that are written; segments: (first source row, rows) of every head."""
    moves = []
    for g in range(len(segments)):
        for t in range(int(head_offsets[g]), int(head_offsets[g + 1])):
            idx, row = int(kept_idx[t]), (0 if first_rows is None else int(first_rows[g])) + t - int(head_offsets[g])
            if idx < 0 or idx >= segments[g][1] or row < 0 or row // page_rows >= max_blocks:
                continue
            page = int(block_table[g, row // page_rows])
            if 0 <= page < pages:
                moves.append((page * page_rows + row % page_rows, segments[g][0] + idx, idx))
    return moves


def paged_decode(q, k_pages, v_pages, block_table, head_rows, scale, softcap=0.0, window=0, slopes=None, pos_pages=None,
                 q_pos=None):
    """q [batch, H, d], pages [n_pages, page_rows, d], in 64 bits.  Returns (out, lse, tol, tol_lse): the last two bound how
    far an evaluation in 32 bits may be off, from the roundings it makes (written beside them)."""
    batch, H, d = q.shape
    n_pages, P = k_pages.shape[:2]
    Hkv = head_rows.shape[1]
    G = H // Hkv
    out, lse = np.zeros((batch, H, d)), np.full((batch, H), -np.inf)
    tol, tol_lse = np.zeros((batch, H, d)), np.zeros((batch, H))
    for b in range(batch):
        for g in range(Hkv):
            n, heads = int(head_rows[b, g]), slice(g * G, (g + 1) * G)
            pages = [int(p) for p in block_table[b, g, : max(0, -(-n // P))]]
            if n < 0 or n > block_table.shape[2] * P or any(p < 0 or p >= n_pages for p in pages):
                out[b, heads], lse[b, heads] = np.nan, np.nan
                continue
            rows = [(pages[r // P], r % P) for r in range(n)]
            back = np.zeros(n)
            if pos_pages is not None and (window or slopes is not None):
                back = np.array([int(q_pos[b]) - int(pos_pages[r]) for r in rows], np.float64).reshape(n)
                seen = (back >= 0) & ((back < window) if window else True)
                rows, back = [r for r, s in zip(rows, seen) if s], back[seen]
            if not rows:
                continue
            k = np.array([k_pages[r] for r in rows])
            v = np.array([v_pages[r] for r in rows])
            z = scale * (q[b, heads] @ k.T)
            size = scale * (np.abs(q[b, heads]) @ np.abs(k).T)                 # what a rounding of a partial sum is relative to
            dz = (d + 4) * 2.0 ** -24 * size
            if softcap:
                z = softcap * np.tanh(z / softcap)
                dz = dz + softcap * 2.0 ** -20
            if slopes is not None:
                bias = np.asarray(slopes, np.float64)[heads, None] * back
                z = z - bias
                dz = dz + 3 * 2.0 ** -24 * (np.abs(bias) + np.abs(z))
            m = z.max(1, keepdims=True)
            e = np.exp(z - m)
            p = e / e.sum(1, keepdims=True)
            # a term of the softmax: error of its logit, of its scaled difference to the maximum (three roundings) and of
            # the exponential; a sum of n terms: n roundings; numerator and denominator
            rel = dz + (np.abs(z) + np.abs(m)) * 2.0 ** -22 + 2.0 ** -21
            top = (p * rel).sum(1, keepdims=True) + len(rows) * 2.0 ** -24
            out[b, heads] = p @ v
            lse[b, heads] = (m[:, 0] + np.log(e.sum(1)))
            tol[b, heads] = (p * rel) @ np.abs(v) + (top + (len(rows) + 8) * 2.0 ** -24) * (p @ np.abs(v))
            tol_lse[b, heads] = top[:, 0] + 2.0 ** -22 * (1.0 + np.abs(lse[b, heads]) + np.abs(m[:, 0]))
    return out, lse, tol, tol_lse
