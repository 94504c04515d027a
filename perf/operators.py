"""The paged cache of a serving program, as calls that can be timed and compared.

Heads of an evicted cache hold different numbers of rows, so every KV head of every sequence owns pages of its own in one
pool.  Four operators keep and read such a cache, each through the entry points of `paper_2509_09754_amd.lava`:

  tables   pages for the rows a step adds, popped from the free stack; block tables, the slot of every new row, positions;
           the pages of finished sequences go back first
  rotary   rotary positions of a step's queries and keys; keys and values go to their slots (`append`), or the transposed
           rotation of a gradient into any layout (`transpose`)
  compact  the rows a selection kept, gathered from the prefill's dense caches into pages
  decode   one new token per sequence over the pages: plain, or with capped scores, a distance bias and a position window

Row counts, head counts and lengths are properties of a case (so its work is known); values, page numbers and the order of
the free stack come from the seed.  Head shapes, windows and budgets are those of the benchmark's configurations and of the
tests.
"""
import functools
import math

import torch

own = False          # whether run() makes the framework's calls or computes the plain forms

DEV = "cuda"


def _heads(hq, hkv, d, dtype):
    return dict(hq=hq, hkv=hkv, d=d, dtype=dtype)


GQA4 = _heads(32, 8, 128, "bf16")     # the benchmark's layer: 32 query heads on 8 KV heads
GQA7 = _heads(28, 4, 128, "bf16")     # a group that is not a power of two
MHA = _heads(16, 16, 64, "bf16")      # a KV head per query head
TINY = _heads(8, 2, 64, "f32")        # the smallest configuration
FULL = _heads(32, 8, 128, "f32")      # the benchmark's layer kept in 32 bits


def _decode(name, heads, batch, lo, hi, page, mix, idle=0, cap=0.0, bias=False, window=0, ctx=4):
    return dict(name=name, kind="decode", batch=batch, lo=lo, hi=hi, page=page, mix=mix, idle=idle, cap=cap, bias=bias,
                window=window, ctx=ctx, **heads)


def _rotary(name, heads, tokens, form, page=64, part=1.0, pairs=False, scaling="none"):
    return dict(name=name, kind="rotary", tokens=tokens, form=form, page=page, part=part, pairs=pairs, scaling=scaling, **heads)


def listed():
    return [
        # the tables of a decode step: 64 sequences, one token each, every 64th row needs a page; latency counts
        dict(name="tables_step64", kind="tables", batch=64, hkv=8, page=64, lo=500, hi=2000, new_lo=1, new_hi=1, mix=1,
             release=0, counts=False),
        # the prompts of 16 sequences, 4096 to 65536 tokens, admitted at once: half a million slots on 8 heads
        dict(name="tables_prompts16", kind="tables", batch=16, hkv=8, page=64, lo=0, hi=0, new_lo=4096, new_hi=65536, mix=2,
             release=0, counts=False),
        # the layers of 64 sequences as one table of 2048 rows: a quarter of the sequences leaves, survivor counts come in for the rest
        dict(name="tables_turnover", kind="tables", batch=2048, hkv=8, page=32, lo=100, hi=700, new_lo=0, new_hi=600, mix=3,
             release=4, counts=True),
        # one decode step of 64 sequences: rotate, append
        _rotary("append_step64", GQA4, 64, "append"),
        # a prefill chunk of odd length, pairs of neighbours, a long context scaled by parts
        _rotary("append_chunk8k", GQA4, 8197, "append", page=128, pairs=True, scaling="parts"),
        # gradient of the 32-bit rotation of half a head, written head by head as the prefill cache has it
        _rotary("transpose_4k_f32", FULL, 4115, "transpose", part=0.5, scaling="linear"),
        # survivors of one 32K-token layer, 512 entries a head
        dict(name="compact_32k", kind="compact", batch=1, lo=32768, hi=32768, keep=512, page=64, mix=4, **GQA4),
        # a ragged batch of 16 prompts, 1024 entries a head kept
        dict(name="compact_batch16", kind="compact", batch=16, lo=4096, hi=32768, keep=1024, page=32, mix=5, **GQA4),
        # a single user's next token over one compressed layer
        _decode("decode1", GQA4, 1, 8192, 8192, 32, 6),
        # the next token of 61 users in a padded batch of 64, ragged lengths
        _decode("decode64_ragged", GQA4, 64, 1024, 16384, 64, 7, idle=3),
        # two users whose 131072-token caches were not evicted, long pages
        _decode("decode2_131k", GQA4, 2, 8 * 131072, 8 * 131072, 128, 8, ctx=1),
        # 7 heads a group, scores capped, a distance bias and a window that leaves out the older half; pages of half a tile
        _decode("decode24_window_g7", GQA7, 24, 4096, 32768, 16, 9, cap=50.0, bias=True, window=2048, ctx=1),
    ]


def _log_int(rng, lo, hi):
    """An integer of [lo, hi], spread over its logarithm."""
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    kind = rng.choice(["tables", "rotary", "compact", "decode", "decode"])
    mix, page = rng.randrange(1 << 20), rng.choice([16, 32, 64, 128, 256])
    if kind == "tables":
        batch, hkv = _log_int(rng, 1, 1024), rng.choice([2, 4, 8])
        counts = rng.random() < 0.3
        most = max(1, min(65536, (1 << 19) // batch))
        new_hi = 1 if rng.random() < 0.3 else _log_int(rng, 1, most)
        return dict(kind="tables", batch=batch, hkv=hkv, page=page, lo=rng.choice([0, 100]), hi=_log_int(rng, 100, 4096),
                    new_lo=rng.choice([0, 1, new_hi]), new_hi=new_hi, mix=mix, release=rng.choice([0, 0, 3, 5]), counts=counts)
    heads = rng.choice([GQA4, GQA4, GQA7, MHA, TINY, FULL])
    if kind == "rotary":
        return dict(kind="rotary", tokens=_log_int(rng, 1, 8192 if heads is not FULL else 4096),
                    form=rng.choice(["append", "append", "transpose"]), page=page, part=rng.choice([1.0, 1.0, 0.5, 0.75, 0.3]),
                    pairs=rng.random() < 0.5, scaling=rng.choice(["none", "linear", "parts"]), **heads)
    size = 2 * heads["d"] * (2 if heads["dtype"] == "bf16" else 4)     # bytes of a row of both caches
    if kind == "compact":
        batch = _log_int(rng, 1, 16)
        hi = _log_int(rng, 1000, min(131072, (1 << 31) // (batch * heads["hkv"] * size)))
        lo = _log_int(rng, 1000, hi)
        return dict(kind="compact", batch=batch, lo=lo, hi=hi, keep=min(_log_int(rng, 64, 1024), lo // 2), page=page, mix=mix,
                    **heads)
    batch = _log_int(rng, 1, 64)
    hi = _log_int(rng, 64 * heads["hkv"], min(131072, (1 << 28) // (batch * size)))
    extra = rng.random() < 0.4
    return dict(kind="decode", batch=batch, lo=_log_int(rng, 32, hi), hi=hi, page=page, mix=mix,
                idle=rng.choice([0, 1]) if batch > 2 else 0, cap=rng.choice([0.0, 30.0, 50.0]) if extra else 0.0,
                bias=extra and rng.random() < 0.5, window=rng.choice([0, 256, 4096]) if extra else 0, ctx=rng.choice([1, 2, 8]),
                **heads)


# ------------------------------------------------------------------------------------------- properties of a case
class _Numbers:
    """Numbers that belong to a case, whatever the seed."""

    def __init__(self, mix):
        self.x = mix * 2654435761 + 12345

    def __call__(self, lo, hi):
        self.x = (self.x * 6364136223846793005 + 1442695040888963407) % (1 << 64)
        return lo + (self.x >> 33) % (hi - lo + 1)


def _split(total, hkv, num):
    """`total` rows over the heads as dynamic head budgets have them: uneven, every head with some."""
    w = [num(20, 100) for _ in range(hkv)]
    rows = [total * x // sum(w) for x in w]
    rows[0] += total - sum(rows)
    return rows


@functools.lru_cache(maxsize=64)
def _decode_rows(batch, lo, hi, hkv, mix, idle, even):
    """Rows of every head; the last `idle` sequences of the padded batch have none."""
    num = _Numbers(mix)
    rows = []
    for b in range(batch):
        total = num(lo, hi)
        rows.append([0] * hkv if b >= batch - idle else [total // hkv] * hkv if even else _split(total, hkv, num))
    return rows


def _rows_of(c):
    return _decode_rows(c["batch"], c["lo"], c["hi"], c["hkv"], c["mix"], c["idle"], c["lo"] == c["hi"] and c["ctx"] == 1)


def _contexts(c):
    """Tokens each sequence has seen, the newest included: `ctx` times its longest head."""
    return [max(1, c["ctx"] * max(r)) for r in _rows_of(c)]


def _visible(n, ctx, window):
    """How many of a head's n rows lie in the window; row r has position (r + 1) * ctx // n - 1."""
    if window <= 0 or window >= ctx or n == 0:
        return n
    return n - (_blocks(n * (ctx - window + 1), ctx) - 1)


@functools.lru_cache(maxsize=64)
def _table_numbers(batch, hkv, lo, hi, new_lo, new_hi, mix, release, counts):
    """(rows held per head, tokens added per sequence, rows added per head, sequences that leave)."""
    num = _Numbers(mix)
    held = [[num(lo, hi) for _ in range(hkv)] for _ in range(batch)]
    leave = [1 if release and b % release == release - 1 else 0 for b in range(batch)]
    new = [0 if leave[b] else num(new_lo, new_hi) for b in range(batch)]
    add = [[0 if leave[b] else num(new_lo, new_hi) if counts else new[b] for _ in range(hkv)] for b in range(batch)]
    return held, new, add, leave


def _tables_of(c):
    return _table_numbers(c["batch"], c["hkv"], c["lo"], c["hi"], c["new_lo"], c["new_hi"], c["mix"], c["release"], c["counts"])


@functools.lru_cache(maxsize=64)
def _compact_numbers(batch, lo, hi, keep, hkv, mix):
    """(tokens of every sequence, rows kept of every head)."""
    num = _Numbers(mix)
    ns = [num(lo, hi) for _ in range(batch)]
    kept = [[min(ns[b], r) for r in _split(keep * hkv, hkv, num)] for b in range(batch)]
    return ns, kept


def _compact_of(c):
    return _compact_numbers(c["batch"], c["lo"], c["hi"], c["keep"], c["hkv"], c["mix"])


def _blocks(rows, page):
    return -(-rows // page)


def _item(c):
    return 2 if c["dtype"] == "bf16" else 4


def _rot_dim(c):
    return int(c["d"] * c["part"]) // 2 * 2


# ------------------------------------------------------------------------------------------- inputs
def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _generator(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _ints(rows, dtype=torch.int32):
    return torch.tensor(rows, dtype=dtype, device=DEV)


def _normal(gen, *shape, dtype):
    """Standard normal values of the storage type, drawn in parts so that large ones need no second copy."""
    out = torch.empty(shape, dtype=dtype, device=DEV)
    for part in out.view(-1).split(1 << 26):
        part.copy_(torch.randn(part.shape, generator=gen, device=DEV))
    return out


def _block_table(rows, page, gen, spare, extra_blocks=0):
    """(block table with -1 behind a head's last page, pages in the pool, numbers of the unused pages) for rows [batch, hkv]."""
    nb = (rows.long() + page - 1) // page
    used = int(nb.sum())
    n_pages = used + max(1, spare)
    order = torch.randperm(n_pages, generator=gen, device=DEV).to(torch.int32)
    width = max(1, int(nb.max()) + extra_blocks)
    table = torch.full((*rows.shape, width), -1, dtype=torch.int32, device=DEV)
    table[torch.arange(width, device=DEV) < nb[..., None]] = order[:used]
    return table, n_pages, order[used:].contiguous()


def _frequencies(c):
    """Radians a position of every pair: base 500000, scaled for a context of eight times 8192 tokens."""
    rot = _rot_dim(c)
    f = 500000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=DEV) / rot)
    if c["scaling"] == "linear":
        return f / 8.0
    if c["scaling"] == "parts":     # pairs that turn more than 4 times in 8192 tokens stay, those under once are stretched
        keep = ((8192.0 * f / (2.0 * math.pi) - 1.0) / 3.0).clamp(0.0, 1.0)
        return keep * f + (1.0 - keep) * f / 8.0
    return f


def _magnitude(c):
    return 0.1 * math.log(8.0) + 1.0 if c["scaling"] == "parts" else 1.0


def _prepare_tables(c, gen):
    held, new, add, leave = _tables_of(c)
    page, batch, hkv = c["page"], c["batch"], c["hkv"]
    rows, adds = _ints(held), _ints(add)
    blocks = int(((rows.long() + adds + page - 1) // page).max())
    need = int(((rows.long() + adds + page - 1) // page - (rows.long() + page - 1) // page).sum())
    table, n_pages, unused = _block_table(rows, page, gen, need + 17)
    table = torch.nn.functional.pad(table, (0, max(0, blocks - table.shape[-1])), value=-1).contiguous()
    free = torch.full((n_pages,), -1, dtype=torch.int32, device=DEV)
    free[: unused.numel()] = unused
    tokens = 0 if c["counts"] else sum(new)
    room = 0 if c["counts"] else tokens + 5                            # a padded step
    pos = _ints([2 * max(r) for r in held])
    return dict(page=page, batch=batch, hkv=hkv, n_pages=n_pages, tokens=tokens, room=room, table=table, rows=rows, pos=pos,
                free=free, n_free=_ints([unused.numel()]), new=_ints(new), add=adds if c["counts"] else None,
                leave=_ints(leave) if c["release"] else None, rows_out=torch.empty_like(rows), pos_out=torch.empty_like(pos),
                n_free_out=torch.empty(1, dtype=torch.int32, device=DEV), error=torch.zeros(1, dtype=torch.int32, device=DEV),
                slots=torch.empty(room, hkv, dtype=torch.int64, device=DEV),
                positions=torch.empty(room, dtype=torch.int32, device=DEV), used=(n_pages - unused.numel()))


def _prepare_rotary(c, gen):
    t, hq, hkv, d, dt, page = c["tokens"], c["hq"], c["hkv"], c["d"], _dtype(c), c["page"]
    f = _frequencies(c)
    s = dict(f=f, turns=(f / (2.0 * math.pi) * 2.0 ** 64).round().to(torch.int64), magnitude=_magnitude(c), rot=_rot_dim(c))
    s["positions"] = torch.randint(0, 131072, (t,), generator=gen, device=DEV).to(torch.int32)
    if c["form"] == "transpose":
        s["x"] = _normal(gen, t, hq, d, dtype=dt)
        s["out"] = torch.empty(hq, t, d, dtype=dt, device=DEV)
        return s
    qkv = _normal(gen, t, (hq + 2 * hkv) * d, dtype=dt)                # one projection's output
    s["q"], s["k"], s["v"] = (x.view(t, -1, d) for x in qkv.split([hq * d, hkv * d, hkv * d], dim=1))
    n_pages = _blocks(t, page) * hkv + 3
    s.update(page=page, n_pages=n_pages, q_out=torch.empty(t, hq, d, dtype=dt, device=DEV))
    s["k_pages"], s["v_pages"] = (torch.zeros(n_pages, page, d, dtype=dt, device=DEV) for _ in range(2))
    s["pos_pages"] = torch.zeros(n_pages, page, dtype=torch.int32, device=DEV)
    pages = torch.randperm(n_pages, generator=gen, device=DEV)[: n_pages - 3].view(-1, hkv)
    at = torch.arange(t, device=DEV)
    s["slots"] = (pages[at // page] * page + (at % page)[:, None]).contiguous()
    return s


def _prepare_compact(c, gen):
    ns, kept = _compact_of(c)
    hkv, d, dt, page = c["hkv"], c["d"], _dtype(c), c["page"]
    rows = sum(ns) * hkv
    s = dict(k=_normal(gen, rows, d, dtype=dt), v=_normal(gen, rows, d, dtype=dt), ns=ns, page=page)
    table, n_pages, _ = _block_table(_ints(kept), page, gen, 3)
    idx = []
    for n, row in zip(ns, kept):
        for x in row:
            idx.append(torch.randperm(n, generator=gen, device=DEV)[:x].sort().values)
    s["kept_idx"] = torch.cat(idx).to(torch.int32)
    s["caps"] = [sum(row) for row in kept]
    s["offsets"] = _ints([[sum(row[:g]) for g in range(hkv + 1)] for row in kept], torch.int64)
    s["n_dev"] = _ints(ns, torch.int64)
    s.update(table=table, n_pages=n_pages, k_pages=torch.zeros(n_pages, page, d, dtype=dt, device=DEV),
             v_pages=torch.zeros(n_pages, page, d, dtype=dt, device=DEV),
             pos_pages=torch.zeros(n_pages, page, dtype=torch.int32, device=DEV))
    return s


def _prepare_decode(c, gen):
    rows_host = _rows_of(c)
    batch, hq, hkv, d, dt, page = c["batch"], c["hq"], c["hkv"], c["d"], _dtype(c), c["page"]
    rows, ctx = _ints(rows_host), _ints(_contexts(c))
    table, n_pages, _ = _block_table(rows, page, gen, 5)
    k = _normal(gen, n_pages, page, d, dtype=dt)
    v = _normal(gen, n_pages, page, d, dtype=dt)
    pos = torch.zeros(n_pages, page, dtype=torch.int32, device=DEV)
    top = max(max(r) for r in rows_host)
    r = torch.arange(table.shape[-1] * page, device=DEV)
    for b in range(batch):                                            # row r of a head: position (r + 1) * ctx // n - 1
        n = rows[b].long()[:, None]
        there = r < n
        slot = table[b].long()[:, r // page] * page + r % page
        pos.view(-1)[slot[there]] = ((r + 1) * ctx[b].long() // n.clamp(min=1) - 1)[there].to(torch.int32)
    return dict(k=k, v=v, pos=pos, table=table, rows=rows, q=_normal(gen, batch, hq, d, dtype=dt), q_pos=ctx - 1, top=top, page=page,
                n_pages=n_pages, slopes=2.0 ** (-8.0 * (1 + torch.arange(hq, device=DEV, dtype=torch.float32)) / hq),
                out=torch.empty(batch, hq, d, device=DEV), lse=torch.empty(batch, hq, device=DEV))


_PREPARE = {"tables": _prepare_tables, "rotary": _prepare_rotary, "compact": _prepare_compact, "decode": _prepare_decode}


def prepare(case, seed):
    s = _PREPARE[case["kind"]](case, _generator(seed))
    s["case"] = case
    return s


# ------------------------------------------------------------------------------------------- plain forms
def _plain_tables(s):
    page, batch, hkv, tokens, room = s["page"], s["batch"], s["hkv"], s["tokens"], s["room"]
    free, width = s["free"], s["table"].shape[-1]
    table = s["table"].view(batch * hkv, width)
    rows = s["rows"].view(-1).long()
    new = s["new"].long()
    pos = s["pos"].long()
    top = s["n_free"].long()
    if s["leave"] is not None:                                        # pages of the sequences that leave, on the stack
        leaves = s["leave"].repeat_interleave(hkv, output_size=batch * hkv) != 0
        back = torch.where(leaves, (rows + page - 1) // page, 0)
        first = back.cumsum(0) - back
        j = torch.arange(width, device=DEV)
        at = top + first[:, None] + j
        at = torch.where(j < back[:, None], at, free.numel())         # one place behind the stack for all the others
        long = torch.cat([free, free.new_zeros(1)])
        long[at.view(-1)] = table.view(-1)
        free.copy_(long[:-1])
        top = top + back.sum()
        rows = torch.where(leaves, 0, rows)
        pos = torch.where(s["leave"] != 0, 0, pos)
    add = s["add"].view(-1).long() if s["add"] is not None else new.repeat_interleave(hkv, output_size=batch * hkv)
    old = (rows + page - 1) // page
    need = (rows + add + page - 1) // page - old
    start = need.cumsum(0) - need
    j = torch.arange(width, device=DEV)
    fresh = (j >= old[:, None]) & (j < (old + need)[:, None])
    popped = (top - 1 - start + old)[:, None] - j
    table.copy_(torch.where(fresh, free[torch.where(fresh, popped, 0)], table))
    s["rows_out"].copy_((rows + add).view(batch, hkv))
    s["pos_out"].copy_(pos + new)
    s["n_free_out"].copy_(top - need.sum())
    if s["add"] is None:
        seq = torch.arange(batch, device=DEV).repeat_interleave(new, output_size=tokens)
        i = torch.arange(tokens, device=DEV) - (new.cumsum(0) - new)[seq]
        r = rows.view(batch, hkv)[seq] + i[:, None]
        pages = s["table"][seq[:, None], torch.arange(hkv, device=DEV), r // page].long()
        s["slots"][:tokens] = pages * page + r % page
        s["slots"][tokens:] = -1
        s["positions"][:tokens] = (pos[seq] + i).to(torch.int32)
        s["positions"][tokens:] = -1
    return _tables_answer(s)


def _tables_answer(s):
    out = [s["table"], s["rows_out"], s["pos_out"], s["n_free_out"], s["free"], s["error"]]
    return out + [s["slots"], s["positions"]] if s["room"] else out


def _turn(x, cos, sin, rot, pairs):
    """The rotation of the first `rot` values of x [tokens, heads, d], in 32 bits; cos and sin [tokens, 1, rot / 2]."""
    x = x.float()
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if pairs else (x[..., : rot // 2], x[..., rot // 2: rot])
    y = a * cos - b * sin, a * sin + b * cos
    y = torch.stack(y, dim=-1).flatten(-2) if pairs else torch.cat(y, dim=-1)
    return torch.cat([y, x[..., rot:]], dim=-1)


def _plain_rotary(s):
    c = s["case"]
    angle = s["positions"].double()[:, None, None] * s["f"]           # far positions need the 64 bits
    cos, sin = (angle.cos() * s["magnitude"]).float(), (angle.sin() * s["magnitude"]).float()
    if c["form"] == "transpose":
        s["out"].copy_(_turn(s["x"], cos, -sin, s["rot"], c["pairs"]).transpose(0, 1))
        return [s["out"]]
    s["q_out"].copy_(_turn(s["q"], cos, sin, s["rot"], c["pairs"]))
    at = s["slots"].view(-1)
    d = c["d"]
    s["k_pages"].view(-1, d)[at] = _turn(s["k"], cos, sin, s["rot"], c["pairs"]).to(s["k"].dtype).reshape(-1, d)
    s["v_pages"].view(-1, d)[at] = s["v"].reshape(-1, d)
    s["pos_pages"].view(-1)[at] = s["positions"].repeat_interleave(c["hkv"], output_size=at.numel())
    return [s["q_out"], s["k_pages"], s["v_pages"], s["pos_pages"]]


def _plain_compact(s):
    c, page = s["case"], s["page"]
    batch, hkv, d, total = c["batch"], c["hkv"], c["d"], s["kept_idx"].numel()
    counts = (s["offsets"][:, 1:] - s["offsets"][:, :-1]).reshape(-1)
    head = torch.arange(batch * hkv, device=DEV).repeat_interleave(counts, output_size=total)
    r = torch.arange(total, device=DEV) - (counts.cumsum(0) - counts)[head]
    n = s["n_dev"]
    base = ((n.cumsum(0) - n) * hkv)[head // hkv] + (head % hkv) * n[head // hkv]
    src = base + s["kept_idx"].long()
    slot = s["table"].view(batch * hkv, -1)[head, r // page].long() * page + r % page
    s["k_pages"].view(-1, d)[slot] = s["k"][src]
    s["v_pages"].view(-1, d)[slot] = s["v"][src]
    s["pos_pages"].view(-1)[slot] = s["kept_idx"]
    return [s["k_pages"], s["v_pages"], s["pos_pages"]]


def _plain_decode(s):
    c, page, top = s["case"], s["page"], s["top"]
    batch, hq, hkv, d = c["batch"], c["hq"], c["hkv"], c["d"]
    g = hq // hkv
    r = torch.arange(top, device=DEV)
    there = r < s["rows"].view(-1, 1)
    slot = s["table"].view(batch * hkv, -1)[:, r // page].long() * page + r % page
    slot = torch.where(there, slot, 0)
    q = s["q"].float().view(batch * hkv, g, d)
    z = torch.bmm(s["k"].view(-1, d)[slot].float(), q.transpose(1, 2).contiguous()) / math.sqrt(d)
    if c["cap"]:
        z = c["cap"] * torch.tanh(z / c["cap"])
    if c["bias"] or c["window"]:
        back = s["q_pos"].repeat_interleave(hkv, output_size=batch * hkv)[:, None] - s["pos"].view(-1)[slot]
        there = there & (back >= 0)
        if c["window"]:
            there = there & (back < c["window"])
        if c["bias"]:
            z = z - s["slopes"].view(hkv, 1, g).repeat(batch, 1, 1) * back[..., None]
    z = torch.where(there[..., None], z, -math.inf)
    m = z.amax(1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    p = torch.exp(z - m)
    total = p.sum(1)
    out = torch.bmm(p.transpose(1, 2).contiguous(), s["v"].view(-1, d)[slot].float())
    s["out"].copy_((out / torch.where(total > 0, total, 1.0)[..., None]).view(batch, hq, d))
    s["lse"].copy_((m[:, 0] + total.log()).view(batch, hq))
    return [s["out"], s["lse"]]


_PLAIN = {"tables": _plain_tables, "rotary": _plain_rotary, "compact": _plain_compact, "decode": _plain_decode}


# ------------------------------------------------------------------------------------------- the framework's calls
@functools.lru_cache(maxsize=64)
def _desc(hq, hkv, d, dtype):
    from paper_2509_09754_amd import lava
    return lava.LayerDesc.make(hq, hkv, d, 1, dtype)


def _desc_of(c):
    return _desc(c["hq"], c["hkv"], c["d"], c["dtype"])


def _handles(s):
    """What a program makes once of its buffers: the pool's description, tables of problems, workspaces."""
    from paper_2509_09754_amd import lava
    c, h = s["case"], {"lava": lava}
    if c["kind"] == "tables":
        h["state"] = lava.PageState(s["table"], s["rows"], s["pos"], s["free"], s["n_free"], page_rows=s["page"],
                                    head_rows_out=s["rows_out"], seq_pos_out=s["pos_out"], n_free_out=s["n_free_out"],
                                    error=s["error"])
        need = lava.lava_page_tables_workspace_bytes(s["batch"], s["hkv"])
        h["workspace"] = torch.empty(need, dtype=torch.uint8, device=DEV)
    elif c["kind"] == "rotary":
        h["rot"] = lava.RotaryDesc.make(s["rot"], interleaved=c["pairs"], magnitude=s["magnitude"])
        if c["form"] == "append":
            h["pool"] = lava.PagePool(s["k_pages"], s["v_pages"], s["pos_pages"])
    elif c["kind"] == "compact":
        h["pool"] = lava.PagePool(s["k_pages"], s["v_pages"], s["pos_pages"], max_blocks=s["table"].shape[-1])
        k, v, idx = (x.split(n) for x, n in ((s["k"], [n * c["hkv"] for n in s["ns"]]), (s["v"], [n * c["hkv"] for n in s["ns"]]),
                                             (s["kept_idx"], s["caps"])))
        table = [lava.paged_compact_problem(_desc_of(c), n, k[b], v[b], s["offsets"][b], idx[b], s["caps"][b], s["table"][b])
                 for b, n in enumerate(s["ns"])]
        h["problems"] = (lava.PagedCompactProblem * len(table))(*table)
        h["keep"] = (k, v, idx)
    else:
        h["pool"] = lava.PagePool(s["k"], s["v"], s["pos"], max_blocks=s["table"].shape[-1])
        h["options"] = lava.DecodeOptions.make(softcap=c["cap"], window=c["window"], slopes=s["slopes"] if c["bias"] else None)
        need = lava.lava_paged_decode_workspace_bytes(_desc_of(c))
        h["workspace"] = torch.empty(need, dtype=torch.uint8, device=DEV)
    return h


def _own(s):
    c = s["case"]
    h = s.get("handles")
    if h is None:
        h = s["handles"] = _handles(s)
    lava = h["lava"]
    if c["kind"] == "tables":
        lava.lava_page_tables(h["state"], s["new"], head_counts=s["add"], release=s["leave"],
                              slots=s["slots"] if s["room"] else None, positions=s["positions"] if s["room"] else None,
                              workspace=h["workspace"])
        return _tables_answer(s)
    if c["kind"] == "rotary" and c["form"] == "transpose":
        lava.lava_rotary(h["rot"], s["turns"], s["positions"], s["x"], out=s["out"].transpose(0, 1), transpose=True)
        return [s["out"]]
    if c["kind"] == "rotary":
        lava.lava_rotary_append(_desc_of(c), h["rot"], s["turns"], s["positions"], s["q"], s["k"], s["v"], h["pool"], s["slots"],
                                q_out=s["q_out"])
        return [s["q_out"], s["k_pages"], s["v_pages"], s["pos_pages"]]
    if c["kind"] == "compact":
        lava.lava_compact_paged(_desc_of(c), h["problems"], h["pool"])
        return [s["k_pages"], s["v_pages"], s["pos_pages"]]
    lava.lava_paged_decode(_desc_of(c), s["q"], h["pool"], s["table"], s["rows"], options=h["options"], q_pos=s["q_pos"],
                           out=s["out"], lse=s["lse"], workspace=h["workspace"])
    return [s["out"], s["lse"]]


def run(state):
    return _own(state) if own else _PLAIN[state["case"]["kind"]](state)


# ------------------------------------------------------------------------------------------- work
def work(case):
    c = case
    if c["kind"] == "tables":
        held, new, add, leave = _tables_of(c)
        page, heads = c["page"], c["batch"] * c["hkv"]
        fresh = sum(_blocks(x + a, page) - _blocks(x, page) for h, r in zip(held, add) for x, a in zip(h, r))
        back = sum(_blocks(x, page) for h, out in zip(held, leave) if out for x in h)
        n = 8 * heads + 8 * c["batch"] + 4 * c["batch"] + 8 * (fresh + back)       # row counts in and out, positions, pages in and out
        n += 4 * heads if c["counts"] else (sum(new) + 5) * (8 * c["hkv"] + 4)     # survivor counts in; slots and positions out
        return {"bytes": n, "flops": n // 4}
    if c["kind"] == "rotary":
        t, row = c["tokens"], c["d"] * _item(c)
        if c["form"] == "transpose":
            return {"bytes": 2 * t * c["hq"] * row + 4 * t, "flops": 3 * t * c["hq"] * _rot_dim(c)}
        return {"bytes": 2 * t * (c["hq"] + 2 * c["hkv"]) * row + t * (4 + 12 * c["hkv"]),
                "flops": 3 * t * (c["hq"] + c["hkv"]) * _rot_dim(c)}
    if c["kind"] == "compact":
        rows = sum(sum(r) for r in _compact_of(c)[1])
        return {"bytes": rows * (4 * c["d"] * _item(c) + 8), "flops": rows}
    seen = rows = 0
    for heads, ctx in zip(_rows_of(c), _contexts(c)):
        rows += sum(heads)
        seen += sum(_visible(n, ctx, c["window"]) for n in heads)
    n = seen * 2 * c["d"] * _item(c) + rows // c["page"] * 4 + (rows * 4 if c["bias"] or c["window"] else 0)
    n += c["batch"] * c["hq"] * (c["d"] * (_item(c) + 4) + 4)
    return {"bytes": n, "flops": seen * 4 * c["hq"] // c["hkv"] * c["d"]}


# ------------------------------------------------------------------------------------------- in 64 bits
def _exact_rotary(s):
    """Every pair as a complex number times m e^(i angle)."""
    c, rot = s["case"], s["rot"]
    unit = torch.polar(torch.full_like(s["f"], s["magnitude"]).expand(c["tokens"], -1).contiguous(),
                       s["positions"].to(torch.float64).unsqueeze(1) * s["f"].unsqueeze(0)).unsqueeze(1)

    def turned(x, unit):
        y = x.to(torch.float64).clone()
        first, second = (slice(0, rot, 2), slice(1, rot, 2)) if c["pairs"] else (slice(0, rot // 2), slice(rot // 2, rot))
        w = torch.complex(y[..., first], y[..., second]) * unit
        y[..., first], y[..., second] = w.real, w.imag
        return y

    if c["form"] == "transpose":
        return [turned(s["x"], unit.conj()).permute(1, 0, 2).contiguous()]
    k_pages, v_pages = (torch.zeros(x.shape, dtype=torch.float64, device=DEV) for x in (s["k_pages"], s["v_pages"]))
    page, slot = s["page"], s["slots"]
    k_pages[slot // page, slot % page] = turned(s["k"], unit)
    v_pages[slot // page, slot % page] = s["v"].to(torch.float64)
    return [turned(s["q"], unit), k_pages, v_pages, None]


def _exact_compact(s):
    c, page, hkv = s["case"], s["page"], s["case"]["hkv"]
    pages = [torch.zeros(x.shape, dtype=torch.float64, device=DEV) for x in (s["k_pages"], s["v_pages"])]
    kept, row, e = _compact_of(c)[1], 0, 0
    for b, n in enumerate(s["ns"]):
        for g in range(hkv):
            idx = s["kept_idx"][e: e + kept[b][g]].long()
            at = torch.arange(idx.numel(), device=DEV)
            for dst, src in zip(pages, (s["k"], s["v"])):
                dst[s["table"][b, g][at // page].long(), at % page] = src[row: row + n][idx].to(torch.float64)
            row, e = row + n, e + kept[b][g]
    return pages + [None]


def _exact_decode(s):
    c, page = s["case"], s["page"]
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    g = hq // hkv
    out = torch.zeros(c["batch"], hq, d, dtype=torch.float64, device=DEV)
    lse = torch.full((c["batch"], hq), -math.inf, dtype=torch.float64, device=DEV)
    for b, heads in enumerate(_rows_of(c)):
        for h, n in enumerate(heads):
            pages = s["table"][b, h, : _blocks(n, page)].long()
            k, v = (x[pages].reshape(-1, d)[:n].to(torch.float64) for x in (s["k"], s["v"]))
            back = s["q_pos"][b].to(torch.float64) - s["pos"][pages].reshape(-1)[:n].to(torch.float64)
            if c["window"]:
                seen = back < c["window"]
                k, v, back = k[seen], v[seen], back[seen]
            if not k.shape[0]:
                continue
            mine = slice(h * g, (h + 1) * g)
            z = (s["q"][b, mine].to(torch.float64) @ k.t()) * d ** -0.5
            if c["cap"]:
                z = torch.tanh(z / c["cap"]) * c["cap"]
            if c["bias"]:
                z = z - s["slopes"][mine].to(torch.float64)[:, None] * back
            lse[b, mine] = torch.logsumexp(z, 1)
            out[b, mine] = torch.softmax(z, 1) @ v
    return [out, lse]


def exact(case, seed):
    if case["kind"] == "tables":                                      # whole numbers only
        return None
    s = prepare(case, seed)
    return {"rotary": _exact_rotary, "compact": _exact_compact, "decode": _exact_decode}[case["kind"]](s)
