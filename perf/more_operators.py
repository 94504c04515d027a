"""Many continuations of one prompt over the paged cache, as calls that can be timed and compared.

Beam search, several samples of one prompt and a common system prompt have sequences that begin alike.  Four operators let
them share pages and choose between them, each through the entry points of `paper_2509_09754_amd.lava`:

  beam     the best continuations of every group of beams: log-probabilities of a step's logits, added to the beams' scores,
           the best of beams x vocabulary with parents, tokens, scores
  fork     sequence b becomes a copy of sequence source[b]: full pages are shared, the last rows copied, what nobody holds any more goes
           back to the stack (a beam step's reordering, a prompt's samples, the end of sequences)
  compact  the rows that a selection keeps of caches in pages, gathered into fewer pages; shared pages stay for those who need them
  shared   one new token per sequence over the pages, a group's common pages read once for all of its sequences

Row counts, sources, head counts and lengths are properties of a case (so its work is known); values, page numbers, the order of the
free stack and the rows kept come from the seed.  Head shapes are those of the benchmark's configurations and of the tests.
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


def _beam(name, batch, beams, vocab, dtype, over=False, pad=0):
    return dict(name=name, kind="beam", batch=batch, beams=beams, vocab=vocab, dtype=dtype, over=over, pad=pad)


def _fork(name, heads, groups, width, lo, hi, new, page, mix, form):
    return dict(name=name, kind="fork", groups=groups, width=width, lo=lo, hi=hi, new=new, page=page, mix=mix, form=form, **heads)


def _compact(name, heads, groups, width, lo, hi, new, keep, sinks, page, mix, every=1):
    return dict(name=name, kind="compact", groups=groups, width=width, lo=lo, hi=hi, new=new, keep=keep, sinks=sinks, page=page, mix=mix,
                every=every, **heads)


def _shared(name, heads, groups, width_lo, width_hi, lo, hi, new, page, mix, cap=0.0, bias=False, window=0, ctx=4):
    return dict(name=name, kind="shared", groups=groups, width_lo=width_lo, width_hi=width_hi, lo=lo, hi=hi, new=new, page=page, mix=mix,
                cap=cap, bias=bias, window=window, ctx=ctx, **heads)


def listed():
    return [
        # one user's four beams, a small vocabulary, 32-bit logits; latency counts
        _beam("beam_1x4_32k_f32", 1, 4, 32000, "f32"),
        # sixteen users, an odd vocabulary whose rows begin anywhere, a fifth of the beams finished
        _beam("beam_16x5_odd", 16, 5, 50021, "bf16", over=True),
        # a full batch of beams over a large vocabulary
        _beam("beam_64x8_131k", 64, 8, 131072, "bf16", over=True),
        # one layer of one user's eight beams after a beam step
        _fork("fork_beams8", GQA4, 1, 8, 4096, 4096, 200, 64, 1, "beams"),
        # the layers of a model as sequences of their own: 32 layers of sixteen beams, reordered at once
        _fork("fork_layers32x16", GQA4, 32, 16, 8192, 8192, 100, 64, 2, "beams"),
        # eight prompts become eight samples each; the places belonged to sequences that are over; long pages
        _fork("fork_samples8x8", GQA4, 8, 8, 32768, 131072, 300, 256, 3, "samples"),
        # one layer of one user's cache is evicted again: 512 of about 768 rows a head stay
        _compact("compact_1", GQA4, 1, 1, 6144, 6144, 40, 512, 4, 64, 4),
        # four layers' worth of eight beams that share a prompt, a fifth of it kept; odd pages' ends
        _compact("compact_4x8_beams", GQA4, 4, 8, 16384, 16384, 77, 400, 64, 32, 5),
        # a ragged batch in 32 bits, every third sequence is left as it is
        _compact("compact_48_f32", FULL, 48, 1, 8192, 32768, 0, 1024, 16, 16, 6, every=3),
        # four beams over a compressed layer
        _shared("shared_4_8k", GQA4, 1, 4, 4, 8192, 8192, 64, 64, 7),
        # sixty-four samples of a prompt of 131072 tokens whose cache was not evicted
        _shared("shared_64_131k", GQA4, 1, 64, 64, 8 * 131072, 8 * 131072, 500, 128, 8, ctx=1),
        # groups of uneven size and length, 7 heads a group, capped scores, a distance bias and a position window; pages of half a tile
        _shared("shared_6_ragged_g7", GQA7, 6, 3, 17, 16384, 65536, 90, 16, 9, cap=50.0, bias=True, window=8192, ctx=1),
    ]


def _log_int(rng, lo, hi):
    """An integer of [lo, hi], spread over its logarithm."""
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    kind = rng.choice(["beam", "fork", "compact", "shared", "shared"])
    mix, page = rng.randrange(1 << 20), rng.choice([16, 32, 64, 128, 256])
    if kind == "beam":
        dtype = rng.choice(["f32", "bf16"])
        beams = rng.choice([1, 2, 3, 4, 5, 8, 11, 16])
        vocab = _log_int(rng, 500, 262144)
        most = (1 << 26) // (beams * vocab) // (2 if dtype == "f32" else 1)
        return dict(kind="beam", batch=_log_int(rng, 1, max(1, min(128, most))), beams=beams, vocab=vocab, dtype=dtype, over=rng.random() < 0.5,
                    pad=rng.randrange(vocab))
    heads = rng.choice([GQA4, GQA4, GQA7, MHA, TINY, FULL])
    size = 2 * heads["d"] * (2 if heads["dtype"] == "bf16" else 4)     # bytes of a row of both caches
    if kind == "fork":
        groups, width = _log_int(rng, 1, 32), _log_int(rng, 2, 16)
        hi = _log_int(rng, 40 * heads["hkv"], min(131072, (1 << 30) // (groups * size)))
        return dict(kind="fork", groups=groups, width=width, lo=_log_int(rng, 20 * heads["hkv"], hi), hi=hi, new=_log_int(rng, 1, 300),
                    page=page, mix=mix, form=rng.choice(["beams", "samples"]), **heads)
    if kind == "compact":
        groups, width = _log_int(rng, 1, 48), rng.choice([1, 1, 2, 4])
        hi = _log_int(rng, 300 * heads["hkv"], max(300 * heads["hkv"], min(32768, (1 << 28) // (groups * width * size))))
        lo = _log_int(rng, 300 * heads["hkv"], hi)
        keep = _log_int(rng, 16, max(16, min(1024, lo // heads["hkv"] // 3)))
        return dict(kind="compact", groups=groups, width=width, lo=lo, hi=hi, new=_log_int(rng, 1, 200), keep=keep,
                    sinks=rng.choice([0, 4, keep // 4]), page=page, mix=mix, every=rng.choice([1, 1, 2, 3]), **heads)
    groups = _log_int(rng, 1, 12)
    width = _log_int(rng, 1, min(64, 128 // groups))
    most = (1 << 28) // (groups * size)
    if heads["dtype"] == "f32":
        most = most // 8
    hi = _log_int(rng, 64 * heads["hkv"], max(64 * heads["hkv"], min(8 * 131072, most)))
    extra = rng.random() < 0.4
    return dict(kind="shared", groups=groups, width_lo=_log_int(rng, 1, width), width_hi=width, lo=_log_int(rng, 32, hi), hi=hi,
                new=_log_int(rng, 1, 600), page=page, mix=mix, cap=rng.choice([0.0, 30.0, 50.0]) if extra else 0.0,
                bias=extra and rng.random() < 0.5, window=rng.choice([0, 256, 4096]) if extra else 0, ctx=rng.choice([1, 2, 8]), **heads)


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


def _blocks(rows, page):
    return -(-rows // page)


def _item(c):
    return 2 if c["dtype"] == "bf16" else 4


@functools.lru_cache(maxsize=64)
def _family(groups, width, lo, hi, new, hkv, mix, form):
    """(prompt rows of every group's heads, tokens that every sequence has seen since, source of every sequence).  In `samples` only the first
    sequence of a group holds the prompt, the others an older one of their own that is over."""
    num = _Numbers(mix)
    prompts, seen, source = [], [], []
    for i in range(groups):
        prompts.append(_split(num(lo, hi), hkv, num))
        seen.append(new if form == "compact" else num(1, new))
        for j in range(width):
            source.append(i * width + (num(0, width - 1) if form == "beams" else 0 if form == "samples" else j))
    return prompts, seen, source


def _family_of(c):
    return _family(c["groups"], c["width"], c["lo"], c["hi"], c["new"], c["hkv"], c["mix"], c["form"] if c["kind"] == "fork" else "compact")


def _head_rows(c):
    """(rows of every head before, pages that it shares with its group) of a fork's or compaction's sequences."""
    prompts, seen, _ = _family_of(c)
    rows, shared = [], []
    for i, prompt in enumerate(prompts):
        for j in range(c["width"]):
            if c["kind"] == "fork" and c["form"] == "samples":
                rows.append(list(prompt) if j == 0 else [seen[i] + x // 8 for x in prompt])
                shared.append([0] * c["hkv"])
            else:
                rows.append([x + seen[i] for x in prompt])
                shared.append([x // c["page"] if c["width"] > 1 else 0 for x in prompt])
    return rows, shared


def _keeper(source, b):
    """Whether sequence b goes on with the last page of the sequence that it is made of: the sequence itself, or else its first copy."""
    s = source[b]
    return b == s if source[s] == s else b == source.index(s)


@functools.lru_cache(maxsize=16)
def _change_numbers(key):
    """Of every head: (sequence it comes from, rows after, leading rows that stay where they are, rows that are copied), and the most rows copied."""
    c = dict(key)
    rows, _ = _head_rows(c)
    source = _family_of(c)[2]
    num = _Numbers(c["mix"] + 77)
    out = []
    for b, s in enumerate(source):
        keeper = _keeper(source, b)
        kept_whole = c["kind"] == "fork" or b % c["every"] != 0 and c["every"] > 1
        for g in range(c["hkv"]):
            old = rows[s][g]
            if kept_whole:
                n = same = old
            else:
                n = min(old - 1, max(1, c["keep"] * num(30, 170) // 100))
                same = min(c["sinks"], n)
            p = c["page"]
            stay = min(same, n) // p * p
            if n % p and same >= n and n // p == old // p and old % p and keeper:
                stay = n
            out.append((s, n, min(same, n), n - stay))
    return out, max(x[3] for x in out)


def _change_of(c):
    return _change_numbers(tuple(sorted((k, v) for k, v in c.items() if k != "name")))


@functools.lru_cache(maxsize=64)
def _groups(groups, width_lo, width_hi, lo, hi, new, hkv, mix, even):
    """(prompt rows of every group's heads, new tokens of each of its sequences)."""
    num = _Numbers(mix)
    prompts, tokens = [], []
    for _ in range(groups):
        total = num(lo, hi)
        prompts.append([total // hkv] * hkv if even else _split(total, hkv, num))
        tokens.append([num(1, new) for _ in range(num(width_lo, width_hi))])
    return prompts, tokens


def _groups_of(c):
    return _groups(c["groups"], c["width_lo"], c["width_hi"], c["lo"], c["hi"], c["new"], c["hkv"], c["mix"], c["lo"] == c["hi"] and c["ctx"] == 1)


def _context(c, prompt):
    """Tokens that a group's prompt had: `ctx` times its longest head, which was evicted to that."""
    return max(1, c["ctx"] * max(prompt))


# ------------------------------------------------------------------------------------------- inputs
def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _generator(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _ints(rows, dtype=torch.int32):
    return torch.tensor(rows, dtype=dtype, device=DEV)


def _normal(gen, *shape, dtype, scale=1.0):
    """Normal values of the storage type, drawn in parts so that large ones need no second copy."""
    out = torch.empty(shape, dtype=dtype, device=DEV)
    for part in out.view(-1).split(1 << 26):
        part.copy_(torch.randn(part.shape, generator=gen, device=DEV) * scale)
    return out


def _prepare_beam(c, gen):
    batch, beams, vocab = c["batch"], c["beams"], c["vocab"]
    logits = _normal(gen, batch, beams, vocab, dtype=_dtype(c), scale=2.5)
    best = torch.randint(0, vocab, (batch, beams, 6), generator=gen, device=DEV)       # a few tokens stand out, as they do in a text
    lift = torch.rand(batch, beams, 6, generator=gen, device=DEV) * 6.0 + 8.0
    logits.scatter_(2, best, lift.to(logits.dtype))
    scores = -40.0 * torch.rand(batch, beams, generator=gen, device=DEV) / beams - 5.0
    i32 = lambda: torch.empty(batch, beams, dtype=torch.int32, device=DEV)
    over = torch.arange(batch * beams, device=DEV).view(batch, beams) % 5 == 4
    return dict(logits=logits, scores=scores, over=over.to(torch.int32) if c["over"] else None, end=vocab // 3, pad=c["pad"], parents=i32(), tokens=i32(),
                out=torch.empty_like(scores), over_out=i32())


def _family_tables(rows, shared, width, page, gen, spare):
    """(block table, pages in the pool, numbers of the unused pages); sequences of a group have the first `shared` pages of their heads in common."""
    batch, hkv = rows.shape
    nb = (rows.long() + page - 1) // page
    blocks = max(1, int(nb.max()))
    j = torch.arange(blocks, device=DEV)
    first = torch.arange(batch, device=DEV) // width * width
    mine = (j < nb[..., None]) & ~((j < shared[..., None]) & (torch.arange(batch, device=DEV) != first)[:, None, None])
    used = int(mine.sum())
    n_pages = used + max(1, spare)
    order = torch.randperm(n_pages, generator=gen, device=DEV).to(torch.int32)
    table = torch.full((batch, hkv, blocks), -1, dtype=torch.int32, device=DEV)
    table[mine] = order[:used]
    there = (j < nb[..., None]) & ~mine
    return torch.where(there, table[first], table).contiguous(), n_pages, order[used:].contiguous()


def _prepare_change(c, gen):
    rows_host, shared = _head_rows(c)
    numbers, most = _change_of(c)
    source = _family_of(c)[2]
    page, hkv, d, dt = c["page"], c["hkv"], c["d"], _dtype(c)
    batch = len(rows_host)
    need = sum(_blocks(n, page) - _blocks(n - copied, page) for _, n, _, copied in numbers)
    rows = _ints(rows_host)
    table, n_pages, unused = _family_tables(rows, _ints(shared), c["width"], page, gen, need + 5)
    after = max(1, max(_blocks(n, page) for _, n, _, _ in numbers))
    table = torch.nn.functional.pad(table, (0, max(0, after - table.shape[-1])), value=-1).contiguous()
    free = torch.full((n_pages,), -1, dtype=torch.int32, device=DEV)
    free[: unused.numel()] = unused
    pos = _ints([2 * max(r) for r in rows_host])
    i32 = lambda *shape: torch.full(shape, -1, dtype=torch.int32, device=DEV)
    s = dict(page=page, batch=batch, n_pages=n_pages, table=table, rows=rows, pos=pos, free=free, n_free=_ints([unused.numel()]), most=most,
             n_copied=sum(x[3] for x in numbers), source=_ints(source), table_out=torch.full_like(table, -1), rows_out=i32(batch, hkv), pos_out=i32(batch),
             free_out=i32(n_pages), n_free_out=i32(1), error=torch.zeros(1, dtype=torch.int32, device=DEV), kept=None, counts=None, evict=None)
    s["k"], s["v"] = (_normal(gen, n_pages, page, d, dtype=dt) for _ in range(2))
    s["pos_pages"] = torch.randint(0, 131072, (n_pages, page), generator=gen, device=DEV).to(torch.int32)
    if c["kind"] == "compact":
        evicted = [c["every"] == 1 or b % c["every"] == 0 for b in range(batch)]
        counts = [[numbers[b * hkv + g][1] if evicted[b] else 0 for g in range(hkv)] for b in range(batch)]
        kept = i32(batch, max(1, max(sum(x) for x in counts)))
        for b in range(batch):
            at = 0
            for g in range(hkv if evicted[b] else 0):
                old, n, same = rows_host[b][g], counts[b][g], numbers[b * hkv + g][2]
                kept[b, at: at + same] = torch.arange(same, dtype=torch.int32, device=DEV)
                rest = torch.randperm(old - same - 1, generator=gen, device=DEV)[: n - same].sort().values + same + 1   # never row `same`
                kept[b, at + same: at + n] = rest.to(torch.int32)
                at += n
        s.update(kept=kept, counts=_ints(counts), evict=_ints([int(x) for x in evicted]) if c["every"] > 1 else None)
    return s


def _prepare_shared(c, gen):
    prompts, tokens = _groups_of(c)
    page, hq, hkv, d, dt = c["page"], c["hq"], c["hkv"], c["d"], _dtype(c)
    sizes = [len(t) for t in tokens]
    batch, wide = sum(sizes), max(sizes)
    group = [i for i, n in enumerate(sizes) for _ in range(n)]
    new = [t for ts in tokens for t in ts]
    prompt = _ints(prompts)[group]                                     # rows of the prompt that every sequence's heads hold
    rows = prompt + _ints(new)[:, None]
    front = torch.where(_ints(sizes)[group][:, None] > 1, prompt // page, 0)
    start = [sum(sizes[:i]) for i in range(len(sizes) + 1)]
    nb = (rows.long() + page - 1) // page
    blocks = max(1, int(nb.max()))
    j = torch.arange(blocks, device=DEV)
    first = _ints(start, torch.int64)[group]
    mine = (j < nb[..., None]) & ~((j < front[..., None]) & (torch.arange(batch, device=DEV) != first)[:, None, None])
    used = int(mine.sum())
    n_pages = used + 5
    table = torch.full((batch, hkv, blocks), -1, dtype=torch.int32, device=DEV)
    table[mine] = torch.randperm(n_pages, generator=gen, device=DEV)[:used].to(torch.int32)
    table = torch.where((j < nb[..., None]) & ~mine, table[first], table).contiguous()
    ctx = _ints([_context(c, p) for p in prompts])[group]
    pos = torch.zeros(n_pages, page, dtype=torch.int32, device=DEV)
    r = torch.arange(blocks * page, device=DEV)
    for b in range(batch):            # row r of a head of n prompt rows: position (r + 1) * ctx // n - 1, then the new tokens one by one
        n = prompt[b].long()[:, None]
        x = torch.where(r < n, (r + 1) * ctx[b].long() // n.clamp(min=1) - 1, ctx[b].long() + r - n)
        there = r < rows[b].long()[:, None]
        slot = table[b].long()[:, r // page] * page + r % page
        pos.view(-1)[slot[there]] = x[there].to(torch.int32)
    member = torch.zeros(len(sizes), wide, dtype=torch.int64, device=DEV)
    place = [b - start[group[b]] for b in range(batch)]
    member[group, place] = torch.arange(batch, device=DEV)
    return dict(page=page, k=_normal(gen, n_pages, page, d, dtype=dt), v=_normal(gen, n_pages, page, d, dtype=dt), pos=pos, table=table, rows=rows,
                q=_normal(gen, batch, hq, d, dtype=dt), q_pos=(ctx + _ints(new) - 1).to(torch.int32), start=_ints(start), batch=batch,
                slopes=2.0 ** (-8.0 * (1 + torch.arange(hq, device=DEV, dtype=torch.float32)) / hq),
                front=front * page, member=member, group=_ints(group, torch.int64), place=_ints(place, torch.int64),
                top_front=max(1, int((front * page).max())), top_rest=int((rows - front * page).max()),
                out=torch.empty(batch, hq, d, device=DEV), lse=torch.empty(batch, hq, device=DEV))


_PREPARE = {"beam": _prepare_beam, "fork": _prepare_change, "compact": _prepare_change, "shared": _prepare_shared}


def prepare(case, seed):
    s = _PREPARE[case["kind"]](case, _generator(seed))
    s["case"] = case
    return s


# ------------------------------------------------------------------------------------------- plain forms
def _plain_beam(s):
    batch, beams, vocab = s["logits"].shape
    x = s["logits"].double()                                           # which of two candidates is better is seen in 64 bits
    m = x.amax(2, keepdim=True)
    x -= m + (x - m).exp_().sum(2, keepdim=True).log()
    x += s["scores"].double()[..., None]
    if s["over"] is not None:                                          # a finished beam goes on as it is, with the padding token
        over = s["over"][..., None] != 0
        token = torch.arange(vocab, device=DEV)
        x = torch.where(over, torch.where(token == s["pad"], s["scores"].double()[..., None], -math.inf), x)
    x = x.view(batch, beams * vocab)
    last = x.topk(beams, 1).values[:, -1:]                             # the last that is good enough, of its equals the first ones
    equal = x == last
    places = beams - (x > last).sum(1, keepdim=True)
    chosen = (x > last) | (equal & (equal.cumsum(1, dtype=torch.int32) <= places))
    at = torch.where(chosen, beams * vocab - torch.arange(beams * vocab, dtype=torch.int32, device=DEV), 0).topk(beams, 1).indices
    value = x.gather(1, at)
    order = value.sort(dim=1, descending=True, stable=True).indices
    at, value = at.gather(1, order), value.gather(1, order)
    beam, token = at // vocab, at % vocab
    s["parents"].copy_(beam + beams * torch.arange(batch, device=DEV)[:, None])
    s["tokens"].copy_(token)
    s["out"].copy_(value)
    done = token == s["end"]
    s["over_out"].copy_(done | (s["over"].gather(1, beam) != 0) if s["over"] is not None else done)
    return [s["parents"], s["tokens"], s["out"], s["over_out"]]


def _change_answer(s):
    return [s["table_out"], s["rows_out"], s["pos_out"], s["free_out"], s["n_free_out"], s["error"], s["k"], s["v"], s["pos_pages"]]


def _plain_change(s):
    page, batch, n_pages = s["page"], s["batch"], s["n_pages"]
    hkv, width = s["table"].shape[1:]
    heads = batch * hkv
    b = torch.arange(batch, device=DEV)
    source = s["source"].long()
    old = s["rows"].long()[source].view(heads)                         # of the sequence that a head comes from
    table = s["table"][source].view(heads, width)
    n = same = old
    if s["kept"] is not None:
        evict = s["evict"].repeat_interleave(hkv, output_size=heads) != 0 if s["evict"] is not None else torch.ones_like(old, dtype=torch.bool)
        counts = s["counts"].long()
        begin = (counts.cumsum(1) - counts).view(heads)
        n = torch.where(evict, counts.view(heads), old)
        i = torch.arange(s["kept"].shape[1], device=DEV)
        seq = b.repeat_interleave(hkv, output_size=heads)
        where = (begin[:, None] + i).clamp(max=s["kept"].shape[1] - 1)
        in_place = (s["kept"][seq[:, None], where] == i) & (i < n[:, None])
        same = torch.where(evict, in_place.cumprod(1).sum(1), old)
    alike = source[:, None] == source
    earlier = (alike & (b < b[:, None])).any(1)
    keeper = torch.where(source[source] == source, b == source, ~earlier).repeat_interleave(hkv, output_size=heads)
    stay = same // page + (keeper & (n % page != 0) & (same >= n) & (n // page == old // page) & (old % page != 0))
    blocks = (n + page - 1) // page
    fresh = blocks - stay
    begin_fresh = fresh.cumsum(0) - fresh
    j = torch.arange(width, device=DEV)
    top = s["n_free"].long()
    is_fresh = (j >= stay[:, None]) & (j < blocks[:, None])
    popped = (top - 1 - begin_fresh + stay)[:, None] - j
    out = torch.where(is_fresh, s["free"][torch.where(is_fresh, popped, 0)], table)
    s["table_out"].copy_(torch.where(j < blocks[:, None], out, s["table_out"].view(heads, width)).view(batch, hkv, width))
    s["rows_out"].copy_(n.view(batch, hkv))
    s["pos_out"].copy_(s["pos"][source])
    # pages that nobody holds any more, in the order in which the old tables name them first
    stays = torch.where(j < stay[:, None], table.long(), n_pages)
    alive = torch.zeros(n_pages + 1, dtype=torch.bool, device=DEV)
    alive[stays.view(-1)] = True
    before = s["table"].view(heads, width)
    held = j < ((s["rows"].view(heads, 1).long() + page - 1) // page)
    entry = torch.arange(heads * width, device=DEV)
    first = torch.full((n_pages + 1,), heads * width, dtype=torch.int64, device=DEV)
    first.scatter_reduce_(0, torch.where(held, before.long(), n_pages).view(-1), entry, "amin")
    first = torch.where(alive, heads * width, first)[:n_pages]
    first, back = first.sort()
    left = top - fresh.sum()
    r = torch.arange(n_pages, device=DEV)
    long = torch.where(r < left, s["free"], s["free_out"])
    long = torch.cat([long, long.new_zeros(1)])
    long[torch.where(first < heads * width, left + r, n_pages)] = back.to(torch.int32)
    s["free_out"].copy_(long[:n_pages])
    s["n_free_out"].copy_(left + (first < heads * width).sum())
    # the rows that change pages
    copied = n - torch.minimum(stay * page, n)
    total = s["n_copied"]
    head = torch.arange(heads, device=DEV).repeat_interleave(copied, output_size=total)
    t = torch.arange(total, device=DEV) - (copied.cumsum(0) - copied)[head] + (stay * page)[head]
    row = t
    if s["kept"] is not None:
        row = torch.where(evict[head], s["kept"][head // hkv, (begin[head] + t).clamp(max=s["kept"].shape[1] - 1)].long(), t)
    src = table[head, row // page].long() * page + row % page
    dst = s["table_out"].view(heads, width)[head, t // page].long() * page + t % page
    d = s["k"].shape[-1]
    s["k"].view(-1, d)[dst] = s["k"].view(-1, d)[src]
    s["v"].view(-1, d)[dst] = s["v"].view(-1, d)[src]
    s["pos_pages"].view(-1)[dst] = s["pos_pages"].view(-1)[src]
    return _change_answer(s)


def _logits(s, q, k, back, slopes):
    """Logits [.., rows, queries] of keys [.., rows, d] and the rows' distances [.., rows, queries] (an unseen row: -inf)."""
    c = s["case"]
    z = torch.bmm(k.float(), q.transpose(1, 2).contiguous()) / math.sqrt(c["d"])
    if c["cap"]:
        z = c["cap"] * torch.tanh(z / c["cap"])
    if c["bias"]:
        z = z - slopes * back
    if c["window"] or c["bias"]:
        z = torch.where((back >= 0) & (back < (c["window"] or 1 << 31)), z, -math.inf)
    return z


def _plain_shared(s):
    c, page, batch = s["case"], s["page"], s["batch"]
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    g = hq // hkv
    q = s["q"].float().view(batch, hkv, g, d)
    k, v, pos = s["k"].view(-1, d), s["v"].view(-1, d), s["pos"].view(-1)
    # the common pages once for all sequences of a group, which are padded to the widest
    groups, wide = s["member"].shape
    r = torch.arange(s["top_front"], device=DEV)
    lead = s["member"][:, 0]
    there = r < s["front"][lead].view(groups * hkv, 1)
    slot = torch.where(there, s["table"][lead].view(groups * hkv, -1)[:, r // page].long() * page + r % page, 0)
    q_group = q[s["member"]].permute(0, 2, 1, 3, 4).reshape(groups * hkv, wide * g, d)
    slopes = s["slopes"].view(hkv, 1, g)
    back = 0
    if c["bias"] or c["window"]:
        q_pos = s["q_pos"][s["member"]][:, None, :, None].expand(groups, hkv, wide, g).reshape(groups * hkv, 1, wide * g)
        back = q_pos - pos[slot][..., None]
    z = _logits(s, q_group, k[slot], back, slopes.repeat(groups, 1, wide))
    z = torch.where(there[..., None], z, -math.inf)
    m_front = z.amax(1, keepdim=True)
    p = torch.exp(z - torch.where(m_front == -math.inf, 0.0, m_front))
    sum_front = p.sum(1)
    front = torch.bmm(p.transpose(1, 2).contiguous(), v[slot].float())
    mine = lambda x: x.reshape(groups, hkv, wide, g, -1)[s["group"], :, s["place"]]       # [batch, hkv, g, ..]
    m_front, sum_front, front = mine(m_front), mine(sum_front), mine(front)
    # every sequence's own rows
    heads = batch * hkv
    skip = s["front"].view(heads, 1).long()
    r = skip + torch.arange(s["top_rest"], device=DEV)
    there = r < s["rows"].view(heads, 1)
    slot = torch.where(there, s["table"].view(heads, -1).gather(1, torch.where(there, r // page, 0)).long() * page + r % page, 0)
    if c["bias"] or c["window"]:
        back = (s["q_pos"].repeat_interleave(hkv, output_size=heads)[:, None] - pos[slot])[..., None]
    z = _logits(s, q.reshape(heads, g, d), k[slot], back, slopes.repeat(batch, 1, 1))
    z = torch.where(there[..., None], z, -math.inf)
    m_rest = z.amax(1).view(batch, hkv, g, 1)
    m = torch.maximum(m_front, m_rest)
    m = torch.where(m == -math.inf, 0.0, m)
    p = torch.exp(z - m.view(heads, 1, g))
    rest = torch.bmm(p.transpose(1, 2).contiguous(), v[slot].float()).view(batch, hkv, g, d)
    weight = torch.exp(m_front - m)
    total = p.sum(1).view(batch, hkv, g, 1) + weight * sum_front
    s["out"].copy_(((rest + weight * front) / torch.where(total > 0, total, 1.0)).view(batch, hq, d))
    s["lse"].copy_((m + total.log()).view(batch, hq))
    return [s["out"], s["lse"]]


_PLAIN = {"beam": _plain_beam, "fork": _plain_change, "compact": _plain_change, "shared": _plain_shared}


# ------------------------------------------------------------------------------------------- the framework's calls
@functools.lru_cache(maxsize=64)
def _desc(hq, hkv, d, dtype):
    from paper_2509_09754_amd import lava
    return lava.LayerDesc.make(hq, hkv, d, 1, dtype)


def _desc_of(c):
    return _desc(c["hq"], c["hkv"], c["d"], c["dtype"])


def _handles(s):
    """What a program makes once of its buffers: the pool's description, the state, workspaces."""
    from paper_2509_09754_amd import lava
    c, h = s["case"], {"lava": lava}
    workspace = lambda need: torch.empty(need, dtype=torch.uint8, device=DEV)
    if c["kind"] == "beam":
        h["workspace"] = workspace(lava.lava_beam_step_workspace_bytes(c["batch"], c["beams"], c["vocab"], c["beams"]))
        return h
    h["pool"] = lava.PagePool(s["k"], s["v"], s["pos"] if c["kind"] == "shared" else s["pos_pages"], max_blocks=s["table"].shape[-1])
    if c["kind"] == "shared":
        h["options"] = lava.DecodeOptions.make(softcap=c["cap"], window=c["window"], slopes=s["slopes"] if c["bias"] else None)
        h["workspace"] = workspace(lava.lava_shared_decode_workspace_bytes(_desc_of(c), s["batch"], s["table"].shape[-1]))
        return h
    h["state"] = lava.PageState(s["table"], s["rows"], s["pos"], s["free"], s["n_free"], page_rows=s["page"], head_rows_out=s["rows_out"],
                                seq_pos_out=s["pos_out"], n_free_out=s["n_free_out"], error=s["error"])
    h["workspace"] = workspace(lava.lava_page_fork_workspace_bytes(s["batch"], c["hkv"], s["table"].shape[-1], s["n_pages"]))
    return h


def _own(s):
    c = s["case"]
    h = s.get("handles")
    if h is None:
        h = s["handles"] = _handles(s)
    lava = h["lava"]
    if c["kind"] == "beam":
        lava.lava_beam_step(s["logits"], s["scores"], done=s["over"], end_token=s["end"], pad_token=s["pad"], parents=s["parents"],
                            tokens=s["tokens"], scores_out=s["out"], done_out=s["over_out"], workspace=h["workspace"])
        return [s["parents"], s["tokens"], s["out"], s["over_out"]]
    if c["kind"] == "fork":
        lava.lava_page_fork(_desc_of(c), h["pool"], h["state"], s["source"], block_table_out=s["table_out"], free_pages_out=s["free_out"],
                            workspace=h["workspace"])
        return _change_answer(s)
    if c["kind"] == "compact":
        lava.lava_page_compact(_desc_of(c), h["pool"], h["state"], s["counts"], s["kept"], evict=s["evict"], block_table_out=s["table_out"],
                               free_pages_out=s["free_out"], workspace=h["workspace"])
        return _change_answer(s)
    lava.lava_shared_decode(_desc_of(c), s["q"], h["pool"], s["table"], s["rows"], s["start"], options=h["options"], q_pos=s["q_pos"],
                            out=s["out"], lse=s["lse"], workspace=h["workspace"])
    return [s["out"], s["lse"]]


def run(state):
    return _own(state) if own else _PLAIN[state["case"]["kind"]](state)


# ------------------------------------------------------------------------------------------- work
def _seen_from(prompt, ctx, first):
    """The first row of a head of `prompt` rows whose position, (r + 1) * ctx // prompt - 1, is at least `first`."""
    return max(0, _blocks(prompt * (first + 1), ctx) - 1) if first > 0 else 0


def work(case):
    c = case
    if c["kind"] == "beam":
        n = c["batch"] * c["beams"]
        rows = n - (n + 0) // 5 if c["over"] else n                    # finished beams' logits need not be read
        return {"bytes": rows * c["vocab"] * _item(c) + n * 24, "flops": rows * c["vocab"] * 4}
    row = 2 * c["d"] * _item(c) + 4                                    # a row of both caches and its position
    if c["kind"] in ("fork", "compact"):
        numbers, _ = _change_of(c)
        rows, _ = _head_rows(c)
        copied, page = sum(x[3] for x in numbers), c["page"]
        n = copied * 2 * row + sum(4 * _blocks(x[1], page) for x in numbers)             # rows both ways, the new tables
        n += sum(4 * _blocks(x, page) for r in rows for x in r) + 16 * len(numbers)      # the old tables, row counts
        n += sum(4 * x[1] for x in numbers) if c["kind"] == "compact" else 0
        return {"bytes": n, "flops": n // 4}
    prompts, tokens = _groups_of(c)
    n = flops = 0
    g = c["hq"] // c["hkv"]
    for prompt, new in zip(prompts, tokens):
        ctx = _context(c, prompt)
        for x in prompt:
            front = x // c["page"] * c["page"] if len(new) > 1 else 0
            first = [_seen_from(x, ctx, ctx + t - c["window"]) if c["window"] else 0 for t in new]   # of each sequence, at position ctx + t - 1
            n += max(0, front - min(first)) * row
            for t, f in zip(new, first):
                own_rows = x + t - max(front, min(f, x)) if not c["window"] else min(c["window"], x + t - max(front, min(f, x)))
                n += own_rows * row
                flops += (max(0, front - f) + own_rows) * 4 * g * c["d"]
    batch = sum(len(t) for t in tokens)
    n += batch * c["hq"] * (c["d"] * (_item(c) + 4) + 4)
    return {"bytes": n, "flops": flops}


# ------------------------------------------------------------------------------------------- in 64 bits
def _exact_beam(s):
    batch, beams, vocab = s["logits"].shape
    best = []
    for b in range(batch):
        found = []
        for i in range(beams):
            score = s["scores"][b, i].to(torch.float64)
            if s["over"] is not None and int(s["over"][b, i]) != 0:
                found.append(score[None])
                continue
            log_p = torch.log_softmax(s["logits"][b, i].to(torch.float64), 0)
            found.append(torch.topk(log_p, min(beams, vocab)).values + score)
        best.append(torch.cat(found).sort(descending=True).values[:beams])
    return [None, None, torch.stack(best), None]


def _exact_shared(s):
    c, page = s["case"], s["page"]
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    g = hq // hkv
    out = torch.zeros(s["batch"], hq, d, dtype=torch.float64, device=DEV)
    lse = torch.full((s["batch"], hq), -math.inf, dtype=torch.float64, device=DEV)
    rows = s["rows"].tolist()
    for b in range(s["batch"]):
        for h in range(hkv):
            n = rows[b][h]
            pages = s["table"][b, h, : _blocks(n, page)].long()
            k, v = (x[pages].reshape(-1, d)[:n].to(torch.float64) for x in (s["k"], s["v"]))
            mine = slice(h * g, (h + 1) * g)
            z = (s["q"][b, mine].to(torch.float64) @ k.t()) * d ** -0.5
            if c["cap"]:
                z = torch.tanh(z / c["cap"]) * c["cap"]
            back = s["q_pos"][b].to(torch.float64) - s["pos"][pages].reshape(-1)[:n].to(torch.float64)
            if c["bias"]:
                z = z - s["slopes"][mine].to(torch.float64)[:, None] * back
            if c["window"]:
                z[:, back >= c["window"]] = -math.inf
            lse[b, mine] = torch.logsumexp(z, 1)
            out[b, mine] = torch.softmax(z, 1) @ v
    return [out, lse]


def exact(case, seed):
    if case["kind"] in ("fork", "compact"):                            # whole numbers and copies only
        return None
    s = prepare(case, seed)
    return {"beam": _exact_beam, "shared": _exact_shared}[case["kind"]](s)
