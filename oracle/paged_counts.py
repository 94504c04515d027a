"""Pages whose attention is a count, for decode steps over pages: keys are on or off for each query head of a group, values are small whole
numbers.  A query's logit is 0 for rows that are on and so low for the others that they weigh nothing, so the output is a sum of whole
numbers over a number of rows, exact in 32 bits up to one division, whatever the order of summation: a row that is lost, read twice
or paired with another row's value moves it by far more than a rounding.  Works on torch tensors of any device, in 64 bits; shares no code with the
library."""
from __future__ import annotations

import torch

SCALE, QUERY, OFF = 0.125, 8.0, -1024.0          # logit of a row that is off: SCALE * QUERY * OFF
MOST = 7                                         # largest value


class Pages:
    """n_pages pages of `page` rows; on[t] says which rows count for query head t of a group."""

    def __init__(self, seed, n_pages, page, d, span=1000, device="cpu"):
        g = torch.Generator(device=device).manual_seed(seed)
        rand = lambda hi, *s: torch.randint(0, hi, s, generator=g, device=device)
        self.n_pages, self.page, self.d, self.device = n_pages, page, d, device
        self.on = rand(2, 8, n_pages, page) == 1
        self.k = rand(3, n_pages, page, d).double() - 1.0          # what a query does not look at
        self.k[..., :8] = torch.where(self.on, 0.0, OFF).permute(1, 2, 0)
        self.v = rand(MOST + 1, n_pages, page, d).double()
        self.pos = rand(span, n_pages, page).to(torch.int32)

    def queries(self, batch, H, group):
        q = torch.zeros(batch, H, self.d, dtype=torch.float64, device=self.device)
        h = torch.arange(H, device=self.device)
        q[:, h, h % group] = QUERY
        return q

    def attend(self, table, rows, group, window=0, q_pos=None, softcap=0.0):
        """table [batch, heads, blocks], rows [batch, heads] (host lists of lengths are fine).  Returns (out, lse, tol, tol_lse)."""
        batch, heads, blocks = table.shape
        rows = torch.as_tensor(rows, device=self.device).long()
        out = torch.zeros(batch, heads * group, self.d, dtype=torch.float64, device=self.device)
        number = torch.zeros(batch, heads * group, dtype=torch.float64, device=self.device)
        off = torch.zeros(batch, heads * group, dtype=torch.bool, device=self.device)
        views = {None: None} if not window else {int(x): None for x in q_pos.unique()}
        for at in views:
            seqs = torch.arange(batch, device=self.device) if at is None else (q_pos == at).nonzero().view(-1)
            back = None if at is None else at - self.pos.long()
            seen = torch.ones(self.n_pages, self.page, dtype=torch.bool, device=self.device) if at is None else (back >= 0) & (back < window)
            tab, n = table[seqs].reshape(-1, blocks).long(), rows[seqs].reshape(-1)
            whole, part = n // self.page, n % self.page
            used = torch.arange(blocks, device=self.device) < whole[:, None]
            times = torch.zeros(tab.shape[0], self.n_pages, dtype=torch.float64, device=self.device)
            times.scatter_add_(1, torch.where(used, tab, 0), used.double())
            last = torch.where(part > 0, tab.gather(1, whole.clamp(max=blocks - 1)[:, None])[:, 0], 0)
            ends = torch.arange(self.page, device=self.device) < part[:, None]

            def count(which):                                       # rows, and their values, of every head
                w = which.double()
                per_page = (w[..., None] * self.v).sum(1)
                e = (which[last] & ends).double()
                tail = torch.stack([(x[:, None] * self.v[p]).sum(0) for x, p in zip(e, last)]) if e.shape[0] < 64 else _weighted(e, self.v, last)
                return times @ w.sum(1) + e.sum(1), times @ per_page + tail

            every = count(seen)
            for t in range(group):
                some = count(seen & self.on[t])
                none = some[0] == 0
                c, s = torch.where(none, every[0], some[0]), torch.where(none[:, None], every[1], some[1])
                h = torch.arange(heads, device=self.device) * group + t
                out[seqs[:, None], h] = (s / c.clamp(min=1.0)[:, None]).view(len(seqs), heads, self.d)
                number[seqs[:, None], h] = c.view(len(seqs), heads)
                off[seqs[:, None], h] = none.view(len(seqs), heads)
        assert MOST * float(number.max()) < 2 ** 24                 # sums of whole numbers are exact
        low = SCALE * QUERY * OFF
        base = torch.where(off, -softcap if softcap else low, 0.0)
        lse = base + number.log()
        # one division (within 2.5 steps, 2^-21.6 of the quotient); with a cap the rows that are off weigh e^-cap each.  The logarithm within two
        # steps, the maximum and the sum of both rounded, the cap's own 2^-20
        extra = float(number.max()) * torch.exp(torch.tensor(-softcap, dtype=torch.float64)).item() if softcap else 0.0
        tol = out * 2.0 ** -21 + MOST * extra
        tol_lse = 2.0 ** -21 * (1.0 + lse.abs() + base.abs()) + extra + softcap * 2.0 ** -19
        return out, lse, tol, tol_lse


def _weighted(w, v, pages):
    """sum over rows of w[i][row] * v[pages[i]][row], in parts."""
    out = torch.empty(w.shape[0], v.shape[2], dtype=v.dtype, device=v.device)
    for i in range(0, w.shape[0], 512):
        out[i: i + 512] = (w[i: i + 512, :, None] * v[pages[i: i + 512]]).sum(1)
    return out
