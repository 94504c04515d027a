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
