"""Decode over shared pages on the GPU: how exactly the parts of a result are weighed.  Logits and values are chosen so that a result follows
from few roundings, which the bounds count."""
import numpy as np
import pytest

from test_gpu_shared import dev, shared_tables, widened

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
DEV = "cuda"
STEP = 2.0 ** -24                                                     # half a step of a 32-bit value, relative


@pytest.fixture(scope="module")
def lava():
    from paper_2509_09754_amd import lava as L
    return L


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("idle", [0, 300], ids=["few", "many"])       # own rows of more than 512 heads are decoded by themselves
def test_large_logits(lava, dtype, d, idle):
    """All logits are 4096: exactly formed, and their scaled values and differences are the same for common and own rows, so that an output is
    a quotient of two counts.  A log-sum-exp that is stored between the two parts would be off by 2^-12, and a weight with it."""
    rng = np.random.default_rng(50)
    G, Hkv, page, sizes = 4, 2, 32, [5, 3, idle]
    fronts = lambda i, g: 9 + 20 * i + g
    table, rows, n_pages = shared_tables(rng, sizes, Hkv, page, fronts, 1, 700, idle=range(8, 8 + idle))
    batch = len(rows)
    table = widened(table, page, 2 * d * (2 if dtype == "bf16" else 4))
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    k = torch.zeros(n_pages, page, d, dtype=dt, device=DEV)
    k[:, :, 5] = 64.0
    q = torch.zeros(batch, G * Hkv, d, dtype=dt, device=DEV)
    q[:, :, 5] = 64.0
    v = torch.ones(n_pages, page, d, dtype=dt, device=DEV)
    common = np.array([[fronts(i, g) for g in range(Hkv)] for i in [0] * 5 + [1] * 3])
    for b in range(8):
        for g in range(Hkv):
            v[torch.from_numpy(table[b, g, : common[b, g]]).long()] = 0.0
    pool = lava.PagePool(k, v, None, max_blocks=table.shape[2])
    desc = lava.LayerDesc.make(G * Hkv, Hkv, d, 1, dtype, softmax_scale=1.0)
    start = dev(np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32))
    out, lse = lava.lava_shared_decode(desc, q, pool, dev(table), dev(rows), start)
    torch.cuda.synchronize()
    own = 1.0 - common * page / rows[:8]
    want = torch.from_numpy(own).to(DEV).repeat_interleave(G, 1)[..., None]
    # counts are sums of exact ones; own rows' average, its weight and sum multiplied (two roundings), their sum and one division (within 2.5
    # steps each, twice)
    assert bool(((out[:8].double() - want).abs() <= 16 * STEP * want).all()), float(((out[:8].double() - want) / want).abs().max() / STEP)
    want_lse = torch.from_numpy(4096.0 + np.log(rows[:8])).to(DEV).repeat_interleave(G, 1)
    # 4096 log2 e, its sum with a logarithm (within 2^-22 of itself), the product with ln 2: half a step each, of up to 5925 and 4107
    assert bool(((lse[:8].double() - want_lse).abs() <= 4 * STEP * 4107 + 2.0 ** -20).all()), float((lse[:8].double() - want_lse).abs().max())
    assert not bool(out[8:].any()) and bool((lse[8:] == -float("inf")).all())
