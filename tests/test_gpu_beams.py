"""A beam step on the GPU against its oracle: parents, tokens and ends are equal, scores are rounded once."""
import numpy as np
import pytest

from oracle import branch_oracle as B

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
DEV = "cuda"


@pytest.fixture(scope="module")
def lava():
    from paper_2509_09754_amd import lava as L
    return L


def dev(a, dtype=torch.float32):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV).to(dtype)


def logits_of(rng, shape, dtype, offset=0, pad=0):
    """A tensor of that shape whose rows are `pad` values apart and that begins `offset` values behind an aligned address."""
    batch, beams, V = shape
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    buf = torch.full((offset + batch * beams * (V + pad) + 8,), float("nan"), dtype=dt, device=DEV)   # a NaN that is read spoils a row
    view = buf[offset: offset + batch * beams * (V + pad)].view(batch, beams, V + pad)[:, :, :V]
    view.copy_(dev(rng.normal(size=shape) * 3.0))
    return view


def check(lava, logits, scores, n_out, done=None, end=-1, pad=0, n_tables=0, workspace=None):
    batch, beams, V = logits.shape
    i32 = lambda x: None if x is None else dev(x, torch.int32)
    sources = torch.full((n_tables, batch * n_out), 77, dtype=torch.int32, device=DEV) if n_tables else None
    got = lava.lava_beam_step(logits, dev(scores), n_out, i32(done), end, pad, sources=sources, workspace=workspace)
    torch.cuda.synchronize()
    parents, tokens, out, over = (t.cpu().numpy() for t in got)
    p, v, s, o, gap = B.beam_step(logits.double().cpu().numpy(), scores.astype(np.float32), n_out, done, end, pad)
    assert ((gap == 0) | (gap > 1e-9)).all()                          # candidates nearer than the sums' rounding would say nothing
    assert np.array_equal(parents, p) and np.array_equal(tokens, v) and np.array_equal(over, o)
    there = np.isfinite(s)
    assert np.array_equal(np.isfinite(out), there)
    # c is formed in 64 bits (its exponentials within 1e-12 of themselves) and rounded once, by half a step
    assert (np.abs(out[there] - s[there]) <= np.abs(s[there]) * 2.0 ** -24 + 1e-9).all()
    for t in range(n_tables):
        want = np.where(p >= 0, p + t * batch * beams, -1).reshape(-1)
        assert np.array_equal(sources[t].cpu().numpy(), want)
    return got


# one token; fewer tokens than places; part ends; a row that is a part exactly, one more and one less; rows at every alignment
@pytest.mark.parametrize("batch,beams,V,n_out", [
    (1, 1, 1, 1), (1, 1, 1, 3), (2, 3, 5, 8), (1, 4, 8191, 4), (1, 4, 8192, 4), (2, 4, 8193, 4), (3, 5, 50021, 5), (1, 2, 131072, 64),
    (2, 64, 700, 64), (5, 1, 1000, 16), (1, 16, 20011, 16), (70, 2, 300, 2)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("over", [False, True])
def test_beams(lava, batch, beams, V, n_out, dtype, over):
    print(f"beams {batch}x{beams}x{V} -> {n_out} {dtype} {over}", flush=True)
    rng = np.random.default_rng(batch * 100 + beams + V)
    for trial in range(2):
        logits = logits_of(rng, (batch, beams, V), dtype, offset=trial * 3, pad=trial * 5)
        scores = -20.0 * rng.random((batch, beams))
        done = (rng.random((batch, beams)) < 0.3).astype(np.int32) * -7 if over else None
        ws = torch.full((lava.lava_beam_step_workspace_bytes(batch, beams, V, n_out),), 0xFF, dtype=torch.uint8, device=DEV)
        check(lava, logits, scores, n_out, done, end=int(rng.integers(0, V)), pad=V - 1 if trial else 0, n_tables=3 * trial, workspace=ws)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_masked_tokens_and_wrong_values(lava, dtype):
    rng = np.random.default_rng(4)
    logits = logits_of(rng, (4, 5, 9001), dtype, offset=1)
    inf = float("inf")
    logits[0, 0, :] = -inf                                             # nothing can follow
    logits[0, 1, 5:] = -inf                                            # five tokens can
    logits[0, 2, 8999] = inf
    logits[0, 3, 17] = float("nan")
    logits[1, :, 3:] = -inf                                            # fifteen in all
    logits[2, :, :] = -inf
    logits[3, 0, 100:9000] = torch.finfo(logits.dtype).min             # the type's lowest value is a logit
    logits[3, 1, 7] = torch.finfo(logits.dtype).max
    scores = -5.0 * rng.random((4, 5))
    scores[3, 2], scores[3, 3], scores[3, 4] = -np.inf, np.inf, np.nan  # no continuations
    done = np.zeros((4, 5), np.int32)
    done[3, 3] = 1                                                     # nor for a beam that is done, at such a score
    check(lava, logits, scores, 16, end=2)
    check(lava, logits, scores, 20, done, end=2)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V,beams", [(9000, 2), (40000, 3), (1025, 1), (1024, 2), (65536, 64)])
def test_equals_go_to_the_lowest(lava, dtype, V, beams):
    """All logits alike, then two values, then equal beams: more equals than any list holds."""
    for n_out in (1, beams, 64):
        scores = np.full((1, beams), -2.0)
        logits = torch.full((1, beams, V), 0.25, device=DEV).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
        if beams < 64:
            logits[..., 0::2] = -0.0
            check(lava, logits, scores, n_out)
        logits[..., V // 3] = 3.0
        got = check(lava, logits, scores, n_out)
        assert int(got[1][0, 0]) == V // 3 and int(got[0][0, 0]) == 0


def test_equal_rows_have_equal_sums_wherever_they_begin(lava):
    """Beams with the same logits at the same score tie exactly, at any alignment of their rows."""
    rng = np.random.default_rng(6)
    V = 20001
    for dtype in ("bf16", "f32"):
        logits = logits_of(rng, (1, 8, V), dtype, offset=1)
        logits[0, 1:] = logits[0, :1]
        got = check(lava, logits, np.full((1, 8), -1.5), 16)
        assert got[0][0].tolist() == [0, 1, 2, 3, 4, 5, 6, 7] * 2


def test_in_place_and_replayed(lava):
    rng = np.random.default_rng(8)
    V = 5003
    logits = logits_of(rng, (3, 4, V), "f32")
    scores, done = dev(-rng.random((3, 4))), dev(rng.integers(0, 2, (3, 4)), torch.int32)
    first = (scores.clone(), done.clone())
    want = lava.lava_beam_step(logits, *[first[0]], done=first[1], end_token=9)
    ws = torch.empty(lava.lava_beam_step_workspace_bytes(3, 4, V, 4), dtype=torch.uint8, device=DEV)
    parents, tokens = (torch.empty(3, 4, dtype=torch.int32, device=DEV) for _ in range(2))
    step = lambda: lava.lava_beam_step(logits, scores, done=done, end_token=9, parents=parents, tokens=tokens, scores_out=scores, done_out=done,
                                       workspace=ws)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(4):
        scores.copy_(first[0]), done.copy_(first[1]), ws.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip((parents, tokens, scores, done), want):
            assert torch.equal(a, b)


def test_long_rows_of_many_parts(lava):
    """More parts than lanes: a vocabulary of two million."""
    rng = np.random.default_rng(11)
    logits = logits_of(rng, (1, 2, (1 << 21) + 3), "bf16")
    check(lava, logits, np.array([[-1.0, -1.25]]), 10)


def test_another_stream(lava):
    rng = np.random.default_rng(12)
    logits = logits_of(rng, (2, 3, 30000), "f32")
    scores = dev(-rng.random((2, 3)))
    want = lava.lava_beam_step(logits, scores)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = lava.lava_beam_step(logits, scores, stream=side)
    junk = [torch.full((1 << s,), 0xFF, dtype=torch.uint8, device=DEV) for s in range(8, 22)]
    torch.cuda.synchronize()
    assert len(junk) == 14 and all(torch.equal(a, b) for a, b in zip(got, want))


def test_binding_refuses(lava):
    x = torch.zeros(2, 3, 50, device=DEV)
    s = torch.zeros(2, 3, device=DEV)
    bad = [dict(logits=x.half()), dict(logits=x[0]), dict(logits=x.transpose(1, 2)), dict(logits=torch.zeros(2, 4, 50, device=DEV)[:, :3]),
           dict(scores=s[0]), dict(scores=s.double()), dict(done=s), dict(done=torch.zeros(5, dtype=torch.int32, device=DEV)),
           dict(parents=torch.zeros(2, 2, dtype=torch.int32, device=DEV)), dict(scores_out=torch.zeros(2, 3, dtype=torch.float64, device=DEV)),
           dict(sources=torch.zeros(7, dtype=torch.int32, device=DEV)), dict(logits=x.cpu())]
    for kw in bad:
        with pytest.raises(ValueError):
            lava.lava_beam_step(**{**dict(logits=x, scores=s), **kw})
    for kw in (dict(pad_token=50), dict(pad_token=-1), dict(n_out=65), dict(n_out=0), dict(workspace=torch.zeros(256, dtype=torch.uint8, device=DEV))):
        with pytest.raises(lava.LavaError):
            lava.lava_beam_step(x, s, **kw)
