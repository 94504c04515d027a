"""Calls on a stream that is not the current one, without buffers: the workspaces and outputs the binding makes are the memory of the
stream the call is enqueued on, so that work on the current stream is not given it while the call still has to run."""
import numpy as np
import pytest

from paper_2509_09754_amd import synth

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
DEV = "cuda"


@pytest.fixture(scope="module")
def lava():
    from paper_2509_09754_amd import lava as L
    return L


def i32(*shape, value=0):
    return torch.full(shape, value, dtype=torch.int32, device=DEV)


def flat(r):
    return [r] if isinstance(r, torch.Tensor) else [t for x in (r.values() if isinstance(r, dict) else r or ()) for t in flat(x)]


def make(lava):
    """{entry point: its call on a stream, without any buffer that may be left out}; small inputs, all on the current stream."""
    H, Hkv, d, w, n, budget, page = 8, 2, 64, 8, 300, 90, 16
    desc = lava.LayerDesc.make(H, Hkv, d, w, "f32")
    g = torch.Generator(device=DEV).manual_seed(5)
    rnd = lambda *s: torch.randn(*s, generator=g, device=DEV)
    q, k, v = rnd(1, H, w, d), rnd(Hkv, n, d), rnd(Hkv, n, d)
    done = lava.evict_layer(desc, n, q, k, v, budget)
    offs, idx, scores = done["head_offsets"], done["kept_idx"], done["scores"]
    q1 = rnd(1, H, d)
    one = [torch.zeros(n, dtype=t, device=DEV) for t in (torch.int32, torch.int64, torch.int32)]
    pool = lava.PagePool(rnd(80, page, d), rnd(80, page, d), max_blocks=20)
    table, rows = torch.randperm(80, generator=g, device=DEV).to(torch.int32)[:40].view(1, 2, 20), i32(1, 2, value=310)
    rot = lava.RotaryDesc.make(d)
    turns = lava.lava_rotary_turns(rot, DEV)
    state = lava.PageState.empty(3, Hkv, 40, 200, page)
    state = lava.PageState(state.block_table, state.head_rows, state.seq_pos, state.free_pages, state.n_free, page, i32(3, Hkv), i32(3), i32(1))
    new = i32(3, value=500)
    slots = torch.zeros(1500, Hkv, dtype=torch.int64, device=DEV)
    at_n, at_1, nowhere = i32(n), i32(1), torch.full((1, Hkv), -1, dtype=torch.int64, device=DEV)
    e, total, lo, hi = rnd(1, 4).abs(), *(torch.full(s, x, dtype=torch.int64, device=DEV) for s, x in (((1,), 400), ((1, 4), 10), ((1, 4), 300)))
    problem = lava.select_problem(scores, budget, one[0], one[1], one[2])
    cascade = lava.CascadeState(desc, 2, 400)
    cascade.e.fill_(1.0)
    keep = (q, k, v, done, q1, one, pool, table, rows, turns, state, new, slots, e, total, lo, hi, problem, cascade, at_n, at_1, nowhere)
    tables = lambda s: (lava.lava_page_tables(state, new, slots=slots, stream=s), state.head_rows_out, state.block_table)
    return keep, {
        "lava_window_scores": lambda s: lava.lava_window_scores(desc, [n], q, k, v, stream=s),
        "lava_select_topk": lambda s: lava.lava_select_topk(Hkv, scores, budget, stream=s),
        "lava_select_topk_batch": lambda s: lava.lava_select_topk_batch(Hkv, [problem], stream=s),
        "lava_layer_budgets": lambda s: lava.lava_layer_budgets(e, total, lo, hi, stream=s),
        "lava_compact_kv": lambda s: lava.lava_compact_kv(desc, n, k, v, offs, idx, budget, stream=s),
        "lava_compact_packed": lambda s: lava.lava_compact_packed(desc, offs, done["k_hat"], done["v_hat"], offs, idx, budget, stream=s),
        "lava_cascade_step": lambda s: lava.lava_cascade_step(desc, 0, n, k, v, scores, cascade, budget, stream=s),
        "evict_layer": lambda s: lava.evict_layer(desc, n, q, k, v, budget, stream=s),
        "lava_decode_attention": lambda s: lava.lava_decode_attention(desc, 1, q1, done["k_hat"], done["v_hat"], offs.view(1, -1), budget, stream=s),
        "lava_page_tables": tables,
        "lava_rotary": lambda s: lava.lava_rotary(rot, turns, at_n, k.transpose(0, 1), stream=s),
        "lava_rotary_append": lambda s: lava.lava_rotary_append(desc, rot, turns, at_1, q1, q1[:, :Hkv], q1[:, Hkv: 2 * Hkv], pool, nowhere, stream=s),
        "lava_paged_decode": lambda s: lava.lava_paged_decode(desc, q1, pool, table, rows, stream=s),
    }


NAMES = ["lava_window_scores", "lava_select_topk", "lava_select_topk_batch", "lava_layer_budgets", "lava_compact_kv", "lava_compact_packed",
         "lava_cascade_step", "evict_layer", "lava_decode_attention", "lava_page_tables", "lava_rotary", "lava_rotary_append", "lava_paged_decode"]


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("kind", ["torch", "handle"])
def test_buffers_are_the_streams_own(lava, monkeypatch, name, kind):
    """Nothing is launched: the addresses that reach the library are looked up in the allocator's segments."""
    print(name, kind, flush=True)
    keep, calls = make(lava)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    seen = []

    class Lib:                                                     # sizes are the library's, everything else is only written down
        def __getattr__(self, entry):
            if entry.endswith("_bytes"):
                return getattr(real, entry)
            return lambda *a: seen.append(a) or lava.LAVA_OK

    class Handle:
        cuda_stream = side.cuda_stream

    real = lava.lib
    monkeypatch.setattr(lava, "lib", Lib())
    result = calls[name](side if kind == "torch" else Handle())
    segments = torch.cuda.memory_snapshot()
    addresses = [x for a in seen for x in a if isinstance(x, int) and x > 1 << 32]
    owners = [s["stream"] for x in addresses for s in segments if s["address"] <= x < s["address"] + s["total_size"]]
    made = sum(o == side.cuda_stream for o in owners)
    print("   addresses", len(addresses), "of the stream's own", made)
    outputs = {"lava_window_scores": 3, "lava_select_topk": 4, "lava_compact_kv": 2, "lava_compact_packed": 3, "lava_decode_attention": 2,
               "lava_paged_decode": 2, "lava_rotary": 1, "lava_rotary_append": 1, "lava_layer_budgets": 1, "evict_layer": 9}.get(name, 0)
    workspace = 0 if name in ("lava_compact_kv", "lava_compact_packed", "lava_rotary", "lava_rotary_append", "lava_layer_budgets") else 1
    assert made >= outputs + workspace
    for t in flat(result)[:outputs]:
        assert any(s["stream"] == side.cuda_stream and s["address"] <= t.data_ptr() < s["address"] + s["total_size"] for s in segments)


@pytest.mark.parametrize("name", ["lava_paged_decode", "lava_page_tables", "lava_decode_attention", "evict_layer", "lava_rotary"])
def test_the_current_stream_allocates_while_the_call_waits(lava, name):
    """The side stream is kept busy first; buffers of every size are made and filled on the current stream before the call can run."""
    print(name, flush=True)
    keep, calls = make(lava)
    want = [t.clone() for t in flat(calls[name](None))]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(200_000_000)
    got = flat(calls[name](side))
    junk = [torch.full((1 << s,), 0xFF, dtype=torch.uint8, device=DEV) for s in range(8, 24) for _ in range(3)]
    waited = not side.query()
    torch.cuda.synchronize()
    assert waited
    assert len(got) == len(want) and len(junk) == 48
    for a, b in zip(got, want):
        assert torch.equal(a, b)


@pytest.mark.parametrize("name", ["lava_paged_decode", "evict_layer", "lava_decode_attention", "lava_rotary"])
def test_a_call_on_a_joined_stream_is_captured(lava, name):
    """A call without buffers on a side stream inside a capture: its buffers are the graph's, replays and eager work between them agree."""
    print(name, flush=True)
    keep, calls = make(lava)
    want = [t.clone() for t in flat(calls[name](None))]
    side = torch.cuda.Stream()
    calls[name](side)                                                # the side stream has memory of its own to begin with
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        side.wait_stream(torch.cuda.current_stream())
        got = flat(calls[name](side))
        torch.cuda.current_stream().wait_stream(side)
    for _ in range(4):
        for t in got:
            t.fill_(1)
        graph.replay()
        junk = [torch.full((1 << s,), 0xFF, dtype=torch.uint8, device=DEV) for s in range(8, 24)]
        eager = flat(calls[name](None))
        torch.cuda.synchronize()
        assert len(junk) == 16
        for a, b, c in zip(got, want, eager):
            assert torch.equal(a, b) and torch.equal(c, b)
