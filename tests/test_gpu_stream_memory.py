"""Calls that name their stream and leave outputs and workspaces to the binding: at once on two streams, and in a captured graph."""
import numpy as np
import pytest
import torch

import paper_2601_21444_amd as apbv
from tests.test_gpu_cache import Batch, dev_int

pytestmark = pytest.mark.gpu


def cache_batches():
    """Cut among workgroups and joined, of one workspace size: what one call frees fits the other."""
    rng = np.random.default_rng(41)
    xs = [Batch(rng, 16, 2, 128, 64, [(1, 6000), (1, 300)]) for _ in range(2)]
    return [(x, dev_int(x.table.tolist()), x.lengths(), dev_int(x.starts)) for x in xs]


def test_cache_attention_at_once_on_two_streams():
    batches = cache_batches()
    want = [x.run() for x, *_ in batches]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    print("two streams, no workspaces", flush=True)
    for _ in range(5):
        got = []
        for (x, table, lengths, starts), stream in zip(batches, streams):
            got.append(apbv.apbv_cache_attention(x.q, x.cache, table, lengths, x.scale, q_starts=starts, max_q=1, return_lse=True, stream=stream))
            torch.full((1 << 20,), 3.0, device="cuda")          # (what the current stream asks for next)
        for stream in streams:
            torch.cuda.current_stream().wait_stream(stream)
        got = [(out.clone(), lse.clone()) for out, lse in got]
        torch.cuda.synchronize()
        for (out, lse), (o, l) in zip(got, want):
            assert torch.equal(out, o) and torch.equal(lse, l)


def test_map_and_load_on_a_side_stream():
    x, table, _, _ = cache_batches()[0]
    slots = dev_int([int(x.table[0, j // 64]) * 64 + j % 64 for j in range(200)])
    k, v = apbv.apbv_cache_load(x.cache, slots)
    args = lambda: (dev_int([10, 0]), dev_int([11, 40]), dev_int([[3, -1], [-1, -1]]), dev_int([5, 6, 7]), dev_int([3]), 64, 60)
    want = apbv.apbv_cache_map(*args())
    side, given = torch.cuda.Stream(), args()
    torch.cuda.synchronize()
    sk, sv = apbv.apbv_cache_load(x.cache, slots, stream=side)
    got = apbv.apbv_cache_map(*given, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(k, sk) and torch.equal(v, sv) and all(torch.equal(a, b) for a, b in zip(want, got))


def test_captured_on_a_stream_that_is_not_the_current_one():
    """A fork of the captured stream: the graph's memory, whichever of its streams asks."""
    x, table, lengths, starts = cache_batches()[0]
    want, want_lse = x.run()
    graph, main, side = torch.cuda.CUDAGraph(), torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=main):
        side.wait_stream(main)
        out, lse = apbv.apbv_cache_attention(x.q, x.cache, table, lengths, x.scale, q_starts=starts, max_q=1, return_lse=True, stream=side)
        main.wait_stream(side)
    print("captured on a fork", flush=True)
    for rep in range(4):
        out.fill_(9.0)
        lse.fill_(9.0)
        eager = x.run()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, want_lse) and torch.equal(eager[0], want), rep


def test_prefill_calls_at_once_on_two_streams():
    """A split query attention, its parts merged, and a compression: each with a workspace of the binding's own."""
    g = torch.Generator(device="cuda").manual_seed(5)
    rows = lambda n, h: torch.randn((n, h, 128), generator=g, device="cuda").bfloat16()
    none = rows(0, 2)
    problems = [(rows(8, 16), rows(300, 2), rows(300, 2), rows(4000, 2), rows(4000, 2), none, none) for _ in range(2)]

    def run(p, **kw):
        parts = [apbv.apbv_query_attention(*p[:3], none, none, none, none, 0.1, return_lse=True, **kw),
                 apbv.apbv_query_attention(p[0], none, none, *p[3:], 0.1, n_splits=9, return_lse=True, **kw)]
        return parts[0] + parts[1] + apbv.apbv_compress_kv(*p[:1], *p[3:5], 100, return_scores=True, **kw)
    want = [run(p) for p in problems]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    print("prefill on two streams", flush=True)
    for _ in range(5):
        got = [run(p, stream=s) for p, s in zip(problems, streams)]
        for s in streams:
            torch.cuda.current_stream().wait_stream(s)
        assert all(torch.equal(a, b) for x, y in zip(got, want) for a, b in zip(x, y))
