"""Keys appended at the ends of the positions' range, and a step of a server -- append, then attention behind a shared prefix -- captured once
and replayed as the requests grow.  Angles of positions beyond 2^29 are those of the float64 product, which the oracle forms too."""
import numpy as np
import pytest
import torch

import paper_2601_21444_amd as apbv
from oracle import cache_oracle as co
from oracle import positions_oracle as po
from tests.test_gpu_cache import check
from tests.test_gpu_positions import Case, check_append, check_rows, f64, held, ints

pytestmark = pytest.mark.gpu

ENDS = [0, 1, -1, 2 ** 28, 2 ** 29 - 1, 2 ** 29, -(2 ** 29), 2 ** 31 - 1, 2 ** 31 - 2, -(2 ** 31), -(2 ** 31) + 1]


@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("d,rot", [(64, 64), (128, 128), (128, 48)])
def test_append_at_the_ends_of_the_positions(d, rot, norm, adjacent):
    tokens = 3 * len(ENDS)
    c = Case(tokens, 4, 2, d, rot, axes=3, adjacent=adjacent, norm=norm, seed=d + rot)
    c.at = np.stack([np.roll(ENDS * 3, shift) for shift in range(3)])
    cache = apbv.apbv_cache_empty(3, 2, d, 16)
    for t in cache:
        t.random_(0, 250)
    before = {name: held(cache, name) for name in "kv"}
    slots = np.random.default_rng(5).permutation(48)[:tokens]
    q = apbv.apbv_cache_append(cache, c.q, c.k, c.v, ints(slots), ints(c.at), c.rotation)
    check_rows(q, c.want(c.q, c.wq))
    check_append(c, cache, before, slots, 3, 16)


def test_a_servers_step_captured_and_replayed():
    """Requests grow by a token a step: their slots, positions and lengths are made on the GPU, the step's rows are new every time."""
    rng = np.random.default_rng(21)
    hq, hkv, d, page, n, frames = 8, 2, 128, 16, 6, 200
    axis = [i % 3 for i in range(d // 2)]
    inv_freq = torch.from_numpy((1e4 ** (-np.arange(d // 2) / (d // 2))).astype(np.float32)).cuda()
    weight = torch.from_numpy(1 + 0.2 * rng.standard_normal(d)).bfloat16().cuda()
    rotation = apbv.ApbvRotation(inv_freq, d, axis=axis, q_weight=weight, k_weight=weight)
    new = lambda m, h: torch.from_numpy(rng.standard_normal((m, h, d))).bfloat16().cuda()
    turned = lambda x, at: po.rotate(f64(x), np.stack([at] * 3), f64(inv_freq), axis, False, f64(weight), np.float64(np.float32(1e-6)))[0]
    n_pages = 64
    cache = apbv.apbv_cache_empty(n_pages, hkv, d, page)
    prefix_table = ints(np.arange(13)[None])
    k, v = new(frames, hkv), new(frames, hkv)
    apbv.apbv_cache_append(cache, None, k, v, ints(np.arange(frames)), ints(np.arange(frames)), rotation)
    prefix = [co.decode(*co.encode(x)) for x in (turned(k, np.arange(frames)), f64(v))]
    table = ints(np.zeros((n, 4)))
    free, count = ints(np.arange(13, n_pages)), ints([n_pages - 13])
    lengths, grow = ints([0] * n), ints([1] * n)
    starts, slots = ints([0] * (n + 1)), ints([0] * n)
    at = ints([300] * n)
    q, k, v = new(n, hq), new(n, hkv), new(n, hkv)
    turned_q, out = torch.empty_like(q), torch.empty_like(q)
    prefix_length = ints([frames])
    ws = torch.empty(apbv.apbv_cache_shared_attention_workspace_bytes(1, n, n, hq, hkv, d, 1), dtype=torch.uint8, device="cuda")
    target = torch.empty_like(lengths)

    def step():
        torch.add(lengths, grow, out=target)
        apbv.apbv_cache_map(lengths, target, table, free, count, page, n, lengths_out=lengths, starts_out=starts, slots_out=slots, free_count_out=count)
        apbv.apbv_cache_append(cache, q, k, v, slots, at, rotation, q_out=turned_q)
        apbv.apbv_cache_shared_attention(turned_q, cache, prefix_table, prefix_length, table, lengths, d ** -0.5, q_starts=starts, max_q=1, out=out, workspace=ws)
        at.add_(1)
    keys, values = [[] for _ in range(n)], [[] for _ in range(n)]
    steps = 0

    def holds(what):
        nonlocal steps
        kt, vt = turned(k, np.full(n, 300 + steps)), f64(v)
        check_rows(turned_q, po.rotate(f64(q), np.full((3, n), 300 + steps), f64(inv_freq), axis, False, f64(weight), np.float64(np.float32(1e-6))))
        for b in range(n):
            keys[b].append(co.decode(*co.encode(kt[b:b + 1])))
            values[b].append(co.decode(*co.encode(vt[b:b + 1])))
            ref, _, spread = co.attention(f64(turned_q)[b:b + 1], np.concatenate([prefix[0], *keys[b]]), np.concatenate([prefix[1], *values[b]]), d ** -0.5, True)
            check(out[b:b + 1], None, ref, None, spread, f"{what} request {b}")
        steps += 1
        assert lengths.tolist() == [steps] * n
    step()                                                            # eager
    torch.cuda.synchronize()
    holds("eager")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for rep in range(20):                                             # over the ends of pages of 16 tokens
        for t in (q, k, v):
            t.copy_(torch.from_numpy(rng.standard_normal(t.shape)).bfloat16())
        ws.fill_(0xFF)
        g.replay()
        torch.cuda.synchronize()
        holds(f"replay {rep}")
        if rep % 7 == 3:                                              # a step of the program's own between the replays
            for t in (q, k, v):
                t.copy_(torch.from_numpy(rng.standard_normal(t.shape)).bfloat16())
            step()
            torch.cuda.synchronize()
            holds("eager between")
