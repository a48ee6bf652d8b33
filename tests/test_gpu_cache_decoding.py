"""apbv_cache_map in decoding steps, where no request grows by more than a few tokens and every thread serves its own requests:
against the oracle, at numbers of requests below, at and beyond a wave, a workgroup's threads and a thread's requests."""
import numpy as np
import pytest
import torch

import paper_2601_21444_amd as apbv
from oracle import cache_oracle as co
from tests.test_gpu_cache import dev_int

pytestmark = pytest.mark.gpu

FEW = 4                  # tokens a request grows by at most


def decoding_step(rng, n, page, blocks, tight, leaving):
    """Lengths before and after, table, free list and count.  A third of the requests end a page or are about to; `leaving` of them
    leave or take tokens back; tight: too few free pages, and lengths that are none."""
    cap = blocks * page
    old = rng.integers(0, cap + 1, n)
    edge = rng.random(n) < 0.33
    old[edge] = np.minimum(old[edge] // page * page + rng.integers(-2, 1, edge.sum()) % page, cap)
    new = np.minimum(old + rng.integers(0, FEW + 1, n), cap)
    gone = rng.random(n) < leaving
    new[gone] = rng.integers(0, old[gone] + 1) * (rng.random(gone.sum()) < 0.5)
    if tight:
        new[rng.random(n) < 0.03] = -1
        full = rng.random(n) < 0.03
        old[full], new[full] = cap, cap + 1 + rng.integers(0, FEW, full.sum())
    had = -(-old // page)
    need = np.where((new >= 0) & (new <= cap), np.maximum(-(-np.maximum(new, 0) // page) - had, 0), 0)
    pool = rng.permutation(int(had.sum() + need.sum()) + 9)
    table, at = np.full((n, blocks), -9), 0
    for b in range(n):
        table[b, :had[b]] = pool[at:at + had[b]]
        at += had[b]
    count = int(need.sum() * (rng.uniform(0.2, 0.9) if tight else 1.0))
    free = list(pool[at:at + count]) + [-8] * (len(pool) - count)
    assert (new - old <= FEW).all()
    ints = lambda x: [int(y) for y in x]
    return ints(old), ints(new), [ints(x) for x in table], ints(free), count, int(np.maximum(new - old, 0).sum())


@pytest.mark.parametrize("leaving", [0.0, 0.2])
@pytest.mark.parametrize("tight", [False, True])
@pytest.mark.parametrize("n,page,blocks", [(1, 16, 3), (64, 64, 5), (65, 16, 9), (300, 128, 3), (1024, 16, 5), (1025, 16, 5), (4096, 32, 3)])
def test_decoding_steps_match_the_oracle(n, page, blocks, tight, leaving):
    rng = np.random.default_rng((51, n, page, tight, int(10 * leaving)))
    # room for the new tokens exactly, for some of them, for more than a workgroup's threads (outputs apart: several workgroups), for
    # more than one workgroup finds the slots of (in place: a second launch)
    for room in ("exact", "less", 3000, 9000):
        for in_place in (False, True):
            old, new, table, free, count, tokens = decoding_step(rng, n, page, blocks, tight, leaving)
            most = tokens if room == "exact" else (2 * tokens // 3 if room == "less" else tokens + room)
            print("decoding", n, page, blocks, tight, leaving, room, in_place, "new tokens", tokens, flush=True)
            args = dev_int(old), dev_int(new), dev_int(table), dev_int(free), dev_int([count])
            kw = dict(lengths_out=args[0], free_count_out=args[4]) if in_place else {}
            got = [x.tolist() for x in apbv.apbv_cache_map(*args, page, most, **kw)]
            torch.cuda.synchronize()
            want = co.cache_map(old, new, table, free, count, page, most)        # (table and free change in place)
            for name, g, w in zip(("lengths", "starts", "slots", "count"), got, list(want[:3]) + [[want[3]]]):
                assert g == w, name
            assert args[2].tolist() == table and args[3].tolist() == free


def test_a_decoding_server_over_many_steps():
    """1500 requests decode in place for more than a page of steps, some leaving and coming back as another: each page has one owner,
    and the slots are those of the oracle."""
    n, page, blocks, steps = 1500, 16, 6, 20
    rng = np.random.default_rng(52)
    n_pages = 5200
    table, free, count = [[-1] * blocks for _ in range(n)], list(range(n_pages)), n_pages
    lengths = [0] * n
    d_len, d_tab, d_free, d_count = dev_int(lengths), dev_int(table), dev_int(free), dev_int([count])
    starts, slots = dev_int([0] * (n + 1)), dev_int([0] * (FEW * n))
    for step in range(steps):
        grow = rng.integers(0, FEW + 1, n)
        leave = rng.random(n) < 0.03
        asked = [0 if g else min(x + int(y), blocks * page) for x, y, g in zip(lengths, grow, leave)]
        print("decoding server", step, flush=True)
        apbv.apbv_cache_map(d_len, dev_int(asked), d_tab, d_free, d_count, page, FEW * n, lengths_out=d_len, starts_out=starts, slots_out=slots,
                            free_count_out=d_count)
        lengths, want_starts, want_slots, count = co.cache_map(lengths, asked, table, free, count, page, FEW * n)
        assert d_len.tolist() == lengths and starts.tolist() == want_starts and slots.tolist() == want_slots and d_count.tolist() == [count]
        assert d_tab.tolist() == table and d_free.tolist() == free
    held = [p for b in range(n) for p in table[b][:-(-lengths[b] // page)]]
    assert sorted(held + free[:count]) == list(range(n_pages))
