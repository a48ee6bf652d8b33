"""The 4-bit key/value cache on the GPU against the fp64 oracle: rows and tables exactly, attention within bounds derived below."""
import itertools
import math

import numpy as np
import pytest
import torch

import paper_2601_21444_amd as apbv
from oracle import cache_oracle as co

pytestmark = pytest.mark.gpu

POISON = 0xFF            # the scale byte of no number: what no visible key names must not be seen


def dev_int(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def bf16(x):
    """float64 -> (bf16 tensor on the GPU, its values)."""
    t = torch.from_numpy(np.ascontiguousarray(x)).to(torch.bfloat16)
    return t.cuda(), t.double().numpy()


def to_f64(t):
    return t.detach().cpu().double().numpy()


def poisoned(n_pages, hkv, d, page):
    c = apbv.apbv_cache_empty(n_pages, hkv, d, page)
    for t in c:
        t.fill_(POISON)
    return c


# ---- rows

def rows_for(rng, n, hkv, d):
    """Magnitudes over many binades, exact ties, zeros and signed zeros, blocks that are all zero or all alike."""
    x = rng.standard_normal((n, hkv, d)) * 2.0 ** rng.integers(-20, 20, (n, hkv, d // 32)).repeat(32, -1)
    x[:, :, ::5] = rng.integers(-14, 15, x[:, :, ::5].shape) / 4.0
    x[rng.random(x.shape) < 0.05] = 0.0
    x[rng.random(x.shape) < 0.02] = -0.0
    x[:, 0, :32] = rng.choice([0.0, 1.0, 7.0, 7.03125, 5.0, 2.0 ** -130, 3e38, 2.0 ** -126], (n, 1))
    return x


@pytest.mark.parametrize("d,hkv,page,n", [(64, 1, 16, 1), (128, 2, 16, 33), (64, 3, 32, 100), (128, 4, 64, 257), (128, 1, 128, 300), (64, 8, 256, 513)])
def test_rows_are_held_exactly_as_defined(d, hkv, page, n):
    rng = np.random.default_rng((1, d, hkv, page, n))
    print("rows", d, hkv, page, n, flush=True)
    n_pages = -(-n // page) + 3
    c = poisoned(n_pages, hkv, d, page)
    # K and V as slices of one wider projection: strides other than the dense ones
    x = rows_for(rng, n, 2 * hkv + 1, d)
    both, val = bf16(x)
    slots = rng.permutation(n_pages * page)[:n]
    slots[rng.random(n) < 0.1] = -1
    if n > 5:
        slots[1], slots[2], slots[3] = n_pages * page, -7, 2 ** 31 - 1
    live = (slots >= 0) & (slots < n_pages * page)
    before = [t.clone() for t in c]
    assert apbv.apbv_cache_store(c, both[:, :hkv], both[:, hkv + 1:], dev_int(slots)) is c
    k, v = apbv.apbv_cache_load(c, dev_int(slots))
    torch.cuda.synchronize()
    for name, t, scales, want, got in (("k", c.k_codes, c.k_scales, val[:, :hkv], k), ("v", c.v_codes, c.v_scales, val[:, hkv + 1:], v)):
        codes, sc = co.encode(want)
        at = slots[live]
        held = co.unpack(t.cpu().numpy()[at // page, :, at % page])
        assert np.array_equal(scales.cpu().numpy()[at // page, :, at % page], sc[live]), name
        # (a negative number that is held as zero may or may not keep its sign)
        zero = (codes[live] & 7) == 0
        assert np.array_equal(held[~zero], codes[live][~zero]) and ((held[zero] & 7) == 0).all(), name
        exact = np.where(live[:, None, None], co.decode(codes, sc), 0.0)
        assert np.array_equal(to_f64(got), exact), name
    # every other slot is as it was
    touched = torch.zeros(n_pages, page, dtype=torch.bool)
    touched[slots[live] // page, slots[live] % page] = True
    for t, b in zip(c, before):
        same = (t == b).all(-1).all(1).cpu()
        assert same[~touched].all()


def test_infinities_and_nan_leave_finite_rows():
    x = torch.randn(4, 1, 64)
    x[0, 0, 3], x[1, 0, 40], x[2, 0, 5], x[3, 0, :] = math.inf, -math.inf, math.nan, math.nan
    t = x.to(torch.bfloat16).cuda()
    c = poisoned(1, 1, 64, 16)
    apbv.apbv_cache_store(c, t, t, dev_int([0, 1, 2, 3]))
    k, v = apbv.apbv_cache_load(c, dev_int([0, 1, 2, 3]))
    want = co.decode(*co.encode(t.cpu().double().numpy()))
    assert np.array_equal(to_f64(k), want) and np.array_equal(to_f64(v), want) and np.isfinite(want).all()
    assert want[0, 0, 3] > 2.0 ** 127 and want[2, 0, 5] == 0


def test_rows_of_interleaved_layers_and_a_slot_read_twice():
    """Pages of three layers, K beside V, in one allocation; only the named layer's bytes change."""
    hkv, d, page, n = 2, 128, 32, 70
    whole = torch.full((4, 3, 2, hkv, page, d // 2), POISON, dtype=torch.uint8, device="cuda")
    scales = torch.full((4, 3, 2, hkv, page, d // 32), POISON, dtype=torch.uint8, device="cuda")
    c = apbv.ApbvCache(whole[:, 1, 0], whole[:, 1, 1], scales[:, 1, 0], scales[:, 1, 1])
    rng = np.random.default_rng(3)
    k, kv = bf16(rng.standard_normal((n, hkv, d)))
    v, vv = bf16(rng.standard_normal((n, hkv, d)))
    slots = rng.permutation(4 * page)[:n]
    apbv.apbv_cache_store(c, k, v, dev_int(slots))
    twice = np.concatenate((slots, slots[::-1], slots[:1]))
    gk, gv = apbv.apbv_cache_load(c, dev_int(twice))
    order = np.concatenate((np.arange(n), np.arange(n)[::-1], [0]))
    assert np.array_equal(to_f64(gk), co.decode(*co.encode(kv))[order]) and np.array_equal(to_f64(gv), co.decode(*co.encode(vv))[order])
    assert (whole[:, 0] == POISON).all() and (whole[:, 2] == POISON).all() and (scales[:, 0] == POISON).all() and (scales[:, 2] == POISON).all()


def test_no_rows_do_nothing():
    c = poisoned(2, 1, 64, 16)
    e = torch.empty((0, 1, 64), dtype=torch.bfloat16, device="cuda")
    apbv.apbv_cache_store(c, e, e, dev_int([]))
    k, v = apbv.apbv_cache_load(c, dev_int([]))
    assert k.shape == (0, 1, 64) and v.shape == (0, 1, 64) and all((t == POISON).all() for t in c)


# ---- tables

def random_step(rng, n, page, blocks, tight):
    cap = blocks * page
    old = rng.integers(0, cap + 1, n) * (rng.random(n) < 0.8)
    kind = rng.random(n)
    new = np.where(kind < 0.5, old + 1, np.where(kind < 0.7, rng.integers(0, cap + 1, n), np.where(kind < 0.85, old, 0)))
    if tight:                                    # lengths that are none, and requests that do not fit
        new[rng.random(n) < 0.1] = -3
        new[rng.random(n) < 0.1] = cap + 5
        new[rng.random(n) < 0.02] = 2 ** 31 - 1
        old[rng.random(n) < 0.05] = -2
        old[rng.random(n) < 0.05] = cap + 9
    else:
        new = np.minimum(new, cap)
    had = -(-np.clip(old, 0, cap) // page)
    pool = rng.permutation(int(had.sum()) + n * blocks + 5)
    table, at = [], 0
    for h in had:
        table.append(list(pool[at:at + h]) + [-9] * (blocks - h))
        at += h
    free = list(pool[at:])
    grown = np.clip(new.astype(np.int64) - np.clip(old, 0, cap), 0, None)
    need = np.where(new <= cap, np.clip(-(-new // page) - had, 0, None), 0)
    count = int(need.sum())
    most = int(grown[grown < 2 ** 30].sum())
    if tight:
        count, most = int(count * rng.uniform(0.2, 1.2)), int(most * rng.uniform(0.3, 1.2))
    count = min(count, len(free))
    free = free[:count] + [-8] * (len(pool) - count)
    return [int(x) for x in old], [int(x) for x in new], [[int(y) for y in x] for x in table], [int(x) for x in free], count, most


@pytest.mark.parametrize("tight", [False, True])
@pytest.mark.parametrize("n,page,blocks", [(1, 16, 1), (1, 64, 300), (3, 32, 7), (64, 64, 40), (65, 16, 9), (300, 128, 5), (1025, 16, 12), (4096, 16, 3), (7, 256, 200)])
def test_map_matches_the_oracle(n, page, blocks, tight):
    rng = np.random.default_rng((2, n, page, blocks, tight))
    for trial in range(3):
        old, new, table, free, count, most = random_step(rng, n, page, blocks, tight)
        print("map", n, page, blocks, tight, trial, "new tokens", most, flush=True)
        args = dev_int(old), dev_int(new), dev_int(table), dev_int(free), dev_int([count])
        got = apbv.apbv_cache_map(*args, page, most)
        torch.cuda.synchronize()
        want = co.cache_map(old, new, table, free, count, page, most)        # (table and free change in place)
        for name, g, w in zip(("lengths", "starts", "slots", "count"), got, want[:3] + ([want[3]],)):
            assert g.tolist() == w, name
        assert args[2].tolist() == table and args[3].tolist() == free
        assert args[0].tolist() == old and args[1].tolist() == new and args[4].tolist() == [count]


@pytest.mark.parametrize("alias", ["lengths", "count", "both"])
@pytest.mark.parametrize("n,page,blocks", [(3, 32, 7), (64, 64, 40), (300, 128, 5), (4096, 16, 3), (7, 256, 200)])
def test_map_in_place_matches_the_oracle(n, page, blocks, alias):
    rng = np.random.default_rng((3, n, page, blocks))
    for tight in (False, True):
        old, new, table, free, count, most = random_step(rng, n, page, blocks, tight)
        print("map in place", n, page, blocks, tight, "new tokens", most, flush=True)
        args = dev_int(old), dev_int(new), dev_int(table), dev_int(free), dev_int([count])
        kw = {}
        if alias != "count":
            kw["lengths_out"] = args[0]
        if alias != "lengths":
            kw["free_count_out"] = args[4]
        got = [x.tolist() for x in apbv.apbv_cache_map(*args, page, most, **kw)]
        want = co.cache_map(old, new, table, free, count, page, most)
        assert got == list(want[:3]) + [[want[3]]] and args[2].tolist() == table and args[3].tolist() == free


def test_map_in_place_and_a_list_that_is_full():
    """lengths_out is old_lengths, free_count_out free_count; what is given back beyond the list's capacity is dropped."""
    old, new, table, free, count = [40, 0, 100], [0, 33, 101], [[1, 2, 3, 0, 0, 0, 0], [0] * 7, [4, 5, 6, 7, 8, 9, 10]], [30, 31], 1
    for out in ("new", "in place"):
        o, nl, t, f, c = dev_int(old), dev_int(new), dev_int(table), dev_int(free), dev_int([count])
        kw = dict(lengths_out=o, free_count_out=c) if out == "in place" else {}
        got = [x.tolist() for x in apbv.apbv_cache_map(o, nl, t, f, c, 16, 40, **kw)]
        tab, fr = [list(x) for x in table], list(free)
        want = co.cache_map(old, new, tab, fr, count, 16, 40)
        assert got == [want[0], want[1], want[2], [want[3]]] and t.tolist() == tab and f.tolist() == fr
        assert got[0] == [0, 0, 101]                                    # two free pages: 33 tokens need three
    # a strided table, and a pool count out of range
    wide = torch.full((3, 11), -1, dtype=torch.int32, device="cuda")
    wide[:, 2:9] = dev_int(table)
    got = apbv.apbv_cache_map(dev_int(old), dev_int(new), wide[:, 2:9], dev_int(free), dev_int([99]), 16, 0)
    assert got[0].tolist() == [0, 0, 100] and got[3].tolist() == [2] and got[2].numel() == 0
    assert (wide[:, :2] == -1).all() and (wide[:, 9:] == -1).all()


# ---- attention
#
# Bounds.  u = 2^-8 is half a step of bf16.  The kernel rounds each probability to bf16 (relative error up to u) and takes the
# row sum of the rounded ones, so the weights it applies are w_j (1 + e_j) / sum w (1 + e) with |e| <= u: the result is off by
# at most u * sum_j w_j |v_j - out| <= u * (sum_j w_j |v_j| + |out|) to first order (2 % allowed for the second), and the
# final rounding by u |out|.  Float32: logits of d products, |error| <= d * 2^-24 * scale * sum |q k|, which shifts a weight by
# as much again; with sum |q k| * scale below 60 here that is below 5e-4, for the sums over keys 2^-24 each: 1e-3 of
# sum w |v| covers both.  The lse is of the sum before the rounding: the same 1e-3, plus 1e-6 of its size.

U = 2.0 ** -8


def check(got, lse, ref, ref_lse, spread, what):
    if ref.size == 0:
        return
    got = to_f64(got)
    bound = 1.02 * U * (spread + 2 * np.abs(ref)) + 1e-3 * spread + 1e-30
    assert np.isfinite(got).all(), what
    worst = (np.abs(got - ref) / bound).max()
    print(f"{what}: error {worst:.3f} of the bound, rms {np.sqrt(((got - ref) ** 2).mean() / max((ref ** 2).mean(), 1e-300)):.2e}", flush=True)
    assert worst <= 1.0, what
    if lse is not None:
        lse = lse.cpu().double().numpy()
        none = np.isneginf(ref_lse)
        assert np.array_equal(np.isneginf(lse), none), what
        assert (np.abs(lse[~none] - ref_lse[~none]) <= 1e-3 + 1e-6 * np.abs(ref_lse[~none])).all(), what


class Batch:
    """Requests of given (queries, keys) in a poisoned cache with scattered pages."""

    def __init__(self, rng, hq, hkv, d, page, requests, blocks=None, lead=0, tail=0, k_scale=1.0):
        self.hq, self.hkv, self.d, self.page, self.requests = hq, hkv, d, page, requests
        need = [-(-k // page) for _, k in requests]
        blocks = blocks or max(need + [1]) + 1
        n_pages = sum(need) + 4
        pool = rng.permutation(n_pages)
        self.cache = poisoned(n_pages, hkv, d, page)
        # entries behind the keys name pages that do not exist, or exist and hold poison
        self.table = rng.choice([-1, n_pages, 2 ** 30, int(pool[-1])], (len(requests), blocks))
        self.k, self.v, at = [], [], 0
        for b, (_, keys) in enumerate(requests):
            self.table[b, :need[b]] = pool[at:at + need[b]]
            at += need[b]
            k, _ = bf16(rng.standard_normal((keys, hkv, d)) * k_scale)
            v, _ = bf16(rng.standard_normal((keys, hkv, d)))
            j = np.arange(keys)
            slots = self.table[b, j // page] * page + j % page
            if keys:
                apbv.apbv_cache_store(self.cache, k, v, dev_int(slots))
                k, v = apbv.apbv_cache_load(self.cache, dev_int(slots))
            self.k.append(to_f64(k))
            self.v.append(to_f64(v))
        self.starts = [lead]
        for n, _ in requests:
            self.starts.append(self.starts[-1] + n)
        self.rows = self.starts[-1] + tail
        self.q, self.qv = bf16(rng.standard_normal((self.rows, hq, d)))
        self.scale = 1.0 / math.sqrt(d)

    def lengths(self):
        return dev_int([k for _, k in self.requests])

    def run(self, causal=True, starts=True, wide=False, **kw):
        """wide: the table has room for longer requests, so that keys are cut among workgroups and parts joined."""
        out = torch.full((self.rows, self.hq, self.d), 77.0, dtype=torch.bfloat16, device="cuda")
        lse = torch.full((self.hq, self.rows), 77.0, device="cuda")
        if starts:
            kw.setdefault("q_starts", dev_int(self.starts))
            kw.setdefault("max_q", max(n for n, _ in self.requests))
        table = np.concatenate((self.table, np.full((len(self.requests), 5000 // self.page), -1)), 1) if wide else self.table
        apbv.apbv_cache_attention(self.q, self.cache, dev_int(table.tolist()), self.lengths(), self.scale, causal=causal, out=out, lse_out=lse, **kw)
        torch.cuda.synchronize()
        if "max_q" in kw and not causal:                    # without the log-sum-exp: the same outputs
            again = torch.full_like(out, 77.0)
            apbv.apbv_cache_attention(self.q, self.cache, dev_int(table.tolist()), self.lengths(), self.scale, causal=causal, out=again, **kw)
            assert torch.equal(out.view(torch.int16), again.view(torch.int16))
        return out, lse

    def check(self, out, lse, causal=True, what=""):
        for b, (n, keys) in enumerate(self.requests):
            lo, hi = self.starts[b], self.starts[b + 1]
            ref, ref_lse, spread = co.attention(self.qv[lo:hi], self.k[b], self.v[b], self.scale, causal)
            check(out[lo:hi], lse[:, lo:hi], ref, ref_lse, spread, f"{what} request {b} ({n} of {keys})")
        for rows in (slice(0, self.starts[0]), slice(self.starts[-1], self.rows)):
            assert (out[rows] == 77.0).all() and (lse[:, rows] == 77.0).all()


SHAPES = [
    # hq, hkv, d, page, [(queries, keys)]
    (2, 1, 64, 16, [(1, 1)]),
    (2, 1, 128, 16, [(1, 15), (1, 16), (1, 17), (1, 63), (1, 64), (1, 65)]),
    (8, 2, 64, 32, [(1, 700), (1, 0), (1, 31), (1, 2049), (1, 128)]),
    (28, 4, 128, 64, [(1, 1000), (1, 5), (1, 3001)]),
    (16, 2, 128, 128, [(1, 9000)]),                                                    # one long request over many workgroups
    (8, 8, 128, 64, [(1, 300 + 97 * i) for i in range(9)]),                            # a head each
    (33, 1, 64, 16, [(1, 400), (1, 77)]),                                              # more heads than a row tile
    (16, 2, 64, 256, [(2, 513), (1, 1), (0, 300), (4, 260)]),                          # rows of unequal number, none among them
    (4, 2, 128, 16, [(3, 2), (5, 0), (2, 1)]),                                         # rows that see no key
    (28, 4, 128, 64, [(64, 700), (1, 2000), (37, 37)]),                                # a prompt of its own, a chunk, a decoding request
    (8, 2, 64, 32, [(130, 1000), (300, 333)]),
    (2, 2, 128, 16, [(200, 260)]),
]


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("case", range(len(SHAPES)))
def test_attention_matches_the_oracle(case, causal, wide):
    hq, hkv, d, page, requests = SHAPES[case]
    print("attention", SHAPES[case], causal, wide, flush=True)
    x = Batch(np.random.default_rng((5, case)), hq, hkv, d, page, requests, lead=case % 3, tail=case % 2 * 3)
    out, lse = x.run(causal, wide=wide)
    x.check(out, lse, causal, f"case {case} causal={causal}")
    again, lse_again = x.run(causal, wide=wide)
    assert torch.equal(out.view(torch.int16), again.view(torch.int16)) and torch.equal(lse, lse_again)
    # max_q changes how the work is cut, not what is computed
    more, lse_more = x.run(causal, wide=wide, max_q=x.rows + 1)
    x.check(more, lse_more, causal, f"case {case} causal={causal}, a large max_q")
    fewer, lse_fewer = x.run(causal, wide=wide, max_q=0)
    x.check(fewer, lse_fewer, causal, f"case {case} causal={causal}, max_q too small")


@pytest.mark.parametrize("queries", [1, 3, 40])
def test_attention_of_equal_blocks_without_starts(queries):
    x = Batch(np.random.default_rng((6, queries)), 8, 2, 128, 32, [(queries, 64 * i + 41) for i in range(5)])
    print("equal blocks", queries, flush=True)
    for wide in (False, True):
        out, lse = x.run(starts=False, wide=wide)
        x.check(out, lse, True, f"{queries} each")


def test_many_requests():
    """More requests than a wave has lanes, most of them short, some without keys, some without rows."""
    rng = np.random.default_rng(7)
    requests = [(int(n), int(k)) for n, k in zip(rng.integers(0, 3, 333), rng.integers(0, 200, 333))]
    requests[200] = (1, 5000)
    x = Batch(rng, 4, 2, 64, 16, requests, tail=2)
    print("333 requests", flush=True)
    out, lse = x.run()
    x.check(out, lse, True, "many")
    x.requests[200], x.k[200], x.v[200] = (1, 1000), x.k[200][:1000], x.v[200][:1000]
    x.table = x.table[:, :63]                               # a short table
    out, lse = x.run()
    x.check(out, lse, True, "many, short")


@pytest.mark.parametrize("n", [65, 200, 1030])
@pytest.mark.parametrize("hq,hkv,d,most", [(2, 2, 64, 3), (8, 1, 64, 4), (6, 1, 128, 9)])      # tiles of 16, of 32 and of 128 rows
def test_many_requests_cut_among_workgroups(n, hq, hkv, d, most):
    """Keys cut (the table has room for long requests), requests without rows and without keys among them, then equal blocks."""
    rng = np.random.default_rng((23, n, hq, most))
    rows = rng.integers(0, most + 1, n)
    rows[n // 2] = most
    keys = np.where(rng.random(n) < 0.15, 0, rng.integers(1, 200, n))
    x = Batch(rng, hq, hkv, d, 16, [(int(a), int(b)) for a, b in zip(rows, keys)], lead=2, tail=1)
    out, lse = x.run(wide=True)
    x.check(out, lse, True, f"{n} requests")
    x = Batch(rng, hq, hkv, d, 16, [(most, int(b)) for b in keys])
    out, lse = x.run(starts=False, wide=True)
    x.check(out, lse, True, f"{n} requests of {most}")


def test_peaked_logits_and_growing_keys():
    """References move along the keys; one key carries nearly all the weight."""
    for factor in (0.0, 8.0):
        x = Batch(np.random.default_rng((8, int(factor))), 8, 1, 128, 64, [(1, 1500), (5, 600)], k_scale=factor)
        x.qv *= 0.25
        x.q = (x.q.float() * 0.25).bfloat16()
        for wide in (False, True):
            out, lse = x.run(wide=wide)
            x.check(out, lse, True, f"keys of scale {factor}")


def test_keys_on_bad_pages_are_not_there():
    """CPU: the oracle without those keys.  Every bad entry names no page, so nothing is read."""
    x = Batch(np.random.default_rng(9), 8, 2, 128, 32, [(1, 300), (2, 500), (1, 32)])
    n_pages = x.cache.n_pages
    gone = [(0, 0, -1), (0, 5, n_pages), (1, 15, -2 ** 31), (1, 3, 2 ** 31 - 1), (2, 0, n_pages + 7)]
    for b, i, page in gone:
        x.table[b, i] = page
    for wide, (b, (n, keys)) in itertools.product((False, True), enumerate(x.requests)):
        out, lse = x.run(causal=False, wide=wide)
        keep = np.ones(keys, bool)
        for bb, i, _ in gone:
            if bb == b:
                keep[i * 32:(i + 1) * 32] = False
        lo, hi = x.starts[b], x.starts[b + 1]
        ref, ref_lse, spread = co.attention(x.qv[lo:hi], x.k[b][keep], x.v[b][keep], x.scale, False)
        check(out[lo:hi], lse[:, lo:hi], ref, ref_lse, spread, f"request {b}")


def test_lengths_and_starts_out_of_range_are_cut_off():
    x = Batch(np.random.default_rng(10), 4, 2, 64, 16, [(2, 64), (3, 48)], blocks=4)
    lengths = x.lengths()
    lengths[0] = 10 ** 9                                    # the table holds 64
    out = torch.full((5, 4, 64), 77.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((4, 5), 77.0, device="cuda")
    apbv.apbv_cache_attention(x.q, x.cache, dev_int(x.table.tolist()), lengths, x.scale, q_starts=dev_int([-4, 2, 900]), max_q=3, out=out, lse_out=lse)
    x.check(out, lse, True, "cut off")
    lengths[0] = -5
    apbv.apbv_cache_attention(x.q, x.cache, dev_int(x.table.tolist()), lengths, x.scale, q_starts=dev_int([0, 2, 5]), max_q=3, out=out, lse_out=lse)
    assert (out[:2] == 0).all() and torch.isneginf(lse[:, :2]).all()


def test_queries_and_tables_of_other_strides_on_another_stream():
    x = Batch(np.random.default_rng(11), 8, 2, 128, 64, [(1, 1111), (6, 200)])
    want, want_lse = x.run()
    wide = torch.full((x.rows, 2 * x.hq + 1, x.d + 8), 9.0, dtype=torch.bfloat16, device="cuda")
    wide[:, 3:3 + x.hq, :x.d] = x.q
    table = torch.full((2, x.table.shape[1] + 5), -1, dtype=torch.int32, device="cuda")
    table[:, 2:2 + x.table.shape[1]] = dev_int(x.table.tolist())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for explicit in (True, False):
        with torch.cuda.stream(torch.cuda.current_stream() if explicit else side):
            out, lse = apbv.apbv_cache_attention(wide[:, 3:3 + x.hq, :x.d], x.cache, table[:, 2:2 + x.table.shape[1]], x.lengths(), x.scale,
                                                 q_starts=dev_int(x.starts), max_q=6, return_lse=True, stream=side if explicit else None)
        side.synchronize()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, want_lse)


def test_parts_of_a_request_on_several_hosts_are_merged():
    """Keys divided between two caches, no causal limit: apbv_merge_lse of the parts is the attention over all."""
    rng = np.random.default_rng(12)
    a, b = Batch(rng, 16, 2, 128, 64, [(3, 900)]), Batch(rng, 16, 2, 128, 64, [(3, 500)])
    b.q, b.qv = a.q, a.qv
    parts = [x.run(causal=False) for x in (a, b)]
    out, lse = apbv.apbv_merge_lse(torch.stack([p[0] for p in parts]), torch.stack([p[1] for p in parts]), return_lse=True)
    ref, ref_lse, spread = co.attention(a.qv, np.concatenate((a.k[0], b.k[0])), np.concatenate((a.v[0], b.v[0])), a.scale, False)
    bound = 1.02 * U * (spread + 3 * np.abs(ref)) + U * spread + 2e-3 * spread        # the parts are rounded to bf16 once more
    assert (np.abs(to_f64(out) - ref) <= bound).all()
    assert np.abs(lse.cpu().numpy() - ref_lse).max() <= U + 2e-3


def test_pages_beyond_32_bit_offsets():
    """A pool of 5 GB: pages whose bytes lie behind 2^32, the last one among them."""
    hkv, d, page, n_pages = 8, 128, 256, 40000
    c = apbv.apbv_cache_empty(n_pages, hkv, d, page)
    assert n_pages * c.k_codes.stride(0) > 2 ** 32
    print("5 GB pool", flush=True)
    rng = np.random.default_rng(13)
    pages = np.array([n_pages - 1, 33000, 0, 32767, 32768])
    n = 5 * page - 3
    j = np.arange(n)
    slots = pages[j // page] * page + j % page
    k, kv = bf16(rng.standard_normal((n, hkv, d)))
    v, vv = bf16(rng.standard_normal((n, hkv, d)))
    apbv.apbv_cache_store(c, k, v, dev_int(slots))
    gk, gv = apbv.apbv_cache_load(c, dev_int(slots))
    assert np.array_equal(to_f64(gk), co.decode(*co.encode(kv))) and np.array_equal(to_f64(gv), co.decode(*co.encode(vv)))
    q, qv = bf16(rng.standard_normal((1, 16, d)))
    out, lse = apbv.apbv_cache_attention(q, c, dev_int([list(pages)]), dev_int([n]), 0.088, return_lse=True)
    ref, ref_lse, spread = co.attention(qv, to_f64(gk), to_f64(gv), 0.088, True)
    check(out, lse, ref, ref_lse, spread, "5 GB pool")


def test_no_rows_of_attention():
    c = poisoned(2, 1, 64, 16)
    out = apbv.apbv_cache_attention(torch.empty((0, 2, 64), dtype=torch.bfloat16, device="cuda"), c, dev_int([[0]]), dev_int([5]), 0.1)
    assert out.shape == (0, 2, 64)


# ---- together

class Server:
    """A few requests that arrive, decode and leave; the oracle keeps every request's rows as they were given."""

    def __init__(self, n, hq, hkv, d, page, n_pages, blocks, max_new):
        self.hq, self.hkv, self.d, self.page, self.max_new = hq, hkv, d, page, max_new
        self.cache = poisoned(n_pages, hkv, d, page)
        self.table = torch.full((n, blocks), -1, dtype=torch.int32, device="cuda")
        self.free = torch.arange(n_pages, dtype=torch.int32, device="cuda")
        self.count = dev_int([n_pages])
        self.lengths = torch.zeros(n, dtype=torch.int32, device="cuda")
        self.asked = torch.zeros(n, dtype=torch.int32, device="cuda")
        i32 = lambda m: torch.zeros(m, dtype=torch.int32, device="cuda")
        self.starts, self.slots = i32(n + 1), i32(max_new)
        row = lambda h: torch.zeros((max_new, h, d), dtype=torch.bfloat16, device="cuda")
        self.q, self.k, self.v, self.out = row(hq), row(hkv), row(hkv), row(hq)
        self.lse = torch.zeros((hq, max_new), device="cuda")
        self.ws = torch.empty(apbv.apbv_cache_attention_workspace_bytes(n, max_new, hq, hkv, d, max_new), dtype=torch.uint8, device="cuda")

    def step(self):
        apbv.apbv_cache_map(self.lengths, self.asked, self.table, self.free, self.count, self.page, self.max_new,
                            lengths_out=self.lengths, starts_out=self.starts, slots_out=self.slots, free_count_out=self.count)
        apbv.apbv_cache_store(self.cache, self.k, self.v, self.slots)
        apbv.apbv_cache_attention(self.q, self.cache, self.table, self.lengths, self.d ** -0.5, q_starts=self.starts, max_q=self.max_new,
                                  out=self.out, lse_out=self.lse, workspace=self.ws)


@pytest.mark.parametrize("captured", [False, True])
def test_a_server_that_admits_decodes_and_releases(captured):
    """apbv_cache_map in place, store, attention, over steps in which requests arrive in chunks, decode, take tokens back and
    leave, the pool never large enough for all: run eagerly, and as one graph replayed with new lengths and rows each step."""
    n, hq, hkv, d, page, n_pages, blocks, max_new = 5, 8, 2, 128, 16, 30, 20, 96
    s = Server(n, hq, hkv, d, page, n_pages, blocks, max_new)
    rng = np.random.default_rng(14)
    graph = None
    if captured:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            s.step()                                       # nothing asked for: no state changes
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                s.step()
        torch.cuda.synchronize()
    keys, values = [np.zeros((0, hkv, d))] * n, [np.zeros((0, hkv, d))] * n
    plan = [[50, 0, 0, 7, 0], [51, 33, 0, 8, 0], [52, 34, 90, 0, 0], [53, 20, 91, 0, 64], [54, 21, 92, 95, 65], [0, 22, 93, 95, 66],
            [16, 23, 0, 95, 130], [17, 24, 200, 95, 131], [17, 400, 200, 0, 132], [18, 25, 201, 3, 0], [0, 0, 0, 0, 0]]
    refusals = 0
    for step, want in enumerate(plan):
        now = [len(x) for x in keys]
        grown = [max(w - o, 0) for w, o in zip(want, now)]
        q, qv = bf16(rng.standard_normal((max_new, hq, d)))
        k, kv = bf16(rng.standard_normal((max_new, hkv, d)))
        v, vv = bf16(rng.standard_normal((max_new, hkv, d)))
        for t, x in ((s.q, q), (s.k, k), (s.v, v), (s.asked, dev_int(want))):
            t.copy_(x)
        s.out.fill_(77.0)
        torch.cuda.synchronize()
        print("server step", step, captured, want, flush=True)
        graph.replay() if graph else s.step()
        torch.cuda.synchronize()
        got, starts, at = s.lengths.tolist(), s.starts.tolist(), 0
        for b in range(n):
            lo, hi = starts[b], starts[b + 1]
            assert lo == min(at, max_new) and hi == min(at + grown[b], max_new)
            at += grown[b]
            if got[b] != want[b]:
                assert got[b] == now[b] and (s.slots[lo:hi] == -1).all()
                refusals += 1
                continue
            keys[b] = np.concatenate((keys[b][:want[b]], co.decode(*co.encode(kv[lo:hi]))))
            values[b] = np.concatenate((values[b][:want[b]], co.decode(*co.encode(vv[lo:hi]))))
            ref, ref_lse, spread = co.attention(qv[lo:hi], keys[b], values[b], d ** -0.5, True)
            check(s.out[lo:hi], s.lse[:, lo:hi], ref, ref_lse, spread, f"step {step} request {b}")
        assert (s.out[min(at, max_new):] == 77.0).all()
        held = sum(-(-x // page) for x in got)
        assert s.count.item() == n_pages - held
        pages = [p for b in range(n) for p in s.table[b, :-(-got[b] // page)].tolist()] + s.free[:s.count.item()].tolist()
        assert sorted(pages) == list(range(n_pages))       # every page has one owner
    assert refusals >= 2 and s.count.item() == n_pages


def test_calls_at_once_on_two_streams():
    """Batches of both kernels, cut and joined, on two streams with a workspace each: as one after the other."""
    rng = np.random.default_rng(31)
    batches = [Batch(rng, 16, 2, 128, 64, [(1, 6000), (1, 300)]), Batch(rng, 8, 2, 64, 32, [(40, 3000), (70, 900)])]
    want = [x.run() for x in batches]
    calls = []
    for x in batches:
        n, most = len(x.requests), max(n for n, _ in x.requests)
        need = apbv.apbv_cache_attention_workspace_bytes(n, x.rows, x.hq, x.hkv, x.d, most)
        calls.append((x, dev_int(x.table.tolist()), x.lengths(), dev_int(x.starts), most, torch.empty(need, dtype=torch.uint8, device="cuda"),
                      torch.empty((x.rows, x.hq, x.d), dtype=torch.bfloat16, device="cuda"), torch.empty((x.hq, x.rows), device="cuda")))
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(5):
        for (x, table, lengths, starts, most, ws, out, lse), stream in zip(calls, streams):
            apbv.apbv_cache_attention(x.q, x.cache, table, lengths, x.scale, q_starts=starts, max_q=most, out=out, lse_out=lse, workspace=ws, stream=stream)
        torch.cuda.synchronize()
        for (_, _, _, _, _, _, out, lse), (o, l) in zip(calls, want):
            assert torch.equal(out, o) and torch.equal(lse, l)


def test_two_graphs_share_a_workspace():
    """Calls ordered on one stream may share it: each replay leaves what its own call gives."""
    xs = [Batch(np.random.default_rng((15, i)), 16, 2, 128, 64, r) for i, r in enumerate(([(1, 3333)], [(1, 200), (4, 999), (1, 2048)]))]
    nbytes = max(apbv.apbv_cache_attention_workspace_bytes(len(x.requests), x.rows, x.hq, x.hkv, x.d, 4) for x in xs)
    ws = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    calls, graphs = [], []
    for x in xs:
        t, l, st = dev_int(x.table.tolist()), x.lengths(), dev_int(x.starts)
        out = torch.zeros((x.rows, x.hq, x.d), dtype=torch.bfloat16, device="cuda")
        call = lambda x=x, t=t, l=l, st=st, out=out: apbv.apbv_cache_attention(x.q, x.cache, t, l, x.scale, q_starts=st, max_q=4, out=out, workspace=ws)
        call()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call()
        calls.append((out, out.clone(), call))            # (the call holds the tensors that the graph reads)
        graphs.append(g)
    for rep in range(3):
        for out, _, _ in calls:
            out.fill_(5.0)
        ws.fill_(0xFF)
        for g in graphs[::-1 if rep % 2 else 1]:
            g.replay()
        torch.cuda.synchronize()
        for out, want, _ in calls:
            assert torch.equal(out, want), rep


def test_the_binding_refuses_what_does_not_fit():
    x = Batch(np.random.default_rng(16), 4, 2, 64, 16, [(1, 20)])
    t, l = dev_int(x.table.tolist()), x.lengths()
    c = x.cache
    bad = [
        (ValueError, lambda: apbv.apbv_cache_attention(x.q[:, :, :32], c, t, l, 0.1)),
        (TypeError, lambda: apbv.apbv_cache_attention(x.q.float(), c, t, l, 0.1)),
        (TypeError, lambda: apbv.apbv_cache_attention(x.q, c, t.long(), l, 0.1)),
        (ValueError, lambda: apbv.apbv_cache_attention(x.q, c, t[:0], l, 0.1)),
        (ValueError, lambda: apbv.apbv_cache_attention(x.q, c, t, l.cpu(), 0.1)),
        (ValueError, lambda: apbv.apbv_cache_attention(x.q, c, t, l, 0.1, q_starts=dev_int([0]))),
        (ValueError, lambda: apbv.apbv_cache_attention(x.q, c, t, l, 0.1, out=x.q[:, :2].contiguous())),
        (ValueError, lambda: apbv.apbv_cache_attention(x.q, c._replace(v_scales=c.v_scales[:1]), t, l, 0.1)),
        (ValueError, lambda: apbv.apbv_cache_attention(x.q, c._replace(v_codes=c.v_codes.transpose(1, 2)), t, l, 0.1)),
        (TypeError, lambda: apbv.apbv_cache_attention(x.q, c._replace(k_codes=c.k_codes.view(torch.int8)), t, l, 0.1)),
        (apbv.ApbvError, lambda: apbv.apbv_cache_attention(x.q, c, t, l, -0.1)),
        (apbv.ApbvError, lambda: apbv.apbv_cache_attention(x.q, c, t, l, 0.1, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))),
        (apbv.ApbvError, lambda: apbv.apbv_cache_attention(x.q[:, :3].contiguous(), c, t, l, 0.1)),
        (ValueError, lambda: apbv.apbv_cache_store(c, x.q, x.q, dev_int([0]))),
        (ValueError, lambda: apbv.apbv_cache_store(c, x.q[:, :2], x.q[:, :2], dev_int([0, 1]))),
        (TypeError, lambda: apbv.apbv_cache_load(c, l.long())),
        (ValueError, lambda: apbv.apbv_cache_load(c, l, k_out=torch.empty(3, dtype=torch.bfloat16, device="cuda"))),
        (apbv.ApbvError, lambda: apbv.apbv_cache_map(l, l + 1, t, l, l, 24, 4)),
        (ValueError, lambda: apbv.apbv_cache_map(l, dev_int([1, 2]), t, l, l, 16, 4)),
        (ValueError, lambda: apbv.apbv_cache_map(l, l + 1, t, l, l, 16, 4, slots_out=dev_int([0, 0, 0]))),
        (TypeError, lambda: apbv.apbv_cache_map(l, l + 1, t, l, l, 16, 4.0)),
    ]
    for i, (error, call) in enumerate(bad):
        with pytest.raises(error):
            call()
            pytest.fail(f"call {i} was accepted")
