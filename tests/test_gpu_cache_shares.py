"""Attention over the cache where a workgroup's share of the keys is long: many tiles a wave, pieces that go on through several waves
and workgroups, more parts than a wave joins at once.  What each call reaches is held against the rules of the cut on the CPU; outputs
are compared with a plain computation in 64 bits, as a whole (root mean square), which a lost or misplaced tile of keys would show."""
import os
import subprocess

import numpy as np
import pytest
import torch

import paper_2601_21444_amd as apbv
from oracle import cache_oracle as co
from tests.test_abi_host import ROOT, SANITIZE
from tests.test_gpu_cache import U, poisoned


def spread(n, lo, hi):
    return [round(lo * (hi / lo) ** (i / (n - 1))) for i in range(n)]


# name: query heads, KV heads, head_dim, page, [(queries, keys)], what the call is cut into: rows of a row tile, whether a workgroup
# takes it whole, waves that join a row, tiles of a share, the most parts of a row tile (whole: 0, its most tiles, its waves)
CASES = {
    # few rows: four waves take five tiles each, the join's waves 26 parts
    "one long request": (16, 2, 128, 64, [(1, 133120)], (16, 0, 4, 20, 104)),
    # four tiles a wave; the join's waves come round twice (49 and 59 parts of 64 elements, 59 of 128: 32 at a time)
    "one long request, small pages": (2, 1, 64, 16, [(1, 200000)], (16, 0, 4, 16, 196)),
    "one very long request": (8, 2, 64, 64, [(1, 600000)], (16, 0, 4, 40, 235)),
    "one long request of one head": (8, 1, 128, 128, [(1, 150001)], (16, 0, 4, 10, 235)),
    # spans, heads and tails in all waves, of requests that end anywhere in a share
    "a batch": (16, 4, 128, 64, [(1, k) for k in spread(64, 50, 10000)], (16, 0, 1, 16, 11)),
    "a batch, head_dim 64": (16, 4, 64, 32, [(1, k) for k in spread(64, 50, 10000)], (16, 0, 1, 16, 11)),
    "a batch of short blocks": (8, 2, 128, 64, [(5, k) for k in spread(30, 300, 9000)], (32, 0, 1, 10, 15)),
    "a batch of short blocks, head_dim 64": (8, 1, 64, 16, [(1 + i % 4, k) for i, k in enumerate(spread(40, 300, 9000))], (32, 0, 4, 7, 21)),
    # more requests than a wave has lanes: the join reads where they begin
    "many requests": (8, 2, 64, 32, [(1, k) for k in spread(200, 65, 6000)], (16, 0, 1, 17, 7)),
    # taken whole, eight tiles a wave
    "many requests, whole": (8, 2, 64, 16, [(1, k) for k in spread(100, 65, 2000)], (16, 1, 0, 32, 4)),
    "many requests, whole, head_dim 128": (16, 2, 128, 64, [(1 + i % 2, k) for i, k in enumerate(spread(100, 65, 2048))], (16, 1, 0, 32, 4)),
    # more rows: 9 to 22 tiles a share, which begin at odd and even tiles; parts joined by four waves and by one, in several passes
    "a query block": (16, 2, 128, 64, [(64, 16512)], (128, 0, 4, 9, 30)),
    "a query block of one head": (8, 1, 128, 64, [(70, 70017)], (128, 0, 4, 22, 51)),
    "a query block of one head, head_dim 64": (8, 1, 64, 32, [(70, 70017)], (128, 0, 4, 11, 101)),
    "a query block, one wave a row": (16, 1, 128, 64, [(70, 70017)], (128, 0, 1, 20, 56)),
    "chunks": (8, 2, 128, 32, [(256, 20001), (100, 17000), (256, 9999), (1, 20000)], (128, 0, 1, 21, 16)),
    "chunks, head_dim 64": (8, 2, 64, 128, [(256, 20001), (100, 17000), (256, 9999), (1, 20000)], (128, 0, 1, 21, 16)),
    "many blocks": (8, 2, 64, 32, [(9 + i % 40, 100 + 40 * i) for i in range(72)], (128, 0, 1, 10, 6)),
}


def table_blocks(page, requests):
    return -(-max(k for _, k in requests) // page)


def test_the_calls_are_cut_as_stated(tmp_path):
    exe = tmp_path / "cache_shares"
    incs = ["-I", os.path.join(ROOT, "paper_2601_21444_amd", "csrc"), "-I", os.path.join(ROOT, "include")]
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", *SANITIZE, *incs, os.path.join(ROOT, "tests", "host", "cache_shares.cpp"), "-o", str(exe)], check=True)
    lines = [" ".join(map(str, (hq, hkv, d, table_blocks(page, r) * page, len(r)) + sum(r, ()))) for hq, hkv, d, page, r, _ in CASES.values()]
    out = subprocess.run([str(exe)], input="\n".join(lines) + "\n", capture_output=True, text=True, check=True).stdout.splitlines()
    assert {name: tuple(map(int, o.split())) for name, o in zip(CASES, out)} == {name: c[-1] for name, c in CASES.items()}


# ---- the plain computation

def attend(q, k, v, scale, causal, there):
    """q [n, Hq, d], k and v [len, Hkv, d] float64, there [len] bool: out, lse, sum w |v|, and the largest scale * sum |q k|."""
    n, hq, d = q.shape
    length, hkv, _ = k.shape
    group = hq // hkv
    out, weighed = torch.zeros_like(q), torch.zeros_like(q)
    lse = torch.full((hq, n), -float("inf"), dtype=torch.float64, device=q.device)
    size = 0.0
    seen = torch.arange(length, device=q.device)[None, :] <= torch.arange(length - n, length, device=q.device)[:, None] if causal else \
        torch.ones(n, length, dtype=torch.bool, device=q.device)
    seen = seen & there
    for h in range(hq):
        kh, vh = k[:, h // group], v[:, h // group]
        s = (scale * (q[:, h] @ kh.T)).masked_fill(~seen, -float("inf"))
        size = max(size, float((scale * (q[:, h].abs() @ kh.abs().T)).max()))
        some = seen.any(1)
        lse[h, some] = torch.logsumexp(s[some], 1)
        w = torch.exp(s[some] - lse[h, some, None])
        out[some, h] = w @ vh
        weighed[some, h] = w @ vh.abs()
    return out, lse, weighed, size


def test_the_plain_computation_is_the_oracles():
    rng = np.random.default_rng(61)
    q, k, v = rng.standard_normal((5, 4, 16)), rng.standard_normal((9, 2, 16)), rng.standard_normal((9, 2, 16))
    for causal in (True, False):
        for keys, there in ((9, np.ones(9, bool)), (3, np.ones(3, bool)), (9, np.arange(9) % 4 != 1)):
            if causal and not there.all():
                continue
            ref, ref_lse, ref_weighed = co.attention(q, k[:keys][there], v[:keys][there], 0.3, causal)
            out, lse, weighed, _ = attend(*map(torch.from_numpy, (q, k[:keys], v[:keys])), 0.3, causal, torch.from_numpy(there))
            for a, b in ((out, ref), (lse, ref_lse), (weighed, ref_weighed)):
                np.testing.assert_allclose(a.numpy(), b, rtol=1e-12, atol=1e-13)


# ---- the calls
#
# Bounds.  (1) Of every output: that of test_gpu_cache.py, u (sum w |v| + 2 |out|) with u = 2^-8 half a step of bf16.  (2) Of the whole:
# the weights' rounding errors e, relative, have a root mean square below 2^-8 / sqrt(3) * sqrt(0.54) = 0.42 u (uniform in a step, 0.54
# the mean of 1 / m^2 over mantissas m), the output's likewise.  Values are independent of mean zero, so out is sum w v with mean
# square sum w^2 and its error sum w e (v - out) has 0.42 u of its root: 0.42 u sqrt(2) = 0.60 u together, whatever the number of
# keys.  Asserted: u.  Sixteen of 133120 keys that are lost leave an error of sqrt(16 / 133120) = 2.8 u.  (3) Of the lse: a logit's error, at
# most (d + 2) 2^-24 of scale * sum |q k|; a sum's, 2^-24 for each term that a lane adds (32 a tile at most) and each part; 2^-24 of the
# exponentials, the joins' weights and the tree over lanes (64 together).

def held(seed, hkv, d, page, blocks):
    """Rows of every slot but a few, and the pages of a table in order: (cache, pages, K, V of these pages in float64)."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    n_pages = blocks + 3
    c = poisoned(n_pages, hkv, d, page)
    pages = torch.randperm(n_pages, generator=g, device="cuda")[:blocks]
    at = torch.arange(blocks * page, device="cuda")
    slots = (pages[at // page] * page + at % page).int()
    rows = [torch.randn((blocks * page, hkv, d), generator=g, device="cuda").bfloat16() for _ in "kv"]
    apbv.apbv_cache_store(c, *rows, slots)
    k, v = apbv.apbv_cache_load(c, slots)
    return c, pages, k.double(), v.double(), g


@pytest.mark.gpu
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("name", CASES)
def test_long_shares(name, causal):
    hq, hkv, d, page, requests, (_, _, _, share, parts) = CASES[name]
    print(name, "causal" if causal else "all keys", flush=True)
    blocks = table_blocks(page, requests)
    c, pages, k, v, g = held(len(name), hkv, d, page, blocks)
    # the requests share the pages, each from another one on; without the causal limit some pages are not there
    shift = [(7 * b) % blocks for b in range(len(requests))]
    table = torch.stack([pages.roll(-s) for s in shift]).int()
    if not causal:
        for b in range(len(requests)):
            for i in range(3 + b % 5, blocks, 41):
                table[b, i] = (-1, c.n_pages, 2 ** 31 - 1)[i % 3]
    rows = sum(q for q, _ in requests)
    starts = [sum(q for q, _ in requests[:b]) for b in range(len(requests) + 1)]
    q = torch.randn((rows + 1, hq, d), generator=g, device="cuda").bfloat16()
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    out = torch.full((rows + 1, hq, d), 77.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((hq, rows + 1), 77.0, device="cuda")
    args = (q, c, table, ints([n for _, n in requests]), d ** -0.5)
    kw = dict(q_starts=ints(starts), max_q=max(n for n, _ in requests), causal=causal)
    apbv.apbv_cache_attention(*args, out=out, lse_out=lse, **kw)
    again = torch.full_like(out, 77.0)
    apbv.apbv_cache_attention(*args, out=again, **kw)                    # without the log-sum-exp: the same outputs
    torch.cuda.synchronize()
    assert torch.equal(out, again) and (out[rows:] == 77.0).all() and (lse[:, rows:] == 77.0).all() and torch.isfinite(out).all()
    worst = [0.0, 0.0, 0.0]
    for b, (n, keys) in enumerate(requests):
        order = (torch.arange(keys, device="cuda") + shift[b] * page) % (blocks * page)
        there = (table[b, torch.arange(keys, device="cuda") // page].long() % 2 ** 32) < c.n_pages
        lo, hi = starts[b], starts[b + 1]
        ref, ref_lse, weighed, size = attend(q[lo:hi].double(), k[order], v[order], d ** -0.5, causal, there)
        err = out[lo:hi].double() - ref
        worst[0] = max(worst[0], float((err.abs() / (1.02 * U * (weighed + 2 * ref.abs()) + 1e-3 * weighed + 1e-30)).max()))
        worst[1] = max(worst[1], float(err.norm() / ref.norm()) / U)
        bound = 2.0 ** -24 * ((d + 2) * size + 32 * share + parts + 64) + 2.0 ** -23 * ref_lse.abs()
        worst[2] = max(worst[2], float(((lse[:, lo:hi].double() - ref_lse).abs() / bound).max()))
    print("of the bounds: each output %.3f, all of a request %.3f, lse %.3f" % tuple(worst), flush=True)
    assert max(worst) <= 1.0
