"""Attention of requests that share cached prefixes, on the GPU against the fp64 oracle.  The bounds are those of the cache's attention
(test_gpu_cache.py): the parts of a row are joined in float32, which adds 2^-24 a part and none of the roundings counted there."""
import itertools
import math

import numpy as np
import pytest
import torch

import paper_2601_21444_amd as apbv
from oracle import cache_oracle as co
from tests.test_gpu_cache import Batch, check, dev_int

pytestmark = pytest.mark.gpu


class Shared:
    """Groups of (prefix, [(queries, own keys) of its requests]) in one poisoned cache; `alone`: requests of no group, in front and behind."""

    def __init__(self, rng, hq, hkv, d, page, groups, alone=((), ()), lead=0, tail=0, **kw):
        self.requests = [*alone[0], *(r for _, rs in groups for r in rs), *alone[1]]
        self.prefixes = [p for p, _ in groups]
        self.x = Batch(rng, hq, hkv, d, page, [(0, p) for p in self.prefixes] + self.requests, lead=lead, tail=tail, **kw)
        self.g = len(groups)
        self.members = [len(alone[0])]
        for _, rs in groups:
            self.members.append(self.members[-1] + len(rs))
        self.starts = self.x.starts[self.g:]
        self.of = [next((g for g in range(self.g) if self.members[g] <= b < self.members[g + 1]), None) for b in range(len(self.requests))]

    def args(self, wide=False):
        """wide: the tables have room for longer prefixes and requests, so that the call is cut and parts are joined; so many keys that
        row tiles are as high as the rows fill."""
        room = 5000 if wide is True else wide
        table = np.concatenate((self.x.table, np.full((len(self.x.table), room // self.x.page), -1)), 1) if wide else self.x.table
        return (dev_int(table[:self.g].tolist()), dev_int(self.prefixes), dev_int(table[self.g:].tolist()), dev_int([k for _, k in self.requests]))

    def run(self, causal=True, args=None, wide=False, **kw):
        x = self.x
        out = torch.full((x.rows, x.hq, x.d), 77.0, dtype=torch.bfloat16, device="cuda")
        lse = torch.full((x.hq, x.rows), 77.0, device="cuda")
        kw.setdefault("group_starts", dev_int(self.members))
        kw.setdefault("q_starts", dev_int(self.starts))
        kw.setdefault("max_q", max(n for n, _ in self.requests))
        pt, pl, t, l = args or self.args(wide)
        apbv.apbv_cache_shared_attention(x.q, x.cache, pt, pl, t, l, x.scale, causal=causal, out=out, lse_out=lse, **kw)
        torch.cuda.synchronize()
        again = torch.full_like(out, 77.0)                            # without the log-sum-exp: the same outputs
        apbv.apbv_cache_shared_attention(x.q, x.cache, pt, pl, t, l, x.scale, causal=causal, out=again, **kw)
        assert torch.equal(out.view(torch.int16), again.view(torch.int16))
        return out, lse

    def reference(self, b, causal, kept=None):
        """Of request b; kept(table row, keys) -> which of its keys are there."""
        x, (n, own) = self.x, self.requests[b]
        lo, at = self.starts[b], self.g + b
        kept = kept or (lambda row, keys: np.ones(keys, bool))
        parts = [(self.of[b], self.prefixes[self.of[b]])] if self.of[b] is not None else []
        pk, pv = (np.concatenate([y[r][kept(r, m)] for r, m in parts] or [np.zeros((0, x.hkv, x.d))]) for y in (x.k, x.v))
        out, lse, spread = np.zeros((n, x.hq, x.d)), np.zeros((x.hq, n)), np.zeros((n, x.hq, x.d))
        here = kept(at, own)
        for i in range(n):
            seen = min(max(own - n + i + 1, 0), own) if causal else own
            k, v = (np.concatenate((p, y[at][:seen][here[:seen]])) for p, y in ((pk, x.k), (pv, x.v)))
            o, l, s = co.attention(x.qv[lo + i:lo + i + 1], k, v, x.scale, False)
            out[i], lse[:, i], spread[i] = o[0], l[:, 0], s[0]
        return out, lse, spread

    def check(self, out, lse, causal=True, what="", only=None, kept=None):
        for b in only if only is not None else range(len(self.requests)):
            lo, hi = self.starts[b], self.starts[b + 1]
            check(out[lo:hi], lse[:, lo:hi], *self.reference(b, causal, kept), f"{what} request {b} {self.requests[b]}")
        for rows in (slice(0, self.starts[0]), slice(self.starts[-1], self.x.rows)):
            assert (out[rows] == 77.0).all() and (lse[:, rows] == 77.0).all()


CASES = [
    # hq, hkv, d, page, [(prefix, [(queries, own keys)])], requests of no group
    (2, 1, 64, 16, [(1, [(1, 1)])], ((), ())),
    (2, 1, 64, 16, [(700, [(1, 3), (1, 40)])], ((), ())),
    (2, 2, 128, 64, [(64, [(1, 64), (1, 63), (1, 65), (1, 0)])], ((), ())),
    (8, 2, 128, 16, [(1000, [(1, 1), (1, 17), (1, 700)]), (0, [(1, 5)]), (15, [(1, 0), (1, 16)])], ((), ())),
    (28, 4, 128, 64, [(3001, [(1, 5), (1, 1000), (1, 64), (1, 2)])], ((), ())),                    # 28 rows a KV head
    (16, 2, 128, 128, [(5000, [(1, 33)] * 9)], ((), ())),                                          # 72: tiles of 128 rows
    (28, 4, 128, 64, [(2000, [(1, 1 + 37 * i) for i in range(23)])], ((), ())),                    # two tiles of rows
    (8, 2, 64, 32, [(1500, [(1, 100), (1, 7)] * 9), (333, [(1, 50)]), (64, [(1, 1)] * 20)], (((1, 70),), ((1, 9), (1, 300)))),
    (8, 8, 128, 64, [(700, [(1, 300)] * 40)], ((), ())),
    (33, 1, 64, 16, [(400, [(1, 77), (1, 30)])], ((), ())),                                        # more heads than a row tile
    (16, 2, 64, 256, [(513, [(2, 30), (1, 1), (0, 300), (4, 26)]), (100, []), (260, [(3, 3)])], ((), ())),       # unequal rows, none, no requests
    (4, 2, 128, 16, [(0, [(3, 2), (5, 0)]), (20, [(3, 2), (5, 0), (2, 1)])], (((4, 1),), ((1, 0),))),      # rows that see no key, or no own key
    (28, 4, 128, 64, [(1111, [(7, 48), (30, 100), (48, 48), (11, 300)])], ((), ())),               # questions of many tokens
    (8, 2, 64, 32, [(640, [(130, 200), (1, 3)]), (65, [(40, 333), (33, 33)])], ((), ())),
    (2, 2, 128, 16, [(333, [(200, 260)])], ((), ())),
    (1, 1, 128, 64, [(6000, [(1, 4000)])], ((), ())),                                              # one row over both
]


@pytest.mark.parametrize("wide", [False, True, 600000])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_matches_the_oracle(case, causal, wide):
    hq, hkv, d, page, groups, alone = CASES[case]
    print("shared", CASES[case], causal, wide, flush=True)
    s = Shared(np.random.default_rng((31, case)), hq, hkv, d, page, groups, alone, lead=case % 3, tail=case % 2 * 3)
    out, lse = s.run(causal, wide=wide)
    s.check(out, lse, causal, f"case {case} causal={causal}")
    again, lse_again = s.run(causal, wide=wide)
    assert torch.equal(out.view(torch.int16), again.view(torch.int16)) and torch.equal(lse, lse_again)
    # max_q changes how the work is cut, not what is computed
    for max_q in (s.x.rows + 1, 0):
        more, lse_more = s.run(causal, wide=wide, max_q=max_q)
        s.check(more, lse_more, causal, f"case {case} causal={causal} max_q={max_q}")


@pytest.mark.parametrize("groups,each,queries", [(3, 4, 1), (1, 5, 1), (2, 3, 13), (5, 1, 2)])
def test_equal_groups_without_starts(groups, each, queries):
    rng = np.random.default_rng((32, groups))
    s = Shared(rng, 8, 2, 128, 32, [(100 + 90 * g, [(queries, queries + 17 * i) for i in range(each)]) for g in range(groups)])
    for wide in (False, True):
        out, lse = s.run(group_starts=None, q_starts=None, max_q=None, wide=wide)
        s.check(out, lse, True, "equal groups")


@pytest.mark.parametrize("n_groups,n", [(1, 100), (3, 200), (80, 90), (70, 300)])
def test_many_requests_and_groups(n_groups, n):
    """More of either than a wave has lanes, some without keys, some groups without requests."""
    rng = np.random.default_rng((33, n))
    sizes = np.bincount(rng.integers(0, n_groups, n), minlength=n_groups)
    groups = [(int(rng.choice([0, 16, 65, int(rng.integers(1, 400))])), [(1, int(rng.choice([0, 1, 64, int(rng.integers(1, 200))]))) for _ in range(m)]) for m in sizes]
    print("many", n_groups, n, flush=True)
    s = Shared(rng, 4, 2, 64, 16, groups, (((1, 10),), ((1, 0),)))
    for wide in (False, True, 600000):
        out, lse = s.run(wide=wide)
        s.check(out, lse, True, "many")


@pytest.mark.parametrize("queries", [1, 9])
def test_short_groups_of_any_size(queries):
    """Few enough keys for one launch, groups of none to ten requests, and requests of no group on both sides."""
    rng = np.random.default_rng((49, queries))
    sizes = [0, 10, 1, 1, 0, 3, 7, 2, *(int(m) for m in rng.integers(0, 5, 100)), 0, 0, 5]
    groups = [(int(rng.integers(0, 100)), [(int(rng.integers(0, queries + 1)), int(rng.integers(0, 100))) for _ in range(m)]) for m in sizes]
    print("short", queries, len(sizes), sum(sizes), flush=True)
    s = Shared(rng, 4, 2, 64, 16, groups, (((1, 10),) * 3, ((1, 0), (2, 70))), lead=2, tail=3)
    assert s.args()[0].shape[1] * 16 <= 128                           # two tiles each
    out, lse = s.run()
    s.check(out, lse, True, "short")


def test_requests_of_one_group_in_many_windows():
    """Rows of a tile that are of requests far apart, with requests of no rows between them."""
    rng = np.random.default_rng(45)
    requests = [(int(rng.random() < 0.1), int(rng.integers(0, 60))) for _ in range(400)]
    s = Shared(rng, 2, 2, 64, 16, [(100, requests), (30, [(3, 40)])], (((0, 5),) * 70 + ((1, 9),), ((2, 17),)))
    for wide in (False, True, 600000):
        out, lse = s.run(wide=wide)
        s.check(out, lse, True, "windows")


@pytest.mark.parametrize("n_groups", [1, 130, 4096])
def test_as_many_requests_as_there_may_be(n_groups):
    rng = np.random.default_rng((46, n_groups))
    members = np.diff(np.concatenate(([0], np.sort(rng.integers(0, 4097, n_groups - 1)), [4096])))
    print("4096 requests", n_groups, flush=True)
    s = Shared(rng, 2, 1, 64, 16, [(int(rng.integers(0, 100)), [(int(rng.random() < 0.8), int(rng.integers(0, 60))) for _ in range(m)]) for m in members])
    looked_at = sorted({0, 1, 63, 64, 4094, 4095, *(int(b) for b in rng.integers(0, 4096, 150))})
    for wide in (False, True):
        out, lse = s.run(wide=wide)
        s.check(out, lse, True, "4096", only=looked_at)
        # every request has been written
        assert torch.isfinite(out.float()).all() and (out.float().abs() < 20).all()


def test_more_rows_allowed_than_there_are():
    """max_q is a bound: the row tiles are those of 128 rows, the results the same to the rounding of the weights and the output."""
    s = Shared(np.random.default_rng(47), 8, 2, 128, 64, [(3000, [(1, 300)] * 20 + [(2, 2)]), (65, [(1, 70)])])
    for wide in (False, True, 600000):
        out, lse = s.run(max_q=1000, wide=wide)
        s.check(out, lse, True, "max_q")


@pytest.mark.parametrize("queries", [1, 40])
def test_pages_beyond_32_bit_offsets(queries):
    """A pool of 5 GB: pages of a prefix and of requests whose bytes lie behind 2^32, the last one among them; cut, and in one launch."""
    hkv, hq, d, page, n_pages = 8, 16, 128, 256, 40000
    print("5 GB pool", queries, flush=True)
    c = apbv.apbv_cache_empty(n_pages, hkv, d, page)
    assert n_pages * c.k_codes.stride(0) > 2 ** 32
    rng = np.random.default_rng(48)
    pages = np.array([[n_pages - 1, 33000, 0, -1], [32767, -1, -1, -1], [39000, 32768, -1, -1]])
    keys = [3 * page - 5, 100, page + 77]
    rows = lambda *shape: torch.from_numpy(rng.standard_normal(shape)).bfloat16().cuda()
    held = []
    for row, n in zip(pages, keys):
        j = np.arange(n)
        slots = dev_int((row[j // page] * page + j % page).tolist())
        apbv.apbv_cache_store(c, rows(n, hkv, d), rows(n, hkv, d), slots)
        held.append([x.double().cpu().numpy() for x in apbv.apbv_cache_load(c, slots)])
    q = rows(2 * queries, hq, d)
    qv = q.double().cpu().numpy()
    for blocks in (4, 60):                                            # (with room for many keys the call is cut)
        table = dev_int(np.concatenate((pages, np.full((3, blocks - 4), -1)), 1).tolist())
        out, lse = apbv.apbv_cache_shared_attention(q, c, table[:1], dev_int(keys[:1]), table[1:], dev_int(keys[1:]), 0.088, return_lse=True)
        for b in range(2):
            at = slice(b * queries, (b + 1) * queries)
            ref, ref_lse, spread = co.attention(qv[at], *(np.concatenate((held[0][i], held[1 + b][i])) for i in range(2)), 0.088, True)
            check(out[at], lse[:, at], ref, ref_lse, spread, f"5 GB pool {blocks} {b}")


def test_long_prefixes_are_compared_as_a_whole():
    """The error of a request's rows stays within a step of bf16 in root mean square, which a few lost keys would exceed."""
    s = Shared(np.random.default_rng(34), 8, 1, 128, 64, [(40000, [(1, 500), (1, 3), (1, 64)] * 6)])
    out, lse = s.run()
    for b in (0, 7, 17):
        ref, ref_lse, spread = s.reference(b, True)
        got = out[s.starts[b]:s.starts[b + 1]].double().cpu().numpy()
        assert np.sqrt(((got - ref) ** 2).mean() / (ref ** 2).mean()) < 2.0 ** -8
        check(out[s.starts[b]:s.starts[b + 1]], lse[:, s.starts[b]:s.starts[b + 1]], ref, ref_lse, spread, "long")


def test_without_a_prefix_it_is_the_caches_attention():
    s = Shared(np.random.default_rng(35), 16, 2, 128, 64, [(0, [(1, 700), (3, 90), (1, 4000)])])
    out, lse = s.run()
    s.check(out, lse, True, "no prefix")
    want, want_lse = apbv.apbv_cache_attention(s.x.q, s.x.cache, s.args()[2], s.args()[3], s.x.scale, q_starts=dev_int(s.starts), max_q=3, return_lse=True)
    # both within half a step (of the weights, then of the output) of the same value
    assert torch.allclose(out.float(), want.float(), rtol=2.0 ** -7, atol=2.0 ** -6) and torch.allclose(lse, want_lse, atol=2e-3)


def test_peaked_logits():
    """One key, of the prefix or of the request, carries nearly all the weight."""
    for factor in (0.0, 8.0):
        s = Shared(np.random.default_rng((36, int(factor))), 8, 1, 128, 64, [(1500, [(1, 300)] * 3), (70, [(5, 600)])], k_scale=factor)
        s.x.qv *= 0.25
        s.x.q = (s.x.q.float() * 0.25).bfloat16()
        for wide in (False, True):
            out, lse = s.run(wide=wide)
            s.check(out, lse, True, f"keys of scale {factor}")


def test_keys_on_bad_pages_are_not_there():
    s = Shared(np.random.default_rng(37), 8, 2, 128, 32, [(300, [(1, 100), (2, 70)]), (32, [(1, 32)])])
    n_pages = s.x.cache.n_pages
    gone = [(0, 0, -1), (0, 5, n_pages), (1, 0, 2 ** 31 - 1), (2, 1, -2 ** 31), (3, 2, n_pages + 7), (4, 0, -5)]
    for row, i, page in gone:
        s.x.table[row, i] = page

    def kept(row, keys):
        keep = np.ones(keys, bool)
        for r, i, _ in gone:
            if r == row:
                keep[i * 32:(i + 1) * 32] = False
        return keep
    for wide in (False, True):
        out, lse = s.run(causal=False, wide=wide)
        s.check(out, lse, False, "bad pages", kept=kept)
    assert (out[s.starts[2]] == 0).all() and torch.isneginf(lse[:, s.starts[2]]).all()      # neither prefix nor own keys


def test_lengths_and_starts_out_of_range_are_cut_off():
    s = Shared(np.random.default_rng(38), 4, 2, 64, 16, [(64, [(2, 64)]), (48, [(3, 64)])], blocks=4)
    pt, pl, t, l = s.args()
    pl[0], l[1] = 10 ** 9, 10 ** 9                                    # the tables hold 64
    out, lse = s.run(args=(pt, pl, t, l), q_starts=dev_int([-4, 2, 900]), group_starts=dev_int([-7, 1, 50]))
    s.check(out, lse, True, "cut off")
    pl[:], l[:] = -5, -1
    out, lse = s.run(args=(pt, pl, t, l))
    assert (out == 0).all() and torch.isneginf(lse).all()


def test_tables_and_queries_of_other_strides_on_another_stream():
    s = Shared(np.random.default_rng(39), 8, 2, 128, 64, [(1111, [(1, 50)] * 7)])
    want, want_lse = s.run()
    pt, pl, t, l = s.args()
    wide_t = torch.full((t.shape[0], t.shape[1] + 9), -3, dtype=torch.int32, device="cuda")
    wide_t[:, 4:4 + t.shape[1]] = t
    wide_q = torch.full((s.x.rows, 2 * s.x.hq + 1, s.x.d + 8), 9.0, dtype=torch.bfloat16, device="cuda")
    wide_q[:, 3:3 + s.x.hq, :s.x.d] = s.x.q
    members, starts = dev_int(s.members), dev_int(s.starts)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    out, lse = apbv.apbv_cache_shared_attention(wide_q[:, 3:3 + s.x.hq, :s.x.d], s.x.cache, pt, pl, wide_t[:, 4:4 + t.shape[1]], l, s.x.scale,
                                                group_starts=members, q_starts=starts, max_q=1, return_lse=True, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(out, want) and torch.equal(lse, want_lse)


def test_graphs_that_share_a_workspace_and_lengths_that_grow():
    """Captured once, replayed as the requests grow; every replay is what an eager call gives."""
    ss = [Shared(np.random.default_rng((40, i)), 16, 2, 128, 64, g) for i, g in enumerate(([(900, [(1, 200)] * 5)], [(64, [(1, 100), (1, 64)]), (333, [(1, 90)])]))]
    nbytes = max(apbv.apbv_cache_shared_attention_workspace_bytes(s.g, len(s.requests), s.x.rows, 16, 2, 128, 1) for s in ss)
    ws = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    calls, graphs = [], []
    for s in ss:
        pt, pl, t, l = s.args()
        members, starts = dev_int(s.members), dev_int(s.starts)
        out = torch.zeros((s.x.rows, 16, 128), dtype=torch.bfloat16, device="cuda")
        call = lambda s=s, a=(pt, pl, t, l), members=members, starts=starts, out=out: apbv.apbv_cache_shared_attention(
            s.x.q, s.x.cache, *a, s.x.scale, group_starts=members, q_starts=starts, max_q=1, out=out, workspace=ws)
        call()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call()
        calls.append((out, l, pl, call))
        graphs.append(g)
    for rep in range(4):
        for _, l, pl, _ in calls:
            l.sub_(rep * 7)
            pl.sub_(rep)
        for (out, _, _, call), g in list(zip(calls, graphs))[::-1 if rep % 2 else 1]:
            ws.fill_(0xFF)
            g.replay()
            torch.cuda.synchronize()
            got = out.clone()
            out.fill_(5.0)
            call()
            assert torch.equal(out, got), rep


def test_calls_at_once_on_two_streams():
    ss = [Shared(np.random.default_rng((41, i)), 8, 2, 64, 32, [(1500 + i, [(1, 300)] * 12)]) for i in range(2)]
    want = [s.run()[0] for s in ss]
    args = [(s.args(), dev_int(s.members), dev_int(s.starts)) for s in ss]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = []
    for _ in range(5):
        for s, (a, members, starts), stream in zip(ss, args, streams):
            got.append(apbv.apbv_cache_shared_attention(s.x.q, s.x.cache, *a, s.x.scale, group_starts=members, q_starts=starts, max_q=1, stream=stream))
    torch.cuda.synchronize()
    assert all(torch.equal(g, w) for g, w in zip(got, itertools.cycle(want)))


def test_no_rows():
    s = Shared(np.random.default_rng(42), 8, 2, 64, 32, [(100, [(0, 3), (0, 0)])])
    out, lse = s.run()
    assert out.shape == (0, 8, 64) and lse.shape == (8, 0)


def test_questions_about_a_video_from_the_frames_to_the_answers():
    """A prefill's rows turned and stored once; questions appended and answered token after token, against the oracle of all of it."""
    from oracle import positions_oracle as po
    rng = np.random.default_rng(43)
    hq, hkv, d, page, frames, n = 8, 2, 128, 32, 300, 5
    axis = [i % 3 for i in range(d // 2)]
    inv_freq = torch.from_numpy((1e4 ** (-np.arange(d // 2) / (d // 2))).astype(np.float32)).cuda()
    weight = torch.from_numpy(1 + 0.2 * rng.standard_normal(d)).bfloat16().cuda()
    rotation = apbv.ApbvRotation(inv_freq, d, axis=axis, q_weight=weight, k_weight=weight)
    f64 = lambda t: t.double().cpu().numpy()
    rows = lambda m, h: torch.from_numpy(rng.standard_normal((m, h, d))).bfloat16().cuda()
    turned = lambda x, at: po.rotate(f64(x), at, f64(inv_freq), axis, False, f64(weight), np.float64(np.float32(1e-6)))[0]
    n_pages = 64
    cache = apbv.apbv_cache_empty(n_pages, hkv, d, page)
    table = dev_int([[0] * 12] * (n + 1))                             # row 0: the video
    free, count = dev_int(list(range(n_pages))), dev_int([n_pages])
    lengths = dev_int([0] * (n + 1))
    # the video
    lengths, starts, slots, count = apbv.apbv_cache_map(lengths, dev_int([frames] + [0] * n), table, free, count, page, frames)
    at = np.stack((np.arange(frames) // 60, np.arange(frames) // 10 % 6, np.arange(frames) % 10))
    k, v = rows(frames, hkv), rows(frames, hkv)
    apbv.apbv_cache_append(cache, None, k, v, slots, dev_int(at.tolist()), rotation)
    keys = [[turned(k, at)], *([] for _ in range(n))]
    values = [[f64(v)], *([] for _ in range(n))]
    held = lambda x: co.decode(*co.encode(np.concatenate(x))) if x else np.zeros((0, hkv, d))
    for step, grow in enumerate(([3, 1, 20, 7, 2], [1] * n, [1, 0, 1, 0, 1], [1] * n)):
        new = dev_int([frames] + [int(a) + g for a, g in zip(lengths.tolist()[1:], grow)])
        before = lengths.tolist()[1:]
        lengths, starts, slots, count = apbv.apbv_cache_map(lengths, new, table, free, count, page, sum(grow))
        pos = np.concatenate([20 + b + np.arange(g) for b, g in zip(before, grow)])
        q, k, v = rows(sum(grow), hq), rows(sum(grow), hkv), rows(sum(grow), hkv)
        qt = apbv.apbv_cache_append(cache, q, k, v, slots, dev_int(pos.tolist()), rotation)
        out = apbv.apbv_cache_shared_attention(qt, cache, table[:1], lengths[:1], table[1:], lengths[1:], d ** -0.5, q_starts=starts[1:], max_q=max(grow))
        lo, kt = 0, turned(k, np.stack([pos] * 3))
        for b, g in enumerate(grow):
            keys[1 + b].append(kt[lo:lo + g])
            values[1 + b].append(f64(v)[lo:lo + g])
            ref, _, spread = co.attention(f64(qt)[lo:lo + g], *(np.concatenate((held(x[0]), held(x[1 + b]))) for x in (keys, values)), d ** -0.5, True)
            check(out[lo:lo + g], None, ref, None, spread, f"step {step} question {b}")
            lo += g
    assert count.tolist()[0] == n_pages - 10 - sum(-(-x // page) for x in lengths.tolist()[1:])


def test_what_does_not_fit_is_refused():
    s = Shared(np.random.default_rng(44), 4, 2, 64, 16, [(64, [(1, 20)] * 3)])
    pt, pl, t, l = s.args()
    call = lambda q=s.x.q, pt=pt, pl=pl, t=t, l=l, **kw: apbv.apbv_cache_shared_attention(q, s.x.cache, pt, pl, t, l, 0.1, **kw)
    call()
    for error, kw in ((TypeError, dict(pl=pl.long())), (ValueError, dict(pt=pt[:0])), (ValueError, dict(pl=pl.cpu())), (ValueError, dict(group_starts=pl)),
                      (ValueError, dict(q_starts=pl)), (ValueError, dict(t=t[:2])), (ValueError, dict(l=l[:2])), (ValueError, dict(q=s.x.q[..., :32])),
                      (ValueError, dict(out=torch.empty(2, 4, 64, dtype=torch.bfloat16, device="cuda"))), (TypeError, dict(group_starts=[0, 3]))):
        with pytest.raises(error):
            call(**kw)
    for kw in (dict(workspace=torch.empty(256, dtype=torch.uint8, device="cuda")), dict(max_q=-1), dict(pt=pt.expand(2, -1).contiguous(), pl=pl.expand(2).contiguous())):
        with pytest.raises(apbv.ApbvError):                           # (three requests do not divide among two groups)
            call(**kw)
