"""Norm and rotation of queries and keys, and appending to the cache, on the GPU against the oracle in 64 bits.

A turned element is a cos t - b sin t, normed before or not: float32 products and sums of at most 2^-24 each (scale, weight, cosine,
sine, product, sum: below 8 of them together, relative to |a cos t| + |b sin t|), and one rounding to bf16, half a step, 2^-8 of the
value.  Codes of the cache are held to those of the oracle's float64 values, exactly: both sides are some 2^-50 off, and a value that
near to a border between two codes does not occur in these inputs."""
import math

import numpy as np
import pytest
import torch

import paper_2601_21444_amd as apbv
from oracle import cache_oracle as co
from oracle import positions_oracle as po

pytestmark = pytest.mark.gpu


def bf16(x):
    return torch.from_numpy(np.ascontiguousarray(x, np.float32)).to("cuda").bfloat16()


def f64(t):
    return t.double().cpu().numpy()


def ints(x):
    return torch.from_numpy(np.ascontiguousarray(x, np.int32)).to("cuda")


def frequencies(rot, base=1e4):
    return torch.from_numpy((base ** (-np.arange(rot // 2) / (rot // 2))).astype(np.float32)).to("cuda")


class Case:
    """Inputs of a step: rows of a joint projection, positions on several axes, weights."""

    def __init__(self, tokens, hq, hkv, d, rot, axes=1, adjacent=False, norm=False, far=1000, seed=0, eps=1e-6, spread=1.0):
        rng = np.random.default_rng(seed)
        self.joint = bf16(rng.standard_normal((tokens, hq + 2 * hkv, d)) * np.exp(spread * rng.standard_normal((tokens, hq + 2 * hkv, 1))))
        self.q, self.k, self.v = self.joint[:, :hq], self.joint[:, hq:hq + hkv], self.joint[:, hq + hkv:]
        self.at = rng.integers(-far, far + 1, (axes, tokens))
        self.positions = ints(self.at)
        self.inv_freq = frequencies(rot)
        self.axis = [int(a) for a in rng.integers(0, axes, rot // 2)]
        self.axis[0] = axes - 1
        self.adjacent, self.eps = adjacent, eps
        self.wq, self.wk = (bf16(1.0 + 0.3 * rng.standard_normal(d)) if norm else None for _ in range(2))
        self.rotation = apbv.ApbvRotation(self.inv_freq, d, axis=self.axis, adjacent=adjacent, q_weight=self.wq, k_weight=self.wk, eps=eps)

    def want(self, x, w):
        return po.rotate(f64(x), self.at, f64(self.inv_freq), self.axis, self.adjacent, None if w is None else f64(w), np.float64(np.float32(self.eps)))


def check_rows(got, want):
    value, parts = want
    off = np.abs(f64(got) - value)
    bound = 2.0 ** -8 * np.abs(value) + 8 * 2.0 ** -24 * parts + 1e-40
    assert off.shape == bound.shape and (off <= bound).all(), (off / bound).max()


SHAPES = [
    # tokens, query heads, KV heads, head_dim, rot_dim
    (1, 2, 1, 64, 64), (1, 28, 4, 128, 128), (2, 1, 1, 128, 16), (3, 8, 2, 64, 32), (7, 33, 11, 64, 48), (17, 16, 2, 128, 96), (64, 28, 4, 128, 128),
    (65, 5, 5, 128, 64), (129, 130, 1, 128, 128), (300, 3, 1, 64, 64), (1000, 31, 4, 128, 112), (1100, 40, 8, 64, 64), (9, 300, 100, 64, 16),
]


@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("shape", SHAPES)
def test_rotate(shape, norm, adjacent):
    c = Case(*shape, axes=1 + shape[0] % 4, adjacent=adjacent, norm=norm, seed=shape[0])
    q, k = apbv.apbv_rotate(c.q, c.k, c.positions, c.rotation)
    check_rows(q, c.want(c.q, c.wq))
    check_rows(k, c.want(c.k, c.wk))


def test_far_positions():
    """Angles of a hundred thousand turns and more, where float32 holds none of the fraction."""
    for far in (300_000, 1 << 28):
        c = Case(40, 4, 2, 128, 128, axes=3, far=far, seed=far % 1000)
        q, k = apbv.apbv_rotate(c.q, c.k, c.positions, c.rotation)
        check_rows(q, c.want(c.q, None))
        check_rows(k, c.want(c.k, None))
    c = Case(2, 4, 2, 64, 64, far=5)
    c.at = np.array([[-(1 << 31), (1 << 31) - 1]])
    q, k = apbv.apbv_rotate(c.q, c.k, ints(c.at), c.rotation)
    check_rows(q, c.want(c.q, None))


def test_turning_back():
    c = Case(50, 4, 2, 64, 64, axes=2, norm=True, seed=3)
    plain = apbv.ApbvRotation(c.inv_freq, 64, axis=c.axis)
    q, k = apbv.apbv_rotate(c.q, c.k, c.positions, plain)
    q, k = apbv.apbv_rotate(q, k, -c.positions, plain)
    # two roundings of half a step each, of rows whose longest element is at most the row's length
    for got, x in ((q, c.q), (k, c.k)):
        assert (np.abs(f64(got) - f64(x)) <= 2.0 ** -8 * (np.abs(f64(x)) + 1.5 * np.abs(f64(x)).max(-1, keepdims=True))).all()


def test_position_zero_copies_the_bits():
    c = Case(33, 4, 2, 128, 128, seed=4)
    x = c.q.clone()
    x[0, 0, :6] = torch.tensor([float("inf"), -float("inf"), 3e38, -1e-39, 0.0, -0.0], dtype=torch.bfloat16)
    x[0, 0, 64:70] = 0.0
    q, _ = apbv.apbv_rotate(x, None, torch.zeros(33, dtype=torch.int32, device="cuda"), c.rotation)
    # (an infinity's partner is b cos 0 + inf sin 0, infinity times zero: not a number by the definition)
    finite = torch.isfinite(x) & torch.isfinite(x.roll(64, -1))
    assert (~finite).sum() == 4 and torch.equal(q[finite], x[finite])


def test_elements_behind_the_turned_ones_keep_their_bits():
    c = Case(33, 4, 2, 128, 32, seed=5)
    q, k = apbv.apbv_rotate(c.q, c.k, c.positions, c.rotation)
    assert torch.equal(q[..., 32:], c.q[..., 32:]) and torch.equal(k[..., 32:], c.k[..., 32:])


def test_norms_of_extreme_rows():
    """Squares beyond and below what float32 holds; rows of zeros; other rows are not touched by what is not a number."""
    c = Case(6, 2, 1, 128, 128, norm=True, seed=6, eps=0.0)
    x = c.q.contiguous()
    x[0] *= 1e25
    x[1] *= 1e-25
    q, _ = apbv.apbv_rotate(x, None, c.positions, c.rotation)
    check_rows(q, c.want(x, c.wq))
    x[2, 0] = 0.0
    x[3, 1, 5] = float("nan")
    soft = apbv.ApbvRotation(c.inv_freq, 128, axis=c.axis, q_weight=c.wq, eps=1e-6)
    q2, _ = apbv.apbv_rotate(x, None, c.positions, soft)
    assert (q2[2, 0] == 0).all() and torch.isnan(q2[3, 1]).any()
    assert torch.equal(q2[0], q[0]) and torch.isfinite(q2[3, 0]).all() and torch.isfinite(q2[4:]).all()


def test_one_tensor_alone_and_in_place():
    c = Case(77, 6, 3, 64, 64, axes=3, norm=True, seed=7)
    q, k = apbv.apbv_rotate(c.q, c.k, c.positions, c.rotation)
    q1, none = apbv.apbv_rotate(c.q, None, c.positions, c.rotation)
    also_none, k1 = apbv.apbv_rotate(None, c.k, c.positions, c.rotation)
    assert none is None and also_none is None and torch.equal(q, q1) and torch.equal(k, k1)
    q2, k2 = c.q.contiguous(), c.k.contiguous()
    r = apbv.apbv_rotate(q2, k2, c.positions, c.rotation, q_out=q2, k_out=k2)
    assert r[0] is q2 and torch.equal(q, q2) and torch.equal(k, k2)


def test_outputs_end_where_they_end():
    """Rows behind the outputs and around strided inputs stay as they were; repeated calls give the same bits."""
    for tokens, hq, hkv, d in ((5, 3, 1, 128), (70, 9, 2, 64), (1, 2, 1, 64), (2000, 20, 4, 128)):
        c = Case(tokens, hq, hkv, d, d, seed=tokens)
        before = c.joint.clone()
        room_q, room_k = (torch.full(((tokens * h + 3) * d,), 7.0, dtype=torch.bfloat16, device="cuda") for h in (hq, hkv))
        q, k = (r[:tokens * h * d].view(tokens, h, d) for r, h in ((room_q, hq), (room_k, hkv)))
        apbv.apbv_rotate(c.q, c.k, c.positions, c.rotation, q_out=q, k_out=k)
        assert (room_q[tokens * hq * d:] == 7).all() and (room_k[tokens * hkv * d:] == 7).all() and torch.equal(c.joint, before)
        again = apbv.apbv_rotate(c.q, c.k, c.positions, c.rotation)
        assert torch.equal(q, again[0]) and torch.equal(k, again[1])


def test_axes_that_are_the_same_and_no_tokens():
    c = Case(21, 4, 2, 64, 64, axes=3, seed=8)
    one = c.positions[0].contiguous()
    a = apbv.apbv_rotate(c.q, c.k, one, c.rotation)
    b = apbv.apbv_rotate(c.q, c.k, one.expand(3, 21), c.rotation)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    wide = torch.zeros(4, 50, dtype=torch.int32, device="cuda")
    wide[:3, 9:30] = c.positions
    assert torch.equal(apbv.apbv_rotate(c.q, None, wide[:, 9:30], c.rotation)[0], apbv.apbv_rotate(c.q, None, c.positions, c.rotation)[0])
    q, k = apbv.apbv_rotate(c.q[:0], c.k[:0], one[:0], c.rotation)
    assert q.shape == (0, 4, 64) and k.shape == (0, 2, 64)


def test_rows_beyond_32_bit_offsets():
    """As many tokens as a call takes, nearly: 2^24 of three heads, strided; rows here and there, the last ones among them."""
    tokens, hq, hkv, d = (1 << 24) - 3, 2, 1, 64
    rng = np.random.default_rng(12)
    print("tokens", tokens, flush=True)
    block = bf16(rng.standard_normal((1 << 12, hq + hkv, d)))
    joint = torch.empty(tokens, hq + hkv, d, dtype=torch.bfloat16, device="cuda")
    joint[:tokens // 4096 * 4096].view(-1, 4096, hq + hkv, d).copy_(block)
    joint[tokens // 4096 * 4096:] = block[:tokens % 4096]
    assert joint.numel() > 2 ** 31
    at = torch.arange(tokens, dtype=torch.int32, device="cuda").mul_(7)
    inv_freq, weight = frequencies(d), bf16(1.0 + 0.3 * rng.standard_normal(d))
    rotation = apbv.ApbvRotation(inv_freq, d, k_weight=weight)
    q, k = apbv.apbv_rotate(joint[:, :hq], joint[:, hq:], at, rotation)
    looked_at = torch.from_numpy(np.unique(np.concatenate((rng.integers(0, tokens, 300), [0, 11184810, 11184811, tokens - 2, tokens - 1])))).cuda()
    for x, got, w in ((joint[:, :hq], q, None), (joint[:, hq:], k, weight)):
        check_rows(got[looked_at], po.rotate(f64(x[looked_at]), f64(at[looked_at])[None], f64(inv_freq), [0] * (d // 2), False,
                                             None if w is None else f64(w), np.float64(np.float32(1e-6))))


# ---- appending to the cache

def slots_of(rng, tokens, n_pages, page, skip):
    s = rng.permutation(n_pages * page)[:tokens]
    s[rng.permutation(tokens)[:skip]] = -1
    return s


def held(cache, name):
    """[pages, heads, page, d] codes and [..., d / 32] scales, on the host."""
    return co.unpack(getattr(cache, name + "_codes").cpu().numpy()), getattr(cache, name + "_scales").cpu().numpy()


def check_append(c, cache, before, slots, n_pages, page):
    k, _ = c.want(c.k, c.wk)
    for name, x in (("k", k), ("v", f64(c.v))):
        codes, scales = (a.copy() for a in before[name])
        for t, s in enumerate(slots):
            if 0 <= s < n_pages * page:
                codes[s // page, :, s % page], scales[s // page, :, s % page] = co.encode(x[t])
        got_codes, got_scales = held(cache, name)
        assert np.array_equal(got_scales, scales)
        assert np.array_equal(co.decode(got_codes, got_scales), co.decode(codes, scales))


@pytest.mark.parametrize("adjacent,norm,page", [(False, False, 16), (False, True, 64), (True, True, 32), (True, False, 128)])
@pytest.mark.parametrize("shape", [(1, 2, 1, 64, 64), (1, 28, 4, 128, 128), (5, 9, 3, 128, 32), (31, 8, 2, 64, 48), (64, 28, 4, 128, 128), (150, 3, 1, 64, 16), (90, 8, 8, 128, 80)])
def test_append(shape, adjacent, norm, page):
    tokens, hq, hkv, d, rot = shape
    rng = np.random.default_rng(tokens + page)
    c = Case(*shape, axes=1 + page % 3, adjacent=adjacent, norm=norm, seed=tokens, far=100_000)
    n_pages = tokens // page + 3
    cache = apbv.apbv_cache_empty(n_pages, hkv, d, page)
    for t in cache:
        t.random_(0, 250)
    before = {name: held(cache, name) for name in "kv"}
    slots = slots_of(rng, tokens, n_pages, page, tokens // 5)
    q = apbv.apbv_cache_append(cache, c.q, c.k, c.v, ints(slots), c.positions, c.rotation)
    assert torch.equal(q, apbv.apbv_rotate(c.q, None, c.positions, c.rotation)[0])
    check_append(c, cache, before, slots, n_pages, page)


def test_append_without_queries_and_slots_out_of_range():
    c = Case(40, 4, 2, 64, 64, norm=True, seed=9)
    cache = apbv.apbv_cache_empty(4, 2, 64, 16)
    for t in cache:
        t.random_(0, 250)
    before = {name: held(cache, name) for name in "kv"}
    slots = np.arange(40) + 20                                        # the last ones lie behind the pool
    slots[3], slots[4] = -(1 << 31), (1 << 31) - 1
    assert apbv.apbv_cache_append(cache, None, c.k, c.v, ints(slots), c.positions, c.rotation) is None
    check_append(c, cache, before, slots, 4, 16)


def test_append_to_pages_beyond_32_bit_offsets():
    """A pool of 5 GB, and slots on both sides of 2^32 bytes, the last one among them."""
    tokens, hkv, d, page, n_pages = 500, 8, 128, 256, 40000
    print("5 GB pool", flush=True)
    cache = apbv.apbv_cache_empty(n_pages, hkv, d, page)
    assert n_pages * cache.k_codes.stride(0) > 2 ** 32
    c = Case(tokens, 16, hkv, d, d, axes=2, norm=True, seed=13)
    slots = np.random.default_rng(14).permutation(n_pages * page)[:tokens]
    slots[0], slots[tokens - 1] = n_pages * page - 1, 0
    apbv.apbv_cache_append(cache, c.q, c.k, c.v, ints(slots), c.positions, c.rotation)
    for got, want in zip(apbv.apbv_cache_load(cache, ints(slots)), (c.want(c.k, c.wk)[0], f64(c.v))):
        assert np.array_equal(f64(got), co.decode(*co.encode(want)))


def test_append_of_extreme_values():
    """Infinities, NaN, zeros and the ends of bf16's range: as a stored row holds them."""
    c = Case(8, 2, 1, 64, 64, seed=10)
    k, v = c.k.contiguous(), c.v.contiguous()
    k[0] = 0.0
    k[1, 0, 3], k[1, 0, 40] = float("nan"), float("inf")
    k[2] *= 1e37
    k[3] *= 1e-38
    k[4, 0, 7] = 3.3e38
    k[4, 0, 39] = 3.3e38                                              # what they turn into may lie beyond bf16
    v[1, 0, 2], v[2, 0, 5] = -float("inf"), float("nan")
    cache = apbv.apbv_cache_empty(2, 1, 64, 16)
    at = torch.zeros(8, dtype=torch.int32, device="cuda")
    at[4:] = 1
    apbv.apbv_cache_append(cache, None, k, v, ints(np.arange(8)), at, c.rotation)
    with np.errstate(invalid="ignore", over="ignore"):
        kk, _ = po.rotate(f64(k), [at.cpu().numpy()] * 1, f64(c.inv_freq), [0] * 32)
    for name, x in (("k", kk), ("v", f64(v))):
        codes, scales = held(cache, name)
        want = co.encode(x)
        for t in range(8):
            assert np.array_equal(scales[0, :, t], want[1][t]), (name, t)
            assert np.array_equal(co.decode(codes[0, :, t], scales[0, :, t]), co.decode(want[0][t], want[1][t])), (name, t)


def test_append_of_turned_keys_is_near_a_store_of_rounded_ones():
    """One rounding or two: at most one code apart, and hardly ever."""
    c = Case(200, 4, 4, 128, 128, axes=3, norm=True, seed=11)
    a, b = apbv.apbv_cache_empty(4, 4, 128, 64), apbv.apbv_cache_empty(4, 4, 128, 64)
    slots = ints(np.arange(200))
    apbv.apbv_cache_append(a, c.q, c.k, c.v, slots, c.positions, c.rotation)
    apbv.apbv_cache_store(b, apbv.apbv_rotate(None, c.k, c.positions, c.rotation)[1], c.v, slots)
    ka, va = (f64(x) for x in apbv.apbv_cache_load(a, slots))
    kb, vb = (f64(x) for x in apbv.apbv_cache_load(b, slots))
    assert np.array_equal(va, vb)
    # a rounding to bf16 moves a value over a border at most 2^-8 of it away; steps are a third of it at most where values are widest apart
    assert (ka != kb).mean() < 2.0 ** -5 and (np.abs(ka - kb) <= 2 / 3 * np.maximum(np.abs(ka), np.abs(kb)) + 0.25 * np.abs(kb).max(-1, keepdims=True)).all()


def test_captured_into_a_graph_and_replayed():
    c = Case(37, 8, 2, 64, 64, axes=2, norm=True, seed=12)
    cache = apbv.apbv_cache_empty(4, 2, 64, 16)
    q_in, k_in, at = c.q.contiguous(), c.k.contiguous(), c.positions.clone()
    slots = ints(np.arange(37))
    out = {n: torch.empty_like(t) for n, t in (("q", q_in), ("k", k_in), ("qa", q_in))}
    kl, vl = torch.empty_like(k_in), torch.empty_like(k_in)

    def step():
        apbv.apbv_rotate(q_in, k_in, at, c.rotation, q_out=out["q"], k_out=out["k"])
        apbv.apbv_cache_append(cache, q_in, k_in, c.v, slots, at, c.rotation, q_out=out["qa"])
        apbv.apbv_cache_load(cache, slots, k_out=kl, v_out=vl)
    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for n in range(4):
        q_in.normal_()
        k_in.normal_()
        at.add_(n)
        g.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (*out.values(), kl, vl)]
        for t in (*out.values(), kl, vl):
            t.fill_(float("nan"))
        step()
        assert all(torch.equal(a, b) for a, b in zip(got, (*out.values(), kl, vl)))


def test_calls_on_other_streams():
    c = Case(500, 16, 2, 128, 128, axes=3, norm=True, seed=13)
    want = apbv.apbv_rotate(c.q, c.k, c.positions, c.rotation)
    cache = apbv.apbv_cache_empty(10, 2, 128, 64)
    slots = ints(np.arange(500))
    side = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = apbv.apbv_rotate(c.q, c.k, c.positions, c.rotation, stream=side[0])
    q = apbv.apbv_cache_append(cache, c.q, c.k, c.v, slots, c.positions, c.rotation, stream=side[1])
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and torch.equal(q, want[0])


def test_what_does_not_fit_is_refused():
    c = Case(6, 4, 2, 64, 64, seed=14)
    cache = apbv.apbv_cache_empty(4, 2, 64, 16)
    slots = ints(np.arange(6))
    for error, call in (
            (ValueError, lambda: apbv.apbv_rotate(c.q, c.k[:5], c.positions, c.rotation)),
            (TypeError, lambda: apbv.apbv_rotate(c.q.float(), c.k, c.positions, c.rotation)),
            (TypeError, lambda: apbv.apbv_rotate(c.q, c.k, c.positions.long(), c.rotation)),
            (ValueError, lambda: apbv.apbv_rotate(c.q, c.k, c.positions[:, :5], c.rotation)),
            (ValueError, lambda: apbv.apbv_rotate(c.q, c.k, c.positions.cpu(), c.rotation)),
            (TypeError, lambda: apbv.apbv_rotate(c.q, c.k, c.positions, "rotation")),
            (ValueError, lambda: apbv.apbv_rotate(c.q, c.k, c.positions, apbv.ApbvRotation(c.inv_freq, 128))),
            (ValueError, lambda: apbv.apbv_rotate(c.q, c.k, c.positions, apbv.ApbvRotation(c.inv_freq.cpu(), 64))),
            (ValueError, lambda: apbv.apbv_rotate(c.q, c.k, c.positions, c.rotation, q_out=torch.empty(5, 4, 64, dtype=torch.bfloat16, device="cuda"))),
            (ValueError, lambda: apbv.apbv_cache_append(cache, c.q, c.k, c.v[:5], slots, c.positions, c.rotation)),
            (ValueError, lambda: apbv.apbv_cache_append(cache, c.q, c.k, c.v, slots[:5], c.positions, c.rotation)),
            (ValueError, lambda: apbv.apbv_cache_append(cache, c.q[:5], c.k, c.v, slots, c.positions, c.rotation)),
            (ValueError, lambda: apbv.apbv_cache_append(cache, c.q, c.q, c.q, slots, c.positions, c.rotation))):
        with pytest.raises(error):
            call()
    q = c.q.contiguous()[:, :2]
    with pytest.raises(ValueError):
        apbv.apbv_rotate(q, None, c.positions, c.rotation, q_out=q)   # in place, but not dense
