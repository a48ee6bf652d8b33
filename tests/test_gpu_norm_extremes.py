"""Norms of rows that hold an infinity, and of rows so small or so large that one over their root mean square is no normal float32, against
the oracle in 64 bits; the bounds are those of test_gpu_positions.py (half a step of bf16, eight roundings of float32)."""
import numpy as np
import pytest
import torch

import paper_2601_21444_amd as apbv
from oracle import cache_oracle as co
from oracle import positions_oracle as po
from tests.test_gpu_positions import Case, check_rows, f64, held, ints

pytestmark = pytest.mark.gpu


def wanted(c, x, w, rotation_eps):
    with np.errstate(all="ignore"):
        return po.rotate(f64(x), c.at, f64(c.inv_freq), c.axis, c.adjacent, f64(w), np.float64(np.float32(rotation_eps)))


@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("tokens", [9, 20000])                        # one row a thread, and four
@pytest.mark.parametrize("d,rot", [(64, 64), (64, 32), (128, 128), (128, 48)])
def test_an_infinity_leaves_the_row_zeros(d, rot, tokens, adjacent):
    """x w / sqrt(infinity): the finite elements are zero, an infinite one is not a number, nor is the element that it turns with."""
    c = Case(tokens, 2, 1, d, rot, axes=2, adjacent=adjacent, norm=True, seed=d + rot)
    x, k = c.q.contiguous(), c.k.contiguous()
    hit = [(1, 0, 3, float("inf")), (1, 1, rot // 2 + 1, -float("inf")), (5, 0, d - 1, float("inf")), (tokens - 1, 1, 0, -float("inf"))]
    for t, h, e, value in hit:
        x[t, h, e] = value
    k[2, 0, 1], k[2, 0, rot - 1] = float("inf"), -float("inf")
    got, got_k = apbv.apbv_rotate(x, k, c.positions, c.rotation)
    for y, out, w, rows in ((x, got, c.wq, {(t, h) for t, h, _, _ in hit}), (k, got_k, c.wk, {(2, 0)})):
        for t, h in rows:
            at = c.at
            c.at = at[:, t:t + 1]
            want, _ = wanted(c, y[t:t + 1, h:h + 1], w, c.eps)
            c.at = at
            have = f64(out[t, h])
            assert np.array_equal(np.isnan(have), np.isnan(want[0, 0])) and (have[~np.isnan(have)] == 0).all(), (t, h)
        others = torch.ones(out.shape[:2], dtype=torch.bool, device="cuda")
        for t, h in rows:
            others[t, h] = False
        assert torch.isfinite(out[others]).all()


ROWS = [
    # eps, what a row's elements are multiplied by: ends of bf16's range, subnormal ones among them
    (0.0, 2.0 ** -128), (0.0, 2.0 ** -131), (0.0, 2.0 ** -100), (0.0, 2.0 ** -61), (0.0, 2.0 ** 59), (0.0, 2.0 ** 61), (0.0, 2.0 ** 100), (0.0, 2.0 ** 124),
    (1e-6, 2.0 ** 124), (1e-6, 2.0 ** -128), (3e38, 1.0), (3e38, 2.0 ** 70), (1e-38, 1e-19),
]


@pytest.mark.parametrize("eps,factor", ROWS)
@pytest.mark.parametrize("tokens", [6, 12000])
def test_norms_over_the_whole_range(tokens, eps, factor):
    for d in (64, 128):
        c = Case(tokens, 2, 1, d, d, axes=1, norm=True, seed=6, eps=eps, spread=0.0)
        rotation = apbv.ApbvRotation(c.inv_freq, d, axis=c.axis, q_weight=c.wq, k_weight=c.wk, eps=eps)
        x, k = ((t.double() * factor).to(torch.bfloat16) for t in (c.q, c.k))
        assert torch.isfinite(x).all() and x.any()
        got, got_k = apbv.apbv_rotate(x, k, c.positions, rotation)
        n = min(tokens, 300)
        c.at = c.at[:, :n]
        check_rows(got[:n], wanted(c, x[:n], c.wq, eps))
        check_rows(got_k[:n], wanted(c, k[:n], c.wk, eps))


def test_one_smallest_element():
    """A row of one subnormal element: sqrt(d) times its weight, whatever the element is."""
    c = Case(4, 2, 1, 128, 128, norm=True, seed=8, eps=0.0)
    x = torch.zeros_like(c.q)
    x[0, 0, 5], x[1, 1, 70], x[2, 0, 127], x[3, 1, 0] = 2.0 ** -133, -(2.0 ** -133), 2.0 ** -126, 3.3e38
    x[:, :, 9] += (x.abs().amax(-1) == 0) * 1.0                       # (rows of zeros are not numbers at eps = 0)
    got, _ = apbv.apbv_rotate(x, None, c.positions, c.rotation)
    check_rows(got, wanted(c, x, c.wq, 0.0))
    assert (got[0, 0].float().norm() > 5).all()


@pytest.mark.parametrize("d", [64, 128])
def test_appended_keys_of_such_rows(d):
    """The codes are those of the float64 value; a row with an infinity is held as zeros."""
    c = Case(16, 2, 2, d, d, axes=2, norm=True, seed=9, eps=0.0)
    k, v = c.k.contiguous(), c.v.contiguous()
    for t, factor in enumerate((2.0 ** -128, 2.0 ** -131, 2.0 ** -100, 2.0 ** 61, 2.0 ** 100, 2.0 ** 124)):
        k[t] = (k[t].double() / k[t].abs().max().double() * factor).to(torch.bfloat16)
    k[8, 0, 3], k[9, 1, d - 1], k[9, 1, 0] = float("inf"), -float("inf"), float("inf")
    cache = apbv.apbv_cache_empty(1, 2, d, 16)
    q = apbv.apbv_cache_append(cache, c.q, k, v, ints(np.arange(16)), c.positions, c.rotation)
    assert torch.equal(q, apbv.apbv_rotate(c.q, None, c.positions, c.rotation)[0])
    want, _ = wanted(c, k, c.wk, 0.0)
    codes, scales = held(cache, "k")
    for t in range(16):
        want_codes, want_scales = co.encode(want[t])
        assert np.array_equal(scales[0, :, t], want_scales), t
        assert np.array_equal(co.decode(codes[0, :, t], scales[0, :, t]), co.decode(want_codes, want_scales)), t
    assert (co.decode(codes[0, 0, 8], scales[0, 0, 8]) == 0).all() and (co.decode(codes[0, 1, 9], scales[0, 1, 9]) == 0).all()
