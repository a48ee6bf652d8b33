"""Attention behind short shared prefixes in one launch, of groups whose sizes only the device knows, against the fp64 oracle
(the bounds are those of test_gpu_shared.py)."""
import numpy as np
import pytest
import torch

from tests.test_gpu_cache import dev_int
from tests.test_gpu_shared import Shared

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("few,most", [(3, 300), (62, 150), (63, 65), (200, 400), (999, 500)])
def test_one_group_has_most_of_the_requests(few, most):
    rng = np.random.default_rng((61, few))
    place = few // 3
    sizes = [1] * place + [most] + [int(m) for m in rng.integers(0, 3, few - place)]
    groups = [(int(rng.integers(0, 65)), [(int(rng.integers(0, 3)), int(rng.integers(0, 65))) for _ in range(m)]) for m in sizes]
    print("groups", few + 1, "requests", sum(sizes), flush=True)
    s = Shared(rng, 4, 2, 64, 64, groups, (((2, 10),), ((1, 0), (3, 33))), lead=3, tail=5)
    looked_at = sorted({0, 1, len(s.requests) - 1, place, place + 1, place + most, *(int(b) for b in rng.integers(0, len(s.requests), 120))})
    for causal in (True, False):
        out, lse = s.run(causal)
        s.check(out, lse, causal, "one large group", only=looked_at)
        rows = slice(s.starts[0], s.starts[-1])
        assert (out[rows] != 77.0).any(-1).all() and (lse[:, rows] != 77.0).all()        # every row has been written


@pytest.mark.parametrize("groups,each", [(1, 7), (1, 130), (5, 3), (70, 2), (65, 40)])
def test_equal_groups_of_unequal_requests(groups, each):
    """Without group_starts, with q_starts: one request of many rows, others of one or none."""
    rng = np.random.default_rng((62, groups))
    requests = [[(int(rng.integers(0, 2)), int(rng.integers(0, 65))) for _ in range(each)] for _ in range(groups)]
    requests[groups // 2][each // 2] = (90, 60)
    print("equal groups", groups, each, flush=True)
    s = Shared(rng, 6, 2, 128, 64, [(int(rng.integers(0, 65)), r) for r in requests], lead=1, tail=2)
    at = groups // 2 * each + each // 2
    looked_at = sorted({0, at - 1, at, at + 1, len(s.requests) - 1, *(int(b) for b in rng.integers(0, len(s.requests), 60))} - {-1})
    for max_q in (90, 1):                                             # (a bound that does not hold: speed only)
        out, lse = s.run(group_starts=None, max_q=max_q)
        s.check(out, lse, True, "equal groups", only=looked_at)
        rows = slice(s.starts[0], s.starts[-1])
        assert (out[rows] != 77.0).any(-1).all()


def test_one_group_of_as_many_requests_as_there_may_be():
    """Row tiles whose requests lie behind thousands of others, equally many rows each."""
    rng = np.random.default_rng(63)
    for page, hq, hkv in ((16, 1, 1), (64, 5, 1)):
        s = Shared(rng, hq, hkv, 64, page, [(50, [(1, int(rng.integers(0, 40))) for _ in range(4096)])])
        looked_at = sorted({0, 1, 15, 16, 63, 64, 4032, 4095, *(int(b) for b in rng.integers(0, 4096, 100))})
        for kw in (dict(), dict(group_starts=None, q_starts=None, max_q=None)):
            out, lse = s.run(**kw)
            s.check(out, lse, True, "4096 requests", only=looked_at)
            assert torch.isfinite(out.float()).all() and (out.float().abs() < 20).all()
