"""Every kernel that a call behind shared prefixes may take, against the fp64 oracle (the bounds are those of test_gpu_shared.py): both head
sizes, pages that hold a whole tile of keys and pages that do not, and each height of row tiles, number of waves and of joining waves.  Which one
a call takes is held against the rules on the CPU."""
import itertools
import os
import subprocess

import numpy as np
import pytest
import torch

from tests.test_abi_host import ROOT, SANITIZE
from tests.test_gpu_cache import dev_int
from tests.test_gpu_shared import Shared

# what is planned: query heads, KV heads, [(prefix, [(queries, own keys)])], room that the tables have besides
CALLS = {
    "whole 8": (8, 2, [(130, [(1, 30), (3, 20), (1, 0)])], 0),
    "whole 4": (28, 4, [(200, [(1, i % 40) for i in range(200)])], 0),
    "cut 16 16 4": (8, 2, [(5000, [(1, 300), (1, 20), (1, 77)])], 20000),
    "cut 16 16 1": (16, 2, [(600 + 40 * g, [(1, 10 + 9 * i) for i in range(5)]) for g in range(20)], 2000),
    "cut 32 16 4": (28, 4, [(4000, [(1, 5), (1, 200), (1, 64), (1, 0)])], 600000),
    "cut 32 16 1": (28, 4, [(900 + 100 * g, [(1, 5), (1, 90), (1, 64), (1, 2 * g)]) for g in range(12)], 600000),
    "cut 128 16 4": (16, 2, [(5000, [(1, 17 * i) for i in range(21)])], 600000),
    "cut 128 16 1": (16, 2, [(3000, [(1, 1 + 3 * i) for i in range(90)])], 600000),
    "cut 128 128 4": (16, 2, [(4500, [(9, 100), (20, 333), (1, 40), (7, 3)])], 600000),
    "cut 128 128 1": (16, 2, [(2500, [(60, 100), (40, 333)]), (0, [(33, 90)])], 600000),
}
PAGES = (16, 32, 64, 128)


def tables(page, groups, room):
    need = max([p for p, _ in groups] + [k for _, r in groups for _, k in r])
    return (-(-need // page) + 1 + room // page) * page               # as Shared makes them


def test_the_calls_take_every_kernel(tmp_path):
    exe = tmp_path / "shared_plans"
    incs = ["-I", os.path.join(ROOT, "paper_2601_21444_amd", "csrc"), "-I", os.path.join(ROOT, "include")]
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", *SANITIZE, *incs, os.path.join(ROOT, "tests", "host", "shared_plans.cpp"), "-o", str(exe)], check=True)
    lines, want = [], []
    for (what, (hq, hkv, groups, room)), d, page in itertools.product(CALLS.items(), (64, 128), PAGES):
        requests = [r for _, rs in groups for r in rs]
        keys = tables(page, groups, room)
        lines.append(" ".join(map(str, (len(groups), len(requests), hq, hkv, d, sum(q for q, _ in requests), max(q for q, _ in requests), keys, keys, 0))))
        want.append(what)
    out = subprocess.run([str(exe)], input="\n".join(lines) + "\n", capture_output=True, text=True, check=True).stdout.splitlines()
    assert out == want, [(a, b, c) for a, b, c in zip(lines, out, want) if b != c]
    # all that there are (launch_dim and short_kernel): row tiles of 16, 32 or 128 rows with 16 of the own keys, or 128 of both
    assert set(CALLS) == {f"whole {w}" for w in (4, 8)} | {f"cut {t} {j}" for t in ("16 16", "32 16", "128 16", "128 128") for j in (1, 4)}


@pytest.mark.gpu
@pytest.mark.parametrize("page", PAGES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("what", CALLS)
def test_matches_the_oracle(what, d, page):
    hq, hkv, groups, room = CALLS[what]
    print(what, d, page, flush=True)
    rng = np.random.default_rng((71, d, page, len(what)))
    s = Shared(rng, hq, hkv, d, page, groups)
    assert s.x.table.shape[1] * page + room // page * page == tables(page, groups, room)
    n = len(s.requests)
    looked_at = range(n) if n <= 6 else sorted({0, 1, n // 2, n - 1, *(int(b) for b in rng.integers(0, n, 8))})
    for causal in (True, False):
        out, lse = s.run(causal, wide=room)
        s.check(out, lse, causal, what, only=looked_at)
        assert torch.isfinite(out.float()).all() and (out.float().abs() < 20).all()
