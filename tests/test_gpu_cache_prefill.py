"""A cached prefix read back for the prefill's calls: rows of apbv_cache_load as the passing and local keys of apbv_host_attention and
apbv_query_attention, beside apbv_cache_attention over the same slots, all against the fp64 oracle."""
import math

import numpy as np
import pytest
import torch

import paper_2601_21444_amd as apbv
from oracle import cache_oracle as co
from tests.test_gpu_cache import U, Batch, check, dev_int, to_f64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hq,hkv,d,page,prefix,n", [(8, 2, 64, 16, 333, 1), (16, 2, 128, 64, 700, 40), (28, 4, 128, 32, 1500, 130)])
def test_a_cached_prefix_in_the_prefills_attention(hq, hkv, d, page, prefix, n):
    x = Batch(np.random.default_rng((71, d, n)), hq, hkv, d, page, [(n, prefix + n)])
    print("cached prefix", hq, hkv, d, page, prefix, n, flush=True)
    out, lse = x.run()
    slots = dev_int([int(x.table[0, j // page]) * page + j % page for j in range(prefix + n)])
    k, v = apbv.apbv_cache_load(x.cache, slots)
    ref, ref_lse, spread = co.attention(x.qv, to_f64(k), to_f64(v), 1 / math.sqrt(d), True)
    check(out, lse, ref, ref_lse, spread, "over the cache")
    none = k[:0]
    for name, call in (("host", apbv.apbv_host_attention), ("query", apbv.apbv_query_attention)):
        got, got_lse = call(x.q, none, none, k[:prefix], v[:prefix], k[prefix:], v[prefix:], 1 / math.sqrt(d), return_lse=True)
        check(got, None, ref, ref_lse, spread, name)
        # (the weights' sum may be of the rounded ones: half a step of bf16)
        assert np.abs(to_f64(got_lse) - ref_lse).max() <= U + 1e-3
