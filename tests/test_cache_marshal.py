"""The cache's calls through the native marshalling: what is not the plain call is handed back (CPU), and the plain call gives the
results and errors of the general way (GPU), which an explicit stream takes."""
import pytest
import torch

import paper_2601_21444_amd as apbv
import paper_2601_21444_amd.binding as binding
from tests.test_marshal import both, native  # noqa: F401


def test_other_than_plain_calls_are_handed_back():
    apbv.load_library()
    nat = binding._native
    i = lambda *s: torch.zeros(s, dtype=torch.int32)
    c = apbv.apbv_cache_empty(4, 2, 64, 16, device="cpu")
    q = torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    assert nat.cache_map(i(3), i(3), i(3, 2), i(5), i(1), 16, 4, i(3), i(4), i(4), i(1)) is None          # not on a GPU
    assert nat.cache_map(1, i(3)) is None and nat.cache_store(c, q, q, i(3)) is None and nat.cache_store(c, q) is None
    assert nat.cache_load(c, i(3), q, q) is None and nat.cache_load((1, 2, 3, 4), i(3), q, q) is None
    assert nat.cache_attention(q, c, i(3, 2), i(3), 0.1, None, None, True, q, None, q) is None
    assert nat.cache_attention(q, tuple(c), i(3, 2), i(3), "x", None, None, True, q, None, q) is None


@pytest.mark.gpu
def test_native_and_general_marshalling_agree(native):  # noqa: F811
    g = torch.Generator(device="cuda").manual_seed(1)
    bf = lambda *s: torch.randn(s, generator=g, device="cuda", dtype=torch.bfloat16)
    i = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    new = lambda *s, dtype=torch.int32: torch.empty(s, dtype=dtype, device="cuda")
    c = apbv.apbv_cache_empty(9, 2, 128, 32)
    table = i([[3, 1, 7, 0], [5, 2, 0, 0]])
    print("cache marshal", flush=True)
    both(native, apbv.apbv_cache_map, (i([70, 40]), i([80, 0]), table, i([4, 6, 0, 0]), i([2]), 32, 12),
         dict(lengths_out=new(2), starts_out=new(3), slots_out=new(12), free_count_out=new(1)))
    k, v, slots = bf(110, 5, 128)[:, :2], bf(110, 5, 128)[:, 3:], i([3 * 32 + j for j in range(32)] + [32 + j for j in range(32)] + [7 * 32 + j for j in range(32)] + [5 * 32 + j for j in range(14)])
    for extra, said in (({}, [0]), ({"stream": torch.cuda.current_stream()}, [])):
        for t in c:
            t.fill_(255)
        native.said.clear()
        assert apbv.apbv_cache_store(c, k, v, slots, **extra) is c and native.said == said
        torch.cuda.synchronize()
        if extra:
            assert all(torch.equal(a, b) for a, b in zip(c, kept))
        kept = [t.clone() for t in c]
    both(native, apbv.apbv_cache_load, (c, slots), dict(k_out=new(110, 2, 128, dtype=torch.bfloat16), v_out=new(110, 2, 128, dtype=torch.bfloat16)))
    q = bf(5, 8, 128)
    ws = new(apbv.apbv_cache_attention_workspace_bytes(2, 5, 8, 2, 128, 5), dtype=torch.uint8)
    outs = dict(out=new(5, 8, 128, dtype=torch.bfloat16), lse_out=new(8, 5, dtype=torch.float32), workspace=ws)
    both(native, apbv.apbv_cache_attention, (q, c, table, i([90, 14]), 0.1), outs, q_starts=i([0, 4, 5]), max_q=4, return_lse=True)
    both(native, apbv.apbv_cache_attention, (q, c, table, i([90, 14]), 0.1), outs, q_starts=i([0, 4, 5]), causal=False, return_lse=True)
    four = dict(out=new(4, 8, 128, dtype=torch.bfloat16), lse_out=new(8, 4, dtype=torch.float32), workspace=ws)
    both(native, apbv.apbv_cache_attention, (q[:4], c, table, i([90, 14]), 0.1), four, return_lse=True)
    # refusals: the library's either way, the binding's handed back
    cases = [lambda **s: apbv.apbv_cache_attention(q, c, table, i([90, 14]), -1.0, q_starts=i([0, 4, 5]), **outs, **s),
             lambda **s: apbv.apbv_cache_attention(q, c, table, i([90, 14]), 0.1, q_starts=i([0, 4, 5]), out=outs["out"], workspace=ws[:256], **s),
             lambda **s: apbv.apbv_cache_attention(q, c, table, i([90, 14]), 0.1, q_starts=i([0, 4]), **outs, **s),
             lambda **s: apbv.apbv_cache_attention(q, c, table.long(), i([90, 14]), 0.1, q_starts=i([0, 4, 5]), **outs, **s),
             lambda **s: apbv.apbv_cache_store(c, k, v, slots[:5], **s),
             lambda **s: apbv.apbv_cache_store(c._replace(v_scales=c.v_scales[:3]), k, v, slots, **s),
             lambda **s: apbv.apbv_cache_load(c, slots, k_out=q, v_out=q, **s),
             lambda **s: apbv.apbv_cache_map(i([70, 40]), i([80, 0]), table, i([4]), i([2]), 24, 12, lengths_out=new(2), starts_out=new(3), slots_out=new(12), free_count_out=new(1), **s)]
    for case, status in zip(cases, (-2, -4, None, None, None, None, None, -3)):
        said = []
        for s in ({}, {"stream": torch.cuda.current_stream()}):
            native.said.clear()
            with pytest.raises(Exception) as err:
                case(**s)
            said.append((err.type, str(err.value)))
            assert native.said == ([] if s else [status])
        assert said[0] == said[1]
