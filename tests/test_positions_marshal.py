"""The calls of include/apbv_positions.h and apbv_shared.h through the native marshalling: what is not the plain call is handed back
(CPU), the plain call gives the results and errors of the general way (GPU), and what a call that names its stream leaves to the
binding is memory of that stream."""
import copy
import pickle

import pytest
import torch

import paper_2601_21444_amd as apbv
import paper_2601_21444_amd.binding as binding
from paper_2601_21444_amd import positions as positions_module
from paper_2601_21444_amd import shared as shared_module
from tests.test_marshal import both, native  # noqa: F401
from tests.test_stream_memory import SIDE, Library, allocations, check  # noqa: F401


def test_other_than_plain_calls_are_handed_back():
    apbv.load_library()
    nat = binding._native
    i = lambda *s: torch.zeros(s, dtype=torch.int32)
    c = apbv.apbv_cache_empty(4, 2, 64, 16, device="cpu")
    q = torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    r = apbv.ApbvRotation(torch.ones(32), 64)
    assert nat.rotate(q, q, i(3), r._plan, q, q) is None and nat.rotate(q, None, i(3), r._plan, q, None) is None          # not on a GPU
    assert nat.rotate(None, None, i(3), r._plan, None, None) is None and nat.rotate(q, q, i(3), (1, 2, 3), q, q) is None
    assert nat.rotate(q, q, i(3), r, q, q) is None and nat.rotate(q, q) is None and nat.rotate(q, q, i(3), (0, 1, 64, 0), q, q) is None
    assert nat.cache_append(c, q, q, q, i(3), i(3), r._plan, q) is None and nat.cache_append(c) is None
    assert nat.cache_shared_attention(q, c, i(1, 2), i(1), i(3, 2), i(3), 0.1, None, None, None, True, q, None, q) is None


def test_a_copy_has_an_address_of_its_own():
    r = apbv.ApbvRotation(torch.ones(32), 64, axis=[i % 2 for i in range(32)], adjacent=True, q_weight=torch.ones(64, dtype=torch.bfloat16), eps=0.5)
    for twin in (copy.copy(r), copy.deepcopy(r), pickle.loads(pickle.dumps(r))):
        assert twin._plan[0] != r._plan[0] and twin._plan[1:] == r._plan[1:] and twin._struct.eps == 0.5 and twin._struct.adjacent == 1
        assert list(twin._struct.axis) == list(r._struct.axis) and twin._struct.q_weight == twin.q_weight.data_ptr()


def test_allocations_are_of_the_named_stream(allocations, monkeypatch):  # noqa: F811
    for module in (positions_module, shared_module):
        for name, value in (("load_library", Library), ("_rows_device", lambda t, name, stream: t.device), ("_check_ints", lambda *a: None)):
            monkeypatch.setattr(module, name, value)
    monkeypatch.setattr(positions_module, "_check_positions", lambda *a: 0)
    monkeypatch.setattr(shared_module, "_check_table", lambda t, n, dev, name="": (t.stride(0), t.shape[1]))
    i = lambda *s: torch.zeros(s, dtype=torch.int32)
    page = lambda width: torch.zeros(4, 2, 16, width, dtype=torch.uint8)
    c = apbv.ApbvCache(page(32), page(32), page(2), page(2))
    q, k = torch.zeros(3, 4, 64, dtype=torch.bfloat16), torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    r = apbv.ApbvRotation(torch.ones(32), 64)
    for call, outputs, workspaces in ((lambda: apbv.apbv_rotate(q, k, i(3), r, stream=SIDE), 2, 0),
                                      (lambda: apbv.apbv_cache_append(c, q, k, k, i(3), i(3), r, stream=SIDE), 1, 0),
                                      (lambda: apbv.apbv_cache_shared_attention(q, c, i(1, 2), i(1), i(3, 2), i(3), 0.1, return_lse=True, stream=SIDE), 2, 1)):
        allocations.clear()
        call()
        check(allocations, outputs, workspaces)


@pytest.mark.gpu
def test_native_and_general_marshalling_agree(native):  # noqa: F811
    g = torch.Generator(device="cuda").manual_seed(1)
    bf = lambda *s: torch.randn(s, generator=g, device="cuda", dtype=torch.bfloat16)
    i = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    new = lambda *s, dtype=torch.bfloat16: torch.empty(s, dtype=dtype, device="cuda")
    r = apbv.ApbvRotation(torch.rand(64, device="cuda"), 128, axis=[a % 3 for a in range(64)], q_weight=bf(128), k_weight=bf(128))
    joint, at = bf(40, 14, 128), torch.randint(0, 9999, (3, 40), dtype=torch.int32, device="cuda")
    q, k, v = joint[:, :8], joint[:, 8:10], joint[:, 12:]
    print("positions marshal", flush=True)
    outs = dict(q_out=new(40, 8, 128), k_out=new(40, 2, 128))
    both(native, apbv.apbv_rotate, (q, k, at, r), outs)
    both(native, apbv.apbv_rotate, (q, k, at[1], r), outs)
    for one in ((q, None), (None, k)):
        for said, extra in (([0], {}), ([], {"stream": torch.cuda.current_stream()})):
            native.said.clear()
            a, b = apbv.apbv_rotate(*one, at, r, **outs, **extra)
            assert native.said == said and (a is outs["q_out"] or one[0] is None) and (b is outs["k_out"] or one[1] is None) and (a is None) != (b is None)
    c, slots = apbv.apbv_cache_empty(9, 2, 128, 32), i(list(range(3, 43)))
    kept = []
    for with_q in (True, False):
        for said, extra in (([0], {}), ([], {"stream": torch.cuda.current_stream()})):
            for t in (*c, outs["q_out"]):
                t.fill_(1)
            native.said.clear()
            got = apbv.apbv_cache_append(c, q if with_q else None, k, v, slots, at, r, q_out=outs["q_out"], **extra)
            torch.cuda.synchronize()
            assert native.said == said and got is (outs["q_out"] if with_q else None)
            kept.append([t.clone() for t in (*c, outs["q_out"])])
    assert all(torch.equal(x, y) for x, y in zip(kept[0], kept[1])) and all(torch.equal(x, y) for x, y in zip(kept[2], kept[3]))
    assert all(torch.equal(x, y) for x, y in zip(kept[0][:4], kept[2][:4])) and (kept[2][4] == 1).all()
    pt, pl, t, l = i([[0, 1]]), i([40]), i([[2, 3], [4, 5], [6, 7]]), i([9, 33, 0])
    x = bf(5, 8, 128)
    ws = new(apbv.apbv_cache_shared_attention_workspace_bytes(1, 3, 5, 8, 2, 128, 5), dtype=torch.uint8)
    outs = dict(out=new(5, 8, 128), lse_out=new(8, 5, dtype=torch.float32), workspace=ws)
    args = (x, c, pt, pl, t, l, 0.1)
    both(native, apbv.apbv_cache_shared_attention, args, outs, group_starts=i([0, 3]), q_starts=i([0, 1, 4, 5]), max_q=3, return_lse=True)
    both(native, apbv.apbv_cache_shared_attention, args, outs, q_starts=i([0, 1, 4, 5]), causal=False, return_lse=True)
    three = dict(out=new(3, 8, 128), lse_out=new(8, 3, dtype=torch.float32), workspace=ws)
    both(native, apbv.apbv_cache_shared_attention, (x[:3], *args[1:]), three, return_lse=True)
    # refusals: the library's either way, the binding's handed back
    turned = dict(q_out=new(40, 8, 128), k_out=new(40, 2, 128))
    cases = [(lambda **s: apbv.apbv_cache_shared_attention(*args[:6], -1.0, q_starts=i([0, 1, 4, 5]), **outs, **s), -2),
             (lambda **s: apbv.apbv_cache_shared_attention(*args, q_starts=i([0, 1, 4, 5]), out=outs["out"], workspace=ws[:256], **s), -4),
             (lambda **s: apbv.apbv_cache_shared_attention(*args, q_starts=i([0, 1, 4]), **outs, **s), None),
             (lambda **s: apbv.apbv_cache_shared_attention(*args, group_starts=i([0, 1, 4]), **outs, **s), None),
             (lambda **s: apbv.apbv_cache_shared_attention(x, c, pt.long(), *args[3:], **outs, **s), None),
             (lambda **s: apbv.apbv_rotate(q, k, at[:2], r, **turned, **s), None),
             (lambda **s: apbv.apbv_rotate(q, k[:39], at, r, **turned, **s), None),
             (lambda **s: apbv.apbv_rotate(q[..., :64], k[..., :64], at, r, **turned, **s), None),
             (lambda **s: apbv.apbv_rotate(joint[:, :8], k, at, r, q_out=joint[:, :8], k_out=turned["k_out"], **s), None),
             (lambda **s: apbv.apbv_cache_append(c, q, k, v[:39], slots, at, r, q_out=turned["q_out"], **s), None),
             (lambda **s: apbv.apbv_cache_append(c, q, k, v, slots[1:], at, r, q_out=turned["q_out"], **s), None)]
    for case, status in cases:
        said = []
        for s in ({}, {"stream": torch.cuda.current_stream()}):
            native.said.clear()
            with pytest.raises(Exception) as err:
                case(**s)
            said.append((err.type, str(err.value)))
            assert native.said == ([] if s else [status])
        assert said[0] == said[1]
