"""A rotation's address of its tensors stays good whatever becomes of the tensor objects that it was made of (no GPU needed)."""
import ctypes

import torch

import paper_2601_21444_amd as apbv


def test_memory_is_kept_where_a_weight_is_given_other_memory():
    """A module that is moved or cast gives its parameters new memory in place: the old one would be free while the rotation names it."""
    f, w = torch.arange(32, dtype=torch.float32), torch.nn.Parameter(torch.full((64,), 3.0, dtype=torch.bfloat16))
    r = apbv.ApbvRotation(f, 64, q_weight=w, k_weight=w)
    f.data, w.data = torch.zeros(32), torch.zeros(64, dtype=torch.bfloat16)
    for held, address in ((r.inv_freq, r._struct.inv_freq), (r.q_weight, r._struct.q_weight), (r.k_weight, r._struct.k_weight)):
        assert held.data_ptr() == address
    assert list((ctypes.c_float * 32).from_address(r._struct.inv_freq)) == list(range(32))
    assert (r.q_weight == 3).all() and torch.equal(r.inv_freq, torch.arange(32, dtype=torch.float32))


def test_what_is_written_into_the_tensors_counts():
    f, w = torch.ones(32), torch.ones(64, dtype=torch.bfloat16, requires_grad=True)
    r = apbv.ApbvRotation(f, 64, k_weight=w)
    f.fill_(2.0)
    with torch.no_grad():
        w.fill_(5.0)
    assert (r.inv_freq == 2).all() and (r.k_weight == 5).all() and r.k_weight.data_ptr() == r._struct.k_weight
