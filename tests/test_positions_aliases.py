"""Positions: outputs that are another's input are refused (no GPU needed)."""
from tests.test_abi_host import view
from tests.test_positions_host import NONE, call_append, call_rotate


def test_an_output_that_is_the_others_is_refused():
    q, k = view(5, 2, 128, ptr=0x1000), view(5, 2, 128, ptr=0x8000)
    both = dict(hq=2, hkv=2, q=q, k=k)
    assert call_rotate(**both, q_out=0x8000, k_out=0x1000) == -2          # exchanged
    assert call_rotate(**both, q_out=0x8000) == -2 and call_rotate(**both, k_out=0x1000) == -2
    assert call_rotate(**both, q_out=0x20000, k_out=0x20000) == -2
    assert call_rotate(hq=2, hkv=2, q=q, k=q, q_out=0x1000) == -2         # in place, and read as keys too
    # the answer is the same where queries or keys are left out and an address that is not read says otherwise
    assert call_rotate(hq=0, hkv=0, q=NONE, k=NONE, positions=None, q_out=0x8000, k_out=0x8000) == 0
    v = view(5, 2, 128, ptr=0x10000)
    assert call_append(q=view(5, 2, 128, ptr=0x30000), hq=2, k=k, v=v, q_out=0x8000) == -2
    assert call_append(q=view(5, 2, 128, ptr=0x30000), hq=2, k=k, v=v, q_out=0x10000) == -2
