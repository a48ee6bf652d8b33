"""Positions without a GPU: pins of the oracle, the refusals of the C ABI and of the binding."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

import paper_2601_21444_amd as apbv
from oracle import positions_oracle as po
from paper_2601_21444_amd.binding import ApbvTensor
from paper_2601_21444_amd.positions import ApbvRotationStruct
from tests.test_abi_host import ROOT, build_and_run_host_check, view
from tests.test_cache_host import BAD_CACHES, cache


# ---- the oracle

def test_rotation_of_worked_rows():
    x = np.zeros((1, 1, 64))
    x[0, 0, :4] = [1.0, 2.0, 3.0, 4.0]
    x[0, 0, 8:10] = [5.0, 6.0]
    quarter = np.pi / 2
    f = [quarter, 2 * quarter, 0.0, 1.0, 0.0, 0.0, 0.0, 0.0]
    axis = [0, 1, 0, 0, 0, 0, 0, 0]
    y, _ = po.rotate(x, [[1], [3]], f, axis)                          # pairs (0, 8), (1, 9), ...: a quarter turn, three halves of a turn
    np.testing.assert_allclose(y[0, 0, [0, 8, 1, 9, 2]], [-5.0, 1.0, -2.0, -6.0, 3.0], atol=1e-14)
    np.testing.assert_allclose(y[0, 0, 3], 4.0 * np.cos(1.0), atol=1e-14)
    y, _ = po.rotate(x, [[1], [3]], f, axis, adjacent=True)           # pairs (0, 1), (2, 3)
    np.testing.assert_allclose(y[0, 0, :4], [-2.0, 1.0, -3.0, -4.0], atol=1e-14)
    y, _ = po.rotate(x, [[0], [0]], f, axis, weight=np.full(64, 2.0), eps=0.0)
    np.testing.assert_allclose(y[0, 0], 2.0 * x[0, 0] / np.sqrt(91.0 / 64), atol=1e-14)


def test_rotation_keeps_lengths_and_relative_positions():
    rng = np.random.default_rng(0)
    a, b = rng.standard_normal((2, 5, 3, 64))
    f, axis = 1e4 ** (-np.arange(32) / 32), [i % 3 for i in range(32)]
    at = rng.integers(-1000, 1000, (3, 5))
    ra, _ = po.rotate(a, at, f, axis)
    rb, _ = po.rotate(b, at + 77, f, axis)
    qa, _ = po.rotate(a, at + 12345, f, axis)
    qb, _ = po.rotate(b, at + 77 + 12345, f, axis)
    np.testing.assert_allclose((ra * ra).sum(-1), (a * a).sum(-1), rtol=1e-12)
    np.testing.assert_allclose((ra * rb).sum(-1), (qa * qb).sum(-1), atol=1e-10)
    back, _ = po.rotate(ra, -at, f, axis)
    np.testing.assert_allclose(back, a, atol=1e-12)


# ---- the C ABI

def test_library_exports_every_symbol():
    lib = apbv.load_library()
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "apbv_positions.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(apbv_[a-z_]+)\s*\(", text)))
    assert names == ["apbv_cache_append", "apbv_rotate"]
    for n in names:
        assert getattr(lib, n) is not None


def rotation(rot=64, **kw):
    r = ApbvRotationStruct(0x9000, 0xa000, 0xb000, 1e-6, rot, 3, 0, (ctypes.c_uint8 * 64)(*([0, 1, 2] * 21 + [0])))
    for k, x in kw.items():
        setattr(r, k, x)
    return r


BAD_ROTATIONS = [
    (dict(rot_dim=0), -2), (dict(rot_dim=24), -2), (dict(rot_dim=144), -2), (dict(rot_dim=-16), -2), (dict(n_axes=0), -2), (dict(n_axes=5), -2),
    (dict(n_axes=2), -2), (dict(adjacent=2), -2), (dict(adjacent=-1), -2), (dict(eps=-1e-6), -2), (dict(eps=float("nan")), -2),
    (dict(eps=float("inf")), -2), (dict(inv_freq=None), -1), (dict(inv_freq=0x9002), -2), (dict(q_weight=0xa008), -2), (dict(k_weight=0xb002), -2),
]
NONE = ApbvTensor(None, 0, 0, 0, 0)


def call_rotate(hq=8, hkv=2, d=128, r="", q=None, k=None, positions=0x5000, stride=5, q_out=0x100000, k_out=0x200000):
    r = rotation() if r == "" else r
    return apbv.load_library().apbv_rotate(hq, hkv, d, ctypes.byref(r) if r is not None else None, q or view(5, hq, d), k or view(5, hkv, d),
                                           positions, stride, q_out, k_out, None)


def test_rotate_refuses_bad_arguments_without_launching():
    assert call_rotate(r=None) == -1 and call_rotate(d=96) == -3 and call_rotate(hq=0) == -2 and call_rotate(hkv=65536) == -2
    for kw, status in BAD_ROTATIONS:
        assert call_rotate(r=rotation(**kw)) == status, kw
    assert call_rotate(d=64, r=rotation(rot=80)) == -2
    assert call_rotate(q=view(4, 8, 128)) == -2 and call_rotate(positions=None) == -1 and call_rotate(positions=0x5002) == -2
    assert call_rotate(stride=-1) == -2 and call_rotate(q_out=None) == -1 and call_rotate(k_out=0x200008) == -2
    assert call_rotate(q=ApbvTensor(0x1008, 5, 1024, 128, 0)) == -2 and call_rotate(k=ApbvTensor(None, 5, 256, 128, 0)) == -1
    assert call_rotate(q=ApbvTensor(0x1000, 5, 1024, 64, 0)) == -2 and call_rotate(q=ApbvTensor(0x1000, -1, 1024, 128, 0)) == -2
    assert call_rotate(q=ApbvTensor(0x1000, 5, 2048, 128, 0), q_out=0x1000) == -2      # in place, but not dense
    assert call_rotate(hq=64, q=view(1 << 23, 64, 128), k=NONE, k_out=None) == -3      # 2^29 rows
    assert call_rotate(q=NONE, k=NONE, hq=0, hkv=0, positions=None, q_out=None, k_out=None) == 0       # nothing to do


def call_append(c="", hq=8, hkv=2, d=128, r="", q=None, k=None, v=None, positions=0x5000, stride=5, slots=0x6000, q_out=0x100000):
    c, r = cache() if c == "" else c, rotation() if r == "" else r
    return apbv.load_library().apbv_cache_append(ctypes.byref(c) if c is not None else None, hq, hkv, d, ctypes.byref(r) if r is not None else None,
                                                 q or view(5, hq, d), k or view(5, hkv, d), v or view(5, hkv, d), positions, stride, slots, q_out, None)


def test_append_refuses_bad_arguments_without_launching():
    assert call_append(c=None) == -1 and call_append(r=None) == -1 and call_append(d=96) == -3 and call_append(hkv=0) == -2 and call_append(hq=0) == -2
    for kw, status in BAD_CACHES:
        assert call_append(c=cache(**kw)) == status, kw
    for kw, status in BAD_ROTATIONS:
        assert call_append(r=rotation(**kw)) == status, kw
    assert call_append(v=view(4, 2, 128)) == -2 and call_append(q=view(4, 8, 128)) == -2 and call_append(slots=None) == -1
    assert call_append(slots=0x6002) == -2 and call_append(positions=None) == -1 and call_append(stride=-5) == -2
    assert call_append(q_out=None) == -1 and call_append(q_out=0x100004) == -2 and call_append(q=ApbvTensor(0x1000, 5, 2048, 128, 0), q_out=0x1000) == -2
    assert call_append(hq=60, q=view(1 << 23, 60, 128), k=view(1 << 23, 4, 128), v=view(1 << 23, 4, 128), hkv=4, c=cache(hkv=4)) == -3
    many = 1 << 24                                                    # 15 * 2^20 workgroups of keys and values, 2^21 of queries
    assert call_append(hkv=15, hq=15, c=cache(hkv=15), q=view(many, 15, 128), k=view(many, 15, 128), v=view(many, 15, 128)) == -3
    assert call_append(q=NONE, k=view(0, 2, 128), v=view(0, 2, 128), slots=None, positions=None, q_out=None) == 0


def test_positions_validation_under_sanitizers(tmp_path):
    res = build_and_run_host_check(tmp_path, "positions_check")
    assert res.returncode == 0 and "positions checks OK" in res.stdout, res.stdout + res.stderr


# ---- the binding

def test_rotations_that_do_not_fit_are_refused():
    f = torch.ones(32)
    w = torch.ones(64, dtype=torch.bfloat16)
    r = apbv.ApbvRotation(f, 64, axis=[i % 3 for i in range(32)], q_weight=w)
    assert (r.n_axes, r.rot_dim, r.head_dim) == (3, 64, 64)
    for error, args, kw in ((ValueError, (f, 96), {}), (TypeError, (f.double(), 64), {}), (ValueError, (torch.ones(64)[::2], 64), {}),
                            (ValueError, (torch.ones(12), 64), {}), (ValueError, (torch.ones(40), 64), {}), (ValueError, (f, 64), dict(axis=[0] * 31)),
                            (ValueError, (f, 64), dict(axis=[4] * 32)), (TypeError, (f, 64), dict(axis=[0.5] * 32)), (ValueError, (f, 64), dict(axis=[-1] * 32)),
                            (TypeError, (f, 64), dict(q_weight=w.float())), (ValueError, (f, 128), dict(k_weight=w)),
                            (ValueError, (f, 64), dict(k_weight=torch.ones(65, dtype=torch.bfloat16)[1:])),
                            (ValueError, (f, 64), dict(eps=-1.0)), (ValueError, (f, 64), dict(eps=float("nan")))):
        with pytest.raises(error):
            apbv.ApbvRotation(*args, **kw)


def test_binding_refuses_what_does_not_fit():
    f = torch.ones(32)
    r = apbv.ApbvRotation(f, 64)
    q = torch.zeros(3, 4, 64, dtype=torch.bfloat16)
    i = lambda *s: torch.zeros(s, dtype=torch.int32)
    c = apbv.apbv_cache_empty(4, 2, 64, 16, device="cpu")
    with pytest.raises(ValueError, match="must live on a GPU"):
        apbv.apbv_rotate(q, q[:, :2], i(3), r)
    with pytest.raises(ValueError, match="one of them is needed"):
        apbv.apbv_rotate(None, None, i(3), r)
    with pytest.raises(ValueError, match="must live on a GPU"):
        apbv.apbv_cache_append(c, q, q[:, :2], q[:, :2], i(3), i(3), r)
