"""Attention behind shared prefixes without a GPU: the refusals of the C ABI and of the binding, and how a call is cut."""
import ctypes
import os
import re

import pytest
import torch

import paper_2601_21444_amd as apbv
from paper_2601_21444_amd.binding import ApbvTensor
from tests.test_abi_host import ROOT, build_and_run_host_check, view
from tests.test_cache_host import BAD_CACHES, cache


def test_library_exports_every_symbol():
    lib = apbv.load_library()
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "apbv_shared.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(apbv_[a-z_]+)\s*\(", text)))
    assert names == ["apbv_cache_shared_attention", "apbv_cache_shared_attention_workspace_bytes"]
    for n in names:
        assert getattr(lib, n) is not None


def call(c="", groups=2, n=4, hq=8, hkv=2, d=128, q=None, ptable=0x5000, pstride=7, pblocks=7, plengths=0x6000, members=0x7000, table=0x8000,
         stride=9, blocks=9, lengths=0x9000, starts=0xa000, max_q=3, scale=0.1, out=0x10000, lse=None, ws=0x100000, ws_bytes=1 << 40):
    c = cache() if c == "" else c
    return apbv.load_library().apbv_cache_shared_attention(
        ctypes.byref(c) if c is not None else None, groups, n, hq, hkv, d, q or view(6, hq, d), ptable, pstride, pblocks, plengths, members, table,
        stride, blocks, lengths, starts, max_q, 1, scale, out, lse, ws, ws_bytes, None)


def test_bad_arguments_are_refused_without_launching():
    assert call(c=None) == -1
    for kw, status in BAD_CACHES:
        assert call(c=cache(**kw)) == status, kw
    assert call(hq=7) == -2 and call(hkv=0) == -2 and call(d=96) == -3
    assert call(n=0) == -2 and call(n=4097) == -3 and call(groups=0) == -2 and call(groups=5) == -2
    assert call(blocks=0) == -2 and call(stride=8) == -2 and call(pblocks=0) == -2 and call(pstride=6) == -2
    assert call(pblocks=(1 << 24) + 1, pstride=1 << 25) == -2
    assert call(table=None) == -1 and call(table=0x5002) == -2 and call(ptable=None) == -1 and call(ptable=0x5001) == -2
    assert call(lengths=None) == -1 and call(plengths=None) == -1 and call(plengths=0x6002) == -2 and call(members=0x7001) == -2 and call(starts=0x7002) == -2
    assert call(groups=3, members=None) == -2                         # four requests do not divide among three groups
    assert call(starts=None) == -2                                    # nor six rows among four requests
    assert call(max_q=-1) == -2 and call(scale=0.0) == -2 and call(scale=float("inf")) == -2
    assert call(out=None) == -1 and call(out=0x8008) == -2 and call(lse=0x9001) == -2
    assert call(q=ApbvTensor(0x1008, 6, 1024, 128, 0)) == -2 and call(q=ApbvTensor(0x1000, (1 << 24) + 1, 1024, 128, 0)) == -2
    assert call(n=4096, groups=4096, q=view(4096, 8, 128), pblocks=1 << 21, pstride=1 << 21) == -3       # more tiles than 32 bits number
    need = apbv.apbv_cache_shared_attention_workspace_bytes(2, 4, 6, 8, 2, 128, 3)
    assert need > 0
    assert call(ws=None) == -4 and call(ws=0x100010) == -4 and call(ws_bytes=need - 1) == -4
    assert call(q=view(0, 8, 128), out=None, ws=None) == 0            # no rows: nothing to do


def test_workspace_query():
    ws = apbv.apbv_cache_shared_attention_workspace_bytes
    assert ws(0, 4, 6, 8, 2, 128, 3) == 0 and ws(5, 4, 6, 8, 2, 128, 3) == 0 and ws(1, 4097, 6, 8, 2, 128, 3) == 0 and ws(2, 4, -1, 8, 2, 128, 3) == 0
    assert ws(2, 4, 6, 7, 2, 128, 3) == 0 and ws(2, 4, 6, 8, 2, 96, 3) == 0 and ws(2, 4, 6, 8, 2, 128, -1) == 0
    assert ws(2, 4, 6, 8, 2, 64, 1) % 256 == 0 and ws(1, 4, 1 << 24, 8, 2, 128, 1) == 0
    assert ws(1, 4, 5000, 8, 2, 128, 1) - ws(1, 4, 4000, 8, 2, 128, 1) == 1000 * 8 * 8 * 131


def test_the_cut_under_sanitizers(tmp_path):
    res = build_and_run_host_check(tmp_path, "shared_check")
    assert res.returncode == 0 and "shared checks OK" in res.stdout, res.stdout + res.stderr


def test_binding_refuses_what_does_not_fit():
    i = lambda *s: torch.zeros(s, dtype=torch.int32)
    q = torch.zeros(3, 4, 64, dtype=torch.bfloat16)
    c = apbv.apbv_cache_empty(4, 2, 64, 16, device="cpu")
    with pytest.raises(ValueError, match="must live on a GPU"):
        apbv.apbv_cache_shared_attention(q, c, i(1, 2), i(1), i(3, 2), i(3), 0.1)
