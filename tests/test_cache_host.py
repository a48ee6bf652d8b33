"""The 4-bit cache without a GPU: pins of its oracle, the refusals of the C ABI and of the binding."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

import paper_2601_21444_amd as apbv
from oracle import cache_oracle as co
from paper_2601_21444_amd.binding import ApbvCacheStruct, ApbvTensor
from tests.test_abi_host import ROOT, build_and_run_host_check, view


# ---- the oracle

def test_encoding_of_worked_blocks():
    x = np.zeros(32)
    x[:9] = [6.0, -4.0, 3.0, 2.0, -1.5, 1.0, 0.5, 0.25, -0.75]        # scale 1; 0.25 and 0.75 lie half way: to 0 and to 1
    codes, scales = co.encode(x)
    assert scales[0] == 127 and list(codes[:9]) == [7, 14, 5, 4, 11, 2, 1, 0, 10]
    assert list(co.decode(codes, scales)[:9]) == [6.0, -4.0, 3.0, 2.0, -1.5, 1.0, 0.5, 0.0, -1.0]
    x[0] = 7.0                                                        # the last maximum of this scale, held as 6
    assert co.encode(x)[1][0] == 127 and co.decode(*co.encode(x))[0] == 6.0
    x[0] = 7.03125                                                    # the next bf16 value: the scale doubles, 3.5 goes to 4
    assert co.encode(x)[1][0] == 128 and co.decode(*co.encode(x))[0] == 8.0
    assert list(co.decode(*co.encode(np.full(32, 5.0)))[:2]) == [4.0, 4.0]          # half way between 4 and 6: the even code
    assert list(co.decode(*co.encode(np.full(32, 2.5 * 2.0 ** 40)))[:1]) == [5.0 * 2.0 ** 39 * 4.0 / 5.0]     # 5 * 2^39: 4
    assert co.encode(np.zeros(32))[1][0] == 2 and co.encode(np.full(32, 2.0 ** -133))[1][0] == 2
    big = co.decode(*co.encode(np.full(32, np.inf)))
    assert big[0] == 6.0 * 2.0 ** 125 and co.decode(*co.encode(np.full(32, np.nan)))[0] == 0.0


def test_error_of_the_encoding_is_at_most_half_a_step():
    """The widest step is 2 (between 4 and 6), and a maximum of up to 7 is held as 6: at most 2^s either way."""
    x = np.random.default_rng(0).standard_normal((64, 128)) * np.exp(np.random.default_rng(1).standard_normal((64, 1)) * 8)
    codes, scales = co.encode(x)
    step = np.repeat(2.0 ** (scales.astype(float) - 127), 32, axis=-1)
    assert (np.abs(co.decode(codes, scales) - x) <= step).all()
    assert np.array_equal(co.unpack(co.pack(codes)), codes)


def test_map_of_a_worked_step():
    """Pages of 16: request 0 grows into its page, 1 leaves, 2 arrives with 20 tokens, 3 asks for more than there is."""
    table = [[5, 0], [7, 8], [0, 0], [9, 0]]
    free = [3, 0, 0, 0]
    lengths, starts, slots, left = co.cache_map([10, 20, 0, 16], [11, 0, 20, 32], table, free, 1, 16, 40)
    assert free[:3] == [3, 7, 8]
    assert table == [[5, 0], [7, 8], [8, 7], [9, 3]]
    assert lengths == [11, 0, 20, 32] and starts == [0, 1, 1, 21, 37] and left == 0
    assert slots[0] == 5 * 16 + 10 and slots[1] == 8 * 16 and slots[17] == 7 * 16 and slots[21] == 3 * 16 and slots[37] == -1
    lengths, starts, slots, left = co.cache_map([10, 0, 0, 16], [11, 0, 20, 32], [[5, 0], [0, 0], [0, 0], [9, 0]], [3], 1, 16, 40)
    assert lengths == [11, 0, 0, 16] and starts == [0, 1, 1, 21, 37] and left == 1 and slots[1:] == [-1] * 39


def test_attention_of_equal_keys_is_the_running_mean():
    v = np.random.default_rng(2).standard_normal((7, 1, 64))
    out, lse, _ = co.attention(np.ones((3, 1, 64)), np.zeros((7, 1, 64)), v, 0.3, True)
    for i, seen in enumerate((5, 6, 7)):
        np.testing.assert_allclose(out[i, 0], v[:seen, 0].mean(0), atol=1e-15)
        assert abs(lse[0, i] - np.log(seen)) < 1e-14
    out, lse, _ = co.attention(np.ones((3, 1, 64)), np.zeros((1, 1, 64)), v[:1], 0.3, True)
    assert (out[:2] == 0).all() and np.isneginf(lse[0, :2]).all() and np.array_equal(out[2], v[0])


# ---- the C ABI

def test_library_exports_every_symbol_of_the_cache():
    lib = apbv.load_library()
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "apbv_cache.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(apbv_cache_[a-z_]+)\s*\(", text)))
    assert names == ["apbv_cache_attention", "apbv_cache_attention_workspace_bytes", "apbv_cache_load", "apbv_cache_map", "apbv_cache_store"]
    for n in names:
        assert getattr(lib, n) is not None


def cache(hkv=2, d=128, page=64, n_pages=10, **kw):
    c = ApbvCacheStruct(0x100000, 0x200000, 0x300000, 0x400000, n_pages, hkv * page * d // 2, hkv * page * d // 32, page)
    for k, x in kw.items():
        setattr(c, k, x)
    return c


BAD_CACHES = [
    (dict(page=48), -3), (dict(page=8), -3), (dict(n_pages=0), -2), (dict(n_pages=1 << 31), -2), (dict(k_codes=None), -1), (dict(v_scales=None), -1),
    (dict(v_codes=0x200008), -2), (dict(k_scales=0x300004), -2), (dict(page_stride_codes=2 * 64 * 64 - 16), -2), (dict(page_stride_scales=2 * 64 * 4 + 8), -2),
    (dict(page_stride_codes=1 << 31), -3),
]


def call_attention(c="", n=2, hq=8, hkv=2, d=128, q=None, table=0x5000, stride=9, blocks=9, lengths=0x6000, starts=0x7000, max_q=3,
                   scale=0.1, out=0x8000, lse=None, ws=0x100000, ws_bytes=1 << 30):
    lib = apbv.load_library()
    c = cache() if c == "" else c
    return lib.apbv_cache_attention(ctypes.byref(c) if c is not None else None, n, hq, hkv, d, q or view(6, hq, d), table, stride, blocks,
                                    lengths, starts, max_q, 1, scale, out, lse, ws, ws_bytes, None)


def test_attention_refuses_bad_arguments_without_launching():
    assert call_attention(c=None) == -1
    for kw, status in BAD_CACHES:
        assert call_attention(c=cache(**kw)) == status, kw
    assert call_attention(hq=7) == -2 and call_attention(hkv=0) == -2 and call_attention(d=96) == -3
    assert call_attention(n=0) == -2 and call_attention(n=4097) == -3
    assert call_attention(blocks=0) == -2 and call_attention(stride=8) == -2 and call_attention(blocks=(1 << 24) + 1, stride=1 << 25) == -2
    assert call_attention(table=None) == -1 and call_attention(table=0x5002) == -2
    assert call_attention(lengths=None) == -1 and call_attention(lengths=0x6001) == -2 and call_attention(starts=0x7002) == -2
    assert call_attention(starts=None, n=4) == -2                     # 6 rows do not divide among 4 requests
    assert call_attention(max_q=-1) == -2 and call_attention(scale=0.0) == -2 and call_attention(scale=float("nan")) == -2
    assert call_attention(out=None) == -1 and call_attention(out=0x8008) == -2 and call_attention(lse=0x9001) == -2
    assert call_attention(q=ApbvTensor(0x1008, 6, 1024, 128, 0)) == -2 and call_attention(q=ApbvTensor(None, 6, 1024, 128, 0)) == -1
    assert call_attention(q=ApbvTensor(0x1000, 6, 1020, 128, 0)) == -2 and call_attention(q=ApbvTensor(0x1000, 6, 64, 128, 0)) == -2
    assert call_attention(q=ApbvTensor(0x1000, (1 << 24) + 1, 1024, 128, 0)) == -2
    assert call_attention(hq=65534, hkv=1, c=cache(hkv=1), q=ApbvTensor(0x1000, 1 << 17, 65534 * 128, 128, 0)) == -3
    assert call_attention(n=4096, q=view(4096, 8, 128), blocks=1 << 21, stride=1 << 21) == -3       # more tiles than 32 bits number
    need = apbv.apbv_cache_attention_workspace_bytes(2, 6, 8, 2, 128, 3)
    assert need > 0
    assert call_attention(ws=None) == -4 and call_attention(ws=0x100010) == -4 and call_attention(ws_bytes=need - 1) == -4
    assert call_attention(q=view(0, 8, 128), out=None, ws=None) == 0        # no rows: nothing to do


def test_attention_workspace_query():
    ws = apbv.apbv_cache_attention_workspace_bytes
    assert ws(0, 6, 8, 2, 128, 3) == 0 and ws(4097, 6, 8, 2, 128, 3) == 0 and ws(2, -1, 8, 2, 128, 3) == 0
    assert ws(2, 6, 7, 2, 128, 3) == 0 and ws(2, 6, 8, 2, 96, 3) == 0 and ws(2, 6, 8, 2, 128, -1) == 0
    assert ws(2, 6, 8, 2, 64, 1) % 256 == 0


def test_a_request_has_no_more_rows_than_there_are():
    # (2^39 rows by max_q alone: a multiple of 2^32 row tiles)
    ws = apbv.apbv_cache_attention_workspace_bytes
    assert ws(1, 1, 32768, 1, 64, 1 << 24) == ws(1, 1, 32768, 1, 64, 1) > 0
    assert ws(2, 6, 8, 2, 128, 1 << 24) == ws(2, 6, 8, 2, 128, 6)


def test_store_and_load_refuse_bad_arguments_without_launching():
    lib = apbv.load_library()

    def store(c="", hkv=2, d=128, k=None, v=None, slots=0x5000):
        c = cache() if c == "" else c
        return lib.apbv_cache_store(ctypes.byref(c) if c is not None else None, hkv, d, k or view(5, hkv, d), v or view(5, hkv, d), slots, None)

    def load(c="", hkv=2, d=128, n=5, slots=0x5000, k=0x6000, v=0x7000):
        c = cache() if c == "" else c
        return lib.apbv_cache_load(ctypes.byref(c) if c is not None else None, hkv, d, n, slots, k, v, None)
    assert store(c=None) == -1 and load(c=None) == -1
    for kw, status in BAD_CACHES:
        assert store(c=cache(**kw)) == status and load(c=cache(**kw)) == status, kw
    assert store(hkv=0) == -2 and store(d=96) == -3 and load(hkv=70000) == -2 and load(d=32) == -3
    assert store(v=view(4, 2, 128)) == -2 and store(slots=None) == -1 and store(slots=0x5002) == -2
    assert store(k=ApbvTensor(0x1008, 5, 256, 128, 0)) == -2 and store(k=ApbvTensor(0x1000, 5, 256, 60, 0)) == -2
    assert load(n=-1) == -2 and load(n=(1 << 24) + 1) == -2 and load(slots=None) == -1 and load(k=None) == -1 and load(v=0x7008) == -2
    assert store(k=view(0, 2, 128), v=view(0, 2, 128), slots=None) == 0 and load(n=0, slots=None, k=None, v=None) == 0


def test_launches_of_more_threads_than_32_bits_count_are_refused():
    lib = apbv.load_library()
    many = 1 << 24
    c = cache(hkv=16)
    assert lib.apbv_cache_load(ctypes.byref(c), 16, 128, many, 0x5000, 0x6000, 0x7000, None) == -3
    assert lib.apbv_cache_store(ctypes.byref(c), 16, 128, view(many, 16, 128), view(many, 16, 128), 0x5000, None) == -3
    assert call_attention(c=cache(hkv=4), hq=4, hkv=4, q=view(many, 4, 128), starts=0x7000) == -3       # 2^26 rows of the output
    wide = cache(hkv=4096, page=16, d=64)
    assert call_attention(c=wide, n=4096, hq=4096, hkv=4096, d=64, q=view(1, 4096, 64), blocks=1, stride=1) == -3


def test_map_refuses_bad_arguments_without_launching():
    lib = apbv.load_library()

    def call(n=3, page=16, blocks=8, old=0x1000, new=0x2000, table=0x3000, stride=8, pages=0x4000, capacity=20, count=0x5000, most=10,
             lengths=0x6000, starts=0x7000, slots=0x8000, left=0x9000):
        return lib.apbv_cache_map(n, page, blocks, old, new, table, stride, pages, capacity, count, most, lengths, starts, slots, left, None)
    assert call(n=0) == -2 and call(n=4097) == -3 and call(page=24) == -3 and call(blocks=0) == -2 and call(blocks=1 << 27, stride=1 << 27) == -2
    assert call(stride=7) == -2 and call(capacity=-1) == -2 and call(most=-1) == -2 and call(most=(1 << 24) + 1) == -2
    for name in ("old", "new", "table", "pages", "count", "lengths", "starts", "slots", "left"):
        assert call(**{name: None}) == -1, name
        assert call(**{name: 0x8002}) == -2, name
    assert call(capacity=1 << 27) == -2 and call(page=256, capacity=1 << 23) == -2        # more pages than a pool can have
    assert call(lengths=0x2000) == -2                                 # the new lengths are still read while these are written


def test_cache_validation_under_sanitizers(tmp_path):
    res = build_and_run_host_check(tmp_path, "cache_check")
    assert res.returncode == 0 and "cache checks OK" in res.stdout, res.stdout + res.stderr


# ---- the binding

def test_binding_refuses_what_does_not_fit():
    i = lambda *s: torch.zeros(s, dtype=torch.int32)
    q = torch.zeros(3, 4, 64, dtype=torch.bfloat16)
    c = apbv.apbv_cache_empty(4, 2, 64, 16, device="cpu")
    assert (c.n_pages, c.n_kv_heads, c.page_size, c.head_dim) == (4, 2, 16, 64)
    with pytest.raises(ValueError):
        apbv.apbv_cache_empty(4, 2, 64, 48, device="cpu")
    with pytest.raises(ValueError, match="must live on a GPU"):
        apbv.apbv_cache_attention(q, c, i(3, 2), i(3), 0.1)
    with pytest.raises(ValueError, match="must live on a GPU"):
        apbv.apbv_cache_store(c, q[:, :2], q[:, :2], i(3))
    with pytest.raises(ValueError, match="must live on a GPU"):
        apbv.apbv_cache_load(c, i(3))
    with pytest.raises(ValueError, match="must live on a GPU"):
        apbv.apbv_cache_map(i(3), i(3), i(3, 2), i(5), i(1), 16, 4)


class Elsewhere:
    """What the binding asks of a tensor's place: a second GPU's."""
    is_cuda, device = True, torch.device("cuda", 1)


def test_tensors_of_another_device_than_the_streams_are_refused(monkeypatch):
    from paper_2601_21444_amd import cache as module
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    with pytest.raises(ValueError, match="the stream of the call on cuda:0"):
        module._rows_device(Elsewhere, "q", None)
    stream = type("Stream", (), {"device": torch.device("cuda", 0)})
    with pytest.raises(ValueError, match="the stream of the call on cuda:0"):
        module._rows_device(Elsewhere, "q", stream)
    stream.device = torch.device("cuda", 1)
    assert module._rows_device(Elsewhere, "q", stream) == torch.device("cuda", 1)
