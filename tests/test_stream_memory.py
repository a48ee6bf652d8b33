"""What the binding allocates for a call that names its stream is memory of that stream, so that neither the current stream nor a
call on a third one is given it while the call runs.  CPU: where each allocation is made is watched, the library is not called."""
import contextlib
from types import SimpleNamespace

import pytest
import torch

import paper_2601_21444_amd as apbv
from paper_2601_21444_amd import binding
from paper_2601_21444_amd import cache as module

SIDE, CURRENT = SimpleNamespace(cuda_stream=7, device=torch.device("cuda", 0)), SimpleNamespace(cuda_stream=3, device=torch.device("cuda", 0))


class Library:
    """Every entry point succeeds, every workspace is of 1000 bytes."""

    def __getattr__(self, name):
        return lambda *args: 1000 if name.endswith("_bytes") else 0


@pytest.fixture
def allocations(monkeypatch):
    """[(of the named stream, dtype, streams told of it)] of the tensors that are made."""
    made, inside = [], []

    @contextlib.contextmanager
    def on(stream):
        inside.append(stream)
        yield
        inside.pop()

    empty = torch.empty

    def watched(*args, **kw):
        t = empty(*args, **kw)
        made.append([inside[-1:] == [SIDE], t.dtype, [], t])
        return t

    def told(t, stream):
        next(m for m in made if m[3] is t)[2].append(stream)

    for where in (binding, module):
        monkeypatch.setattr(where, "load_library", Library)
    monkeypatch.setattr(module, "_rows_device", lambda t, name, stream: t.device)
    monkeypatch.setattr(module, "_check_ints", lambda *args: None)
    monkeypatch.setattr(module, "_check_table", lambda t, n, dev: (t.stride(0), t.shape[1]))
    monkeypatch.setattr(torch, "empty", watched)
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *args: CURRENT)
    monkeypatch.setattr(torch.Tensor, "record_stream", told, raising=False)
    return made


def check(made, outputs, workspaces):
    assert len(made) == outputs + workspaces
    assert all(m[0] for m in made), "an allocation of the current stream"
    for m in made:
        assert m[2] == ([] if m[1] is torch.uint8 else [CURRENT])


def test_of_the_cache(allocations):
    i = lambda *s: torch.zeros(s, dtype=torch.int32)
    page = lambda width: torch.zeros(4, 2, 16, width, dtype=torch.uint8)
    c = apbv.ApbvCache(page(32), page(32), page(2), page(2))
    q = torch.zeros(3, 4, 64, dtype=torch.bfloat16)
    apbv.apbv_cache_map(i(3), i(3), i(3, 2), i(5), i(1), 16, 4, stream=SIDE)
    check(allocations, 4, 0)
    allocations.clear()
    apbv.apbv_cache_load(c, i(3), stream=SIDE)
    check(allocations, 2, 0)
    allocations.clear()
    apbv.apbv_cache_attention(q, c, i(3, 2), i(3), 0.1, return_lse=True, stream=SIDE)
    check(allocations, 2, 1)
    allocations.clear()
    apbv.apbv_cache_attention(q, c, i(3, 2), i(3), 0.1, return_lse=True, stream=CURRENT)      # nothing to tell the current stream
    assert len(allocations) == 3 and not any(m[2] for m in allocations)


def test_of_the_prefill(allocations):
    rows = lambda *s: torch.zeros(s, dtype=torch.bfloat16)
    prob = (rows(5, 4, 64),) + tuple(rows(n, 2, 64) for n in (3, 3, 4, 4, 5, 5))
    empty = (rows(0, 2, 64),) * 2

    def calls(call, outputs, workspaces):
        allocations.clear()
        call()
        check(allocations, outputs, workspaces)
    calls(lambda: apbv.apbv_compress_kv(rows(3, 4, 64), *prob[5:], 2, return_scores=True, stream=SIDE), 4, 1)
    calls(lambda: apbv.apbv_compress_kv(rows(3, 4, 64), *prob[5:], 2, reducer="max", softmax_scale=0.1, stream=SIDE), 3, 1)
    calls(lambda: apbv.apbv_host_attention(*prob, 0.1, return_lse=True, stream=SIDE), 2, 0)
    calls(lambda: apbv.apbv_host_attention_group([prob, prob], 0.1, return_lse=True, stream=SIDE), 4, 0)
    calls(lambda: apbv.apbv_query_attention(*prob[:5], *empty, 0.1, return_lse=True, stream=SIDE), 2, 1)
    calls(lambda: apbv.apbv_merge_lse(rows(2, 5, 4, 64), torch.zeros(2, 4, 5), return_lse=True, stream=SIDE), 2, 0)
