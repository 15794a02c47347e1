"""Two threads on one cache: an attention call takes the workspace of its own sizes (no kernel is launched here)."""
import sys

import pytest
import torch

from paper_2505_09142_amd import _elis as E
from paper_2505_09142_amd import device as D


@pytest.mark.parametrize("keys,other", [(100, 16000), (16000, 100)])
def test_another_call_between_any_two_lines(monkeypatch, keys, other):
    """A call of other sizes, as another thread would make it, before every line of a call."""
    seen = []

    def attention(c, q, qs, cu, n, total, max_q, blocks, br, bc, rows, lens, max_kv, heads, scale, window, out, os_, ws, wsb, stream):
        seen.append((wsb, E.elis_kv_attention_workspace_bytes(n, total, max_q, max_kv, heads, 2, 64)))
        return E.ELIS_OK

    monkeypatch.setattr(E, "elis_kv_attention", attention)
    monkeypatch.setattr(D, "_dev", lambda: -1)
    monkeypatch.setattr(D, "_stream", lambda stream: 0)
    cache = D.KVCache(1024, 16, 2, 64, buf=torch.zeros(E.elis_kv_cache_bytes(1024, 16, 2, 64) + 256, dtype=torch.uint8))
    q, blocks = torch.zeros((1, 4, 64), dtype=torch.bfloat16), torch.zeros((1, 1024), dtype=torch.int32)
    cu, lens = torch.tensor([0, 1], dtype=torch.int32), torch.tensor([5], dtype=torch.int32)

    def call(max_kv):
        cache.attention(q, cu, lens, blocks, 1, max_kv)

    inside, between = False, 0

    def trace(frame, event, arg):
        nonlocal inside, between
        if frame.f_code is D.KVCache.attention.__code__ and not inside:
            if event == "line":
                inside, between = True, between + 1
                call(other)
                inside = False
            return trace
        return None

    call(keys)
    before = sys.gettrace()
    sys.settrace(trace)
    try:
        call(keys)
    finally:
        sys.settrace(before)
    assert between > 20 and len({need for _, need in seen}) == 2
    assert all(got == need for got, need in seen)
