"""Kernels run on the stream's device: a cache on another one is refused before the launch,
by every call that reads or writes it."""
from types import SimpleNamespace

import pytest
import torch

from paper_2607_00466_amd import binding as B
from tests.kv_cache_util import i32

pytestmark = pytest.mark.gpu

KINDS = {"bf16": torch.bfloat16, "fp8": torch.float8_e4m3fn, "int8": torch.int8}


def calls(kind):
    """Each call's name and the call, on a cache of two pages."""
    d = B.attn_dims(1, 2, 2, 64, 16, 2, 2, KINDS[kind])
    k, v = (torch.zeros((2, 2, 16, 64), device="cuda").to(KINDS[kind]) for _ in "kv")
    s = torch.ones((2, 2), device="cuda") if kind == "int8" else None
    q, rows = torch.zeros((1, 2, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros((1, 2, 64), device="cuda")
    table, lens, pos = i32([[0, 1]]), i32([3]), i32([[0]])
    lse, w, tokens = torch.zeros((1, 2), device="cuda"), torch.zeros((1, 2, 32), device="cuda"), torch.zeros((1, 2, 32), dtype=torch.int32, device="cuda")
    turns = pos, i32([]), torch.zeros((1, 0), device="cuda"), torch.zeros((1, 0), device="cuda")
    ws, out = B.attn_workspace(d), torch.empty_like(q)
    every = {
        "decode": lambda **kw: B.moe_attn_decode(q, k, v, table, lens, d, out, lse, ws, k_scale=s, v_scale=s, **kw),
        "fork": lambda **kw: B.moe_kv_fork(i32([]), i32([]), i32([]), table, lens, d, k, v, s, s, **kw),
        "compact": lambda **kw: B.moe_kv_compact(i32([0, 1]), table, table, d, k, v, s, s, **kw),
    }
    if kind == "int8":
        every["append"] = lambda **kw: B.moe_kv_append_int8(rows, rows, rows, *turns, i32([0, 1]), table, lens, d, out, k, v, s, s, **kw)
        return every
    every["append"] = lambda **kw: B.moe_kv_append(rows, rows, rows, *turns, i32([3]), d, out, k, v, **kw)
    every["append_norm"] = lambda **kw: B.moe_kv_append_norm(rows, rows, rows, *turns, i32([3]), d, out, k, v, None, None, **kw)
    every["weights"] = lambda **kw: B.moe_attn_weights(q, k, table, lens, lse, d, None, w, **kw)
    every["evict"] = lambda **kw: B.moe_kv_evict(w, tokens, lens, lens, table, d, 4, 1, k, v, i32([0] * 8), i32([0]), w.clone(), tokens.clone(), **kw)
    return every


@pytest.mark.parametrize("kind", KINDS)
def test_a_cache_on_another_device_is_named(kind, monkeypatch):
    every = calls(kind)
    stream = torch.cuda.Stream()
    for call in every.values():
        call()
        call(stream=stream)
    torch.cuda.synchronize()
    # (a stream of the second of two devices; its address is not looked at)
    there = SimpleNamespace(device=torch.device("cuda", 1), cuda_stream=None)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    for name, call in every.items():
        with pytest.raises(ValueError, match="k_cache: is on cuda:0, and the current device is cuda:1"):
            call()
        with pytest.raises(ValueError, match="k_cache: is on cuda:0, and the (stream on|current device is) cuda:1"):
            call(stream=there)
