"""Decode attention and its weights with NaN and infinities in places that count: against
the 64-bit oracle."""
import numpy as np
import pytest
import torch

from paper_2607_00466_amd import binding as B
from tests import attention_util as U
from tests import gpu_util as G
from tests.attention_edges import INF, NAN, SHAPES, agree, cache_of, decode, reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lens,Hq,Hkv,D,shared,fp8", SHAPES)
@pytest.mark.parametrize("sunk", [False, True])
@pytest.mark.parametrize("value", [NAN, INF])
def test_queries_that_are_not_finite(lens, Hq, Hkv, D, shared, fp8, sunk, value):
    G.say(f"case: a head's query with {value}, lens={lens[:5]} heads {Hq}/{Hkv} D={D} shared={shared} sinks={sunk}")
    cache, clean = cache_of(lens, Hkv, D, shared, fp8), U.queries(len(lens), Hq, D)
    sinks = torch.randn(Hq, device="cuda") if sunk else None
    q = clean.clone()
    for r in range(len(lens)):
        q[r, (3 * r + 1) % Hq, 5 * r % D] = value
    mass = reference(cache, clean, shared, sinks)[2]
    agree(decode(cache, q, shared, sinks), reference(cache, q, shared, sinks), cache, clean, mass)


@pytest.mark.parametrize("lens,Hq,Hkv,D,shared,fp8", SHAPES)
def test_visible_keys_and_values_that_are_nan(lens, Hq, Hkv, D, shared, fp8):
    G.say(f"case: a key and a value of NaN in cached slots, lens={lens[:5]} heads {Hq}/{Hkv} D={D} shared={shared}")
    cache, q = cache_of(lens, Hkv, D, shared, fp8), U.queries(len(lens), Hq, D)
    clean = reference(cache, q, shared)
    first = next(r for r, n in enumerate(lens) if n > 0)
    last = max(r for r, n in enumerate(lens) if n > 0)
    for which, plain, r, j in (("k", "k_np", first, 0), ("v", "v_np", first, lens[first] - 1), ("k", "k_np", last, lens[last] - 1)):
        b = int(cache.table_np[r, j // 16])
        getattr(cache, which)[b, Hkv - 1, j % 16, D - 3] = NAN
        getattr(cache, plain)[b, Hkv - 1, j % 16, D - 3] = NAN
        agree(decode(cache, q, shared), reference(cache, q, shared), cache_of(lens, Hkv, D, shared, fp8), q, clean[2])


def test_sinks_that_are_nan():
    G.say("case: a head's sink is NaN")
    for lens, shared in (([0, 9, 300], ()), ([9000, 0], ()), ([200, 190, 0], ((0, 3, 128),))):
        cache, q = cache_of(lens, 2, 64, shared, False), U.queries(len(lens), 4, 64)
        sinks = torch.tensor([0.5, NAN, -1.0, 2.0], device="cuda")
        got, want = decode(cache, q, shared, sinks), reference(cache, q, shared, sinks)
        agree(got, want, cache, q, reference(cache, q, shared)[2])


@pytest.mark.parametrize("shared", [(), ((0, 3, 128),)])
def test_weights_of_a_head_without_a_sum_are_nan(shared):
    G.say(f"case: the weights that a NaN sink gives, shared={shared}")
    lens = [300, 170, 0]
    cache, q = cache_of(lens, 2, 128, shared, False), U.queries(3, 8, 128)
    sinks = torch.randn(8, device="cuda")
    sinks[1] = NAN
    gs, pl, _, _ = U.groups_of(shared, 3)
    _, lse = U.run_decode(cache, q, shared, sinks, check=False)
    w = torch.zeros((3, 2, cache.N), device="cuda")
    B.moe_attn_weights(q, cache.k, cache.table, cache.lens, lse, cache.dims(8), None, w, gs, pl)
    torch.cuda.synchronize()
    for r, n in enumerate(lens):
        assert w[r, 0, :n].isnan().all() and torch.isfinite(w[r, 1, :n]).all() and not w[r, :, n:].any()
