"""moe_attn_decode over pages of 8-bit integers, with queries, sinks and scales that are not
finite, or far from 1, in places that count: against the 64-bit oracle."""
import numpy as np
import pytest
import torch

from tests import attention_util as U
from tests.attention_edges import INF, LOWEST, NAN, SHAPES, agree, decode, reference
from tests.test_gpu_attention_int8 import Cache

pytestmark = pytest.mark.gpu

SHAPES = [s[:5] for s in SHAPES]


def cache_of(lens, Hkv, D, shared):
    return Cache(lens, Hkv, D, 16, seed=len(lens) + D, shared=shared, max_blocks=-(-max(lens) // 16) + 1)


@pytest.mark.parametrize("lens,Hq,Hkv,D,shared", SHAPES)
@pytest.mark.parametrize("sunk", [False, True])
@pytest.mark.parametrize("value", [NAN, INF])
def test_queries_that_are_not_finite(lens, Hq, Hkv, D, shared, sunk, value):
    cache, clean = cache_of(lens, Hkv, D, shared), U.queries(len(lens), Hq, D)
    sinks = torch.randn(Hq, device="cuda") if sunk else None
    q = clean.clone()
    for r in range(len(lens)):
        q[r, (3 * r + 1) % Hq, 5 * r % D] = value
    mass = reference(cache, clean, shared, sinks)[2]
    agree(decode(cache, q, shared, sinks), reference(cache, q, shared, sinks), cache, clean, mass)


@pytest.mark.parametrize("lens,Hq,Hkv,D,shared", SHAPES)
@pytest.mark.parametrize("which", ["k", "v"])
def test_pages_that_are_nan(lens, Hq, Hkv, D, shared, which):
    """The scale of a page of which only the first slot counts, and of one in the middle."""
    cache, q = cache_of(lens, Hkv, D, shared), U.queries(len(lens), Hq, D)
    clean = reference(cache, q, shared)[2]
    for r in (next(r for r, n in enumerate(lens) if n > 0), max(r for r, n in enumerate(lens) if n > 0)):
        b = int(cache.table_np[r, (lens[r] - 1) // 16])
        getattr(cache, which + "_scale")[b, Hkv - 1] = NAN
        getattr(cache, which + "_np")[b, Hkv - 1] = NAN
        agree(decode(cache, q, shared), reference(cache, q, shared), cache_of(lens, Hkv, D, shared), q, clean)


@pytest.mark.parametrize("lens,Hq,Hkv,D,shared", SHAPES)
def test_sinks_that_are_switched_off(lens, Hq, Hkv, D, shared):
    cache, q = cache_of(lens, Hkv, D, shared), U.queries(len(lens), Hq, D)
    empty = np.array(lens) == 0
    none = decode(cache, q, shared)
    for value in (-INF, LOWEST):
        sinks = torch.randn(Hq, device="cuda")
        sinks[::2] = value
        got, want = decode(cache, q, shared, sinks), reference(cache, q, shared, sinks)
        agree(got, want, cache, q, want[2])
        assert not got[0][empty].any() and np.array_equal(got[0][~empty, ::2], none[0][~empty, ::2])


@pytest.mark.parametrize("amp", [1e-30, 1e-20, 1e20, 1e30])
@pytest.mark.parametrize("lens,Hq,Hkv,D,shared", [SHAPES[0], SHAPES[4], ([4000, 300], 8, 2, 64, ())])
def test_values_far_from_one(lens, Hq, Hkv, D, shared, amp):
    """A page's scale multiplies the weights before they are split in two bf16 parts."""
    cache, q = cache_of(lens, Hkv, D, shared), U.queries(len(lens), Hq, D)
    cache.v_scale = cache.v_scale * amp
    cache.v_np = cache.v.cpu().numpy() * cache.v_scale.double().cpu().numpy()[:, :, None, None]
    U.run_decode(cache, q, shared)
