"""The output of decode attention is the exact one rounded once: its weights keep more
bits than a bf16 in the product with the values."""
import numpy as np
import pytest
import torch

from oracle import attention as A
from tests import attention_util as U
from tests import gpu_util as G

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lens,Hq,Hkv,D,shared,fp8", [
    ([1, 2, 17, 700], 8, 2, 128, (), False),
    ([900, 33], 16, 2, 256, (), False),
    ([1000, 64], 64, 8, 64, (), True),
    ([700, 690, 640], 32, 4, 128, ((0, 3, 640),), False),
    ([640] * 20, 8, 1, 64, ((0, 20, 512),), True),
    ([600] * 5, 16, 2, 256, ((0, 5, 592),), False),
])
def test_weights_in_the_product_with_values(lens, Hq, Hkv, D, shared, fp8):
    G.say(f"case: the weights' bits, lens={lens[:5]} heads {Hq}/{Hkv} D={D} shared={shared} fp8={fp8}")
    cache = U.Cache(lens, Hkv, D, 16, fp8, seed=D, shared=shared, max_blocks=-(-max(lens) // 16) + 1)
    q = U.queries(len(lens), Hq, D, amp=1.0)
    out, _ = U.run_decode(cache, q, shared)
    _, _, gs, pl = U.groups_of(shared, len(lens))
    want, _, mass = A.decode(q.double().cpu().numpy(), cache.k_np, cache.v_np, cache.table_np, cache.lens_np, D ** -0.5, gs, pl)
    # a weight in two bf16 parts is off by at most 2^-15 of itself (the second part's rounding, of what is
    # below 2^-7 of the weight); the sums by a rounding to fp32 a slot; the scores as in check_decode; then
    # one rounding of the result
    rel = np.expm1(2 * U.score_bound(q, cache, D ** -0.5)) + (max(lens) + 64) * U.U_FP32
    tol = (2.0 ** -15 + rel) * mass * 1.01 + U.U_BF16 * 1.01 * np.abs(want)
    off = np.abs(out.double().cpu().numpy() - want)
    assert (off <= tol).all(), f"out off by {(off / tol).max():.3g} of its bound"
