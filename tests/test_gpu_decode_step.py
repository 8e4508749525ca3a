"""The decode-step example: attention, MoE layer and eviction together, each step
against the oracle on what the cache holds."""
import numpy as np
import pytest
import torch

from examples import decode_step as E
from oracle import attention as A
from paper_2607_00466_amd import synth
from tests import attention_util as U
from tests import gpu_util as G

pytestmark = pytest.mark.gpu


class View:
    """What check_decode needs to know of a cache."""

    def __init__(self, w):
        self.D = w.heads.D
        scale = 1.0 if w.k_scale is None else float(w.k_scale[0])
        self.k_np, self.v_np = (c.cpu().double().numpy() * scale for c in (w.k_cache, w.v_cache))


@pytest.mark.parametrize("fp8", [False, True])
def test_steps_match_the_oracle(fp8):
    G.say(f"case: 8 decode steps of 6 requests in 2 groups, evicting from the third on, fp8={fp8}")
    w = E.Worker(synth.SHAPES["tiny"], E.Heads(8, 2, 64), R=6, groups=2, prefix=32, own=20, budget=54, steps=8, recent=4, fp8=fp8)
    table, gs, pl = w.table.cpu().numpy(), w.group_start.tolist(), w.prefix_len.tolist()
    x = torch.randn((6, w.shape.H), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    scale = w.heads.D ** -0.5
    for step in range(8):
        out = w.attend(x)
        torch.cuda.synchronize()
        cache, lens = View(w), w.lens.cpu().numpy()
        assert lens.tolist() == [min(53 + step, 55)] * 6
        q = w.q.double().cpu().numpy()
        ref = A.decode(q, cache.k_np, cache.v_np, table, lens, scale, gs, pl)
        U.check_decode(out, w.lse, w.q, cache, scale, ref)
        before = w.weights.double().cpu().numpy()
        pos, seen = w.pos.cpu().numpy(), w.seen.cpu().numpy()
        held = [c.float().cpu().numpy() for c in (w.k_cache, w.v_cache)]
        w.evict()
        torch.cuda.synchronize()
        # the step's weights sum to the query heads of each kv head, wherever they moved
        kept = np.minimum(lens, 54)
        assert w.lens.tolist() == kept.tolist()
        added = A.weights(q, cache.k_np, table, lens, w.lse.double().cpu().numpy(), scale, before, before, gs, pl)
        src = w.src.cpu().numpy()
        for r in range(6):
            for h in range(2):
                n = int(kept[r])
                assert np.allclose(w.weights[r, h, :n].double().cpu().numpy(), added[r, h, src[r, h, :n]], rtol=1e-5, atol=1e-6)
                assert np.array_equal(w.pos[r, h, :n].cpu().numpy(), pos[r, h, src[r, h, :n]])
                # protected and recent tokens are still there
                now = set(w.pos[r, h, :n].tolist())
                assert set(range(32)) | set(range(int(seen[r]) - 4, int(seen[r]))) <= now
        for c, ref_c in zip((w.k_cache, w.v_cache), held):
            assert np.array_equal(c.float().cpu().numpy(), A.moved(ref_c, table, src, lens, 54))


def test_example_runs():
    G.say("case: the decode-step example, tiny shape, 3 steps")
    y = E.main(["--shape", "tiny", "--heads", "4", "2", "64", "--requests", "5", "--prefix", "32", "--own", "9", "--budget", "64",
                "--steps", "3"])
    assert y.shape == (5, synth.SHAPES["tiny"].H) and bool(torch.isfinite(y).all())
