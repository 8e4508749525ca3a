"""The decode-step example refuses what its cache and its tables have no room for, before
anything reaches the device (no GPU needed)."""
import pytest

from examples import decode_step as E
from paper_2607_00466_amd import synth


@pytest.mark.parametrize("bad", [dict(steps=0), dict(steps=-1), dict(own=-1), dict(groups=0), dict(prefix=40), dict(budget=60)])
def test_sizes_refused(bad):
    sizes = dict(R=4, groups=2, prefix=32, own=16, budget=64, steps=3) | bad
    with pytest.raises(ValueError):
        E.Worker(synth.SHAPES["tiny"], E.Heads(4, 2, 64), **sizes)


def test_no_step_past_the_last_one():
    # with 32 + 16 tokens in whole pages a step more would have no page: its slot lies past the block table
    w = object.__new__(E.Worker)
    w.left = 0
    with pytest.raises(RuntimeError, match="step"):
        w.attend(None)
