"""The decode-step example refuses what its cache and its tables have no room for, before
anything reaches the device (no GPU needed)."""
import os

import pytest

from examples import decode_step as E
from paper_2607_00466_amd import synth

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


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


def documented():
    """The example's commands in the README and in its own help."""
    text = open(os.path.join(ROOT, "README.md")).read()
    lines = [l.split("#")[0].split()[2:] for l in text.splitlines() if l.strip().startswith("python examples/decode_step.py")]
    assert len(lines) >= 2
    return lines + [[], ["--int8"], ["--fp8"], ["--norm"], ["--int8", "--own", "0", "--steps", "1"], ["--int8", "--prefix", "4096"]]


@pytest.mark.parametrize("argv", documented(), ids=" ".join)
def test_documented_commands_have_room(argv):
    a = E.arguments(argv)
    E.check_sizes(a.groups, a.prefix, a.own, a.budget, a.steps, fp8=a.fp8, int8=a.int8)


def test_a_budget_that_is_given_is_kept():
    a = E.arguments(["--int8", "--budget", "2304"])
    assert a.budget == 2304
    with pytest.raises(ValueError, match="8-bit integers"):
        E.check_sizes(a.groups, a.prefix, a.own, a.budget, a.steps, fp8=a.fp8, int8=a.int8)
