"""Tables of Rotary.make that tests/test_oracle_kv8.py does not pin (no GPU): the ramp of
yarn between the pairs that stay and those that are divided, and what goes with
frequencies that are given."""
import math

import pytest

import paper_2606_00535_gb300 as dreams


def radians(r):
    """Frequencies that a table's phases stand for, up to whole turns."""
    return [2 * math.pi * u / 2.0 ** 64 for u in r.phase.tolist()]


@pytest.mark.parametrize("rot,base,factor,original,fast,slow", [(128, 10000.0, 8.0, 4096, 32.0, 1.0), (64, 500000.0, 40.0, 8192, 20.0, 2.0)])
def test_the_ramp_of_yarn_is_linear_in_turns(rot, base, factor, original, fast, slow):
    got = radians(dreams.Rotary.make(rot, base=base, scaling="yarn", factor=factor, original=original, fast=fast, slow=slow, device="cpu"))
    between = 0
    for i, x in enumerate(got):
        f = base ** (-2.0 * i / rot)
        turns = original * f / (2 * math.pi)  # of this pair over the original context
        if turns >= fast:
            want = f
        elif turns <= slow:
            want = f / factor
        else:
            between += 1
            keep = (turns - slow) / (fast - slow)
            want = keep * f + (1 - keep) * f / factor
        assert abs(x - want) <= 1e-12 * want + 1e-17, i  # (doubles: some 2^-50 of f; phases: 2^-64 of a turn)
    assert between >= 5


def test_given_frequencies_are_scaled_or_refused():
    f = [1.0, 0.25, 0.01, 0.002]
    assert radians(dreams.Rotary.make(8, frequencies=f, scaling="linear", factor=4.0, device="cpu")) == pytest.approx([x / 4 for x in f], rel=1e-12)
    a, b = (dreams.Rotary.make(8, scaling="yarn", factor=4.0, device="cpu", frequencies=g) for g in (None, [10000.0 ** (-i / 4) for i in range(4)]))
    assert a.phase.tolist() == b.phase.tolist() and a.factor == b.factor
    with pytest.raises(ValueError):  # ntk scales the base, which given frequencies do not have
        dreams.Rotary.make(8, frequencies=f, scaling="ntk", factor=4.0, device="cpu")
