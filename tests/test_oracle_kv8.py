"""Pins of the oracle of rotary positions and 8-bit pages, and of the tables that
Rotary.make works out (no GPU)."""
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

import paper_2606_00535_gb300 as dreams
from oracle import rotary_kv8 as R


def test_values_are_those_of_e4m3():
    codes = torch.arange(256, dtype=torch.uint8)
    want = codes.view(torch.float8_e4m3fn).double().numpy()
    got = R.decode(codes.numpy(), np.zeros(256))
    assert np.array_equal(got[~np.isnan(want)], want[~np.isnan(want)]) and np.array_equal(np.isnan(got), np.isnan(want))


def test_rounding_is_to_nearest_even():
    x = torch.cat([torch.randn(20000) * 10.0 ** torch.linspace(-4, 2.6, 20000), torch.tensor([0.0, -0.0, 448.0, 447.9])]).clamp(-448, 448)
    t = torch.tensor(R.values())
    x = torch.cat([x, ((t[1:] + t[:-1]) / 2).float()])  # the ties
    assert np.array_equal(R.encode(x.numpy(), 0), x.to(torch.float8_e4m3fn).view(torch.uint8).numpy())


@pytest.mark.parametrize("amax,e", [(448.0, 0), (448.0 * 1.01, 1), (1.75, -8), (1.76, -7), (0.0, R.EXP_MIN), (2.0 ** 127 * 1.99, 119), (math.inf, R.NOT_FINITE),
                                    (math.nan, R.NOT_FINITE), (2.0 ** -140, R.EXP_MIN)])
def test_power(amax, e):
    assert R.power(amax) == e


def test_stored_values_are_exact_in_bf16():
    for e in (R.EXP_MIN, -1, 0, 7, 8, R.EXP_MAX):
        v = torch.tensor(R.decode(np.arange(127, dtype=np.uint8), np.full(127, e)))
        assert torch.equal(v.to(torch.bfloat16).double(), v)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rotation_keeps_lengths_and_relative_angles(layout):
    rng = np.random.default_rng(1)
    ph = [R.phase_of(10000.0 ** (-i / 4)) for i in range(4)]
    q, k = rng.standard_normal((2, 12))
    for p in (0, 1, 77, 10 ** 6):
        a, b = R.rotate(q, ph, p + 13, layout), R.rotate(k, ph, p, layout)
        assert np.isclose(a @ b, R.rotate(q, ph, 13, layout) @ k, atol=1e-9)
        assert np.isclose(a @ a, q @ q) and np.array_equal(a[8:], q[8:])
        assert np.allclose(R.rotate(a, ph, p + 13, layout, transpose=True), q)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_transposed_map_is_the_gradient(layout):
    """Against differences: the map is linear, so any step gives its derivative."""
    rng = np.random.default_rng(2)
    ph, x, g = [R.phase_of(0.3), R.phase_of(0.007)], rng.standard_normal(6), rng.standard_normal(6)
    f = lambda y: g @ R.rotate(y, ph, 41, layout, 1.3)  # noqa: E731
    num = [(f(x + 0.5 * d) - f(x - 0.5 * d)) for d in np.eye(6)]
    want = R.rotate(g, ph, 41, layout, 1.3, transpose=True)
    assert np.allclose(num, want)  # (dimensions behind the pairs: as they are, factor or not)


def test_tables():
    for kw, f in ((dict(rot_dim=8, base=100.0), [100.0 ** (-i / 4) for i in range(4)]),
                  (dict(rot_dim=8, base=100.0, scaling="linear", factor=4.0), [100.0 ** (-i / 4) / 4 for i in range(4)]),
                  (dict(rot_dim=8, base=100.0, scaling="ntk", factor=4.0), [(100.0 * 4 ** (8 / 6)) ** (-i / 4) for i in range(4)]),
                  (dict(rot_dim=4, frequencies=[7.5, -0.25]), [7.5, -0.25])):
        r = dreams.Rotary.make(device="cpu", **kw)
        assert r.factor == 1.0 and r.n_pairs == len(f)
        for u, x in zip(r.phase.tolist(), f):
            exact = Fraction(x) / Fraction(2 * math.pi)
            assert abs(Fraction(u % 2 ** 64, 2 ** 64) - exact % 1) <= Fraction(1, 2 ** 51)  # (x / 2 pi in doubles)
    # ntk leaves the fastest pair and slows the slowest by the factor
    a, b = (dreams.Rotary.make(64, scaling=s, factor=8.0, device="cpu") for s in ("none", "ntk"))
    assert a.phase[0] == b.phase[0] and abs(int(a.phase[-1]) / int(b.phase[-1]) - 8.0) < 1e-9
    # yarn: fast pairs as they were, slow ones divided, and a gain
    y = dreams.Rotary.make(128, scaling="yarn", factor=8.0, original=4096, device="cpu")
    n = dreams.Rotary.make(128, device="cpu")
    assert abs(y.factor - (0.1 * math.log(8.0) + 1)) < 1e-12 and y.phase[0] == n.phase[0]
    assert abs(int(n.phase[-1]) / int(y.phase[-1]) - 8.0) < 1e-9
    assert dreams.Rotary.make(128, scaling="yarn", factor=8.0, gain=1.0, device="cpu").factor == 1.0


@pytest.mark.parametrize("kw", [dict(rot_dim=0), dict(rot_dim=7), dict(rot_dim=8, layout="other"), dict(rot_dim=8, scaling="other"), dict(rot_dim=8, factor=0.0),
                                dict(rot_dim=8, base=-1.0), dict(rot_dim=2, scaling="ntk", factor=2.0), dict(rot_dim=8, frequencies=[1.0]),
                                dict(rot_dim=4, frequencies=[1.0, math.nan]), dict(rot_dim=4, axis=[0]), dict(rot_dim=4, axis=[0, 4]),
                                dict(rot_dim=4, gain=math.inf), dict(rot_dim=8, scaling="yarn", original=0)])
def test_tables_refused(kw):
    with pytest.raises(ValueError):
        dreams.Rotary.make(device="cpu", **kw)
