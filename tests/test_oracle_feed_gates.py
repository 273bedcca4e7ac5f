"""The oracle's account of the activations' 32-bit steps: its values are the activations, its bounds hold for the same steps in numpy's fp32 and are small
beside small values too."""
import math

import numpy as np
import pytest

from oracle import feed

f = np.float32


def steps(name, g):
    """act and act' in fp32, step by step."""
    if name == "gelu":
        share = f(0.5) * np.array([math.erfc(z) for z in g * f(-0.70710678118655)], f)
        return g * share, share + g * (f(0.398942280401433) * np.exp2(g * g * f(-0.72134752044448)))
    y, bend = (g, f(1)) if name == "silu" else (f(1.59576912160573) * g * (f(1) + f(0.044715) * g * g), f(1.59576912160573) * (f(1) + f(0.134145) * g * g))
    share = f(1) / (f(1) + np.exp2(y * f(-1.44269504088896)))
    return g * share, share + g * (share * (f(1) - share)) * bend


@pytest.mark.parametrize("name,least", [("silu", -70), ("gelu", -11), ("gelu_tanh", -8)])
def test_steps_in_fp32_are_within_the_bounds(name, least):
    g = np.linspace(least, 12, 20001).astype(f)
    act, act_off, slope, slope_off = feed.activation_steps(name, g.astype(np.float64))
    got = steps(name, g)
    assert (np.abs(got[0] - act) <= act_off).all() and (np.abs(got[1] - slope) <= slope_off).all()
    assert (act_off <= 2.0 ** -13 * np.abs(act) + 2.0 ** -119).all()


@pytest.mark.parametrize("name", ["silu", "gelu", "gelu_tanh"])
def test_values_are_the_activations(name):
    g = np.linspace(-4, 12, 1001)
    act, _, slope, _ = feed.activation_steps(name, g)
    expect = feed.activation(name, g)
    assert np.allclose(act, expect[0], rtol=1e-11, atol=0) and np.allclose(slope, expect[1], rtol=1e-9, atol=1e-12)


def test_the_normal_distributions_tail():
    # Phi(-5) = 2.866515718791939e-7, Phi(-8) = 6.220960574271785e-16
    act = feed.activation_steps("gelu", np.array([-5.0, -8.0]))[0]
    assert np.allclose(act, [-5 * 2.866515718791939e-7, -8 * 6.220960574271785e-16], rtol=1e-12, atol=0)
