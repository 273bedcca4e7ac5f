"""The feed-forward oracle against torch's own 8-bit floats, against differences, and against the definition written out."""
import numpy as np
import pytest
import torch

from oracle import feed


def test_8_bit_floats_are_torchs():
    values = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(feed.e4m3_values(), values, equal_nan=True)


def test_rounding_to_8_bits_is_torchs():
    v = feed.e4m3_values()[:127]
    middle = (v[1:] + v[:-1]) / 2
    x = np.concatenate((v, middle, np.nextafter(middle.astype(np.float32), np.float32(0)), np.nextafter(middle.astype(np.float32), np.float32(1e9)))).astype(np.float32)
    x = np.concatenate((x, -x))
    assert np.array_equal(feed.e4m3_bits(x), torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy())


def test_scales_are_the_smallest_power_that_fits():
    x = np.zeros((3, 130), np.float32)
    x[0, 0], x[1, 5], x[1, 129], x[2, 3] = 448.0, np.nextafter(np.float32(448), np.float32(1e9)), 1e-45, -3.0e38
    bits, scale = feed.quantize(x, 1)
    assert scale[0, 0] == 1 and scale[0, 1] == 1 and scale[1, 0] == 2 and scale[1, 1] == 2.0 ** -126
    assert scale[2, 0] / 2 * 448 < 3.0e38 <= scale[2, 0] * 448
    assert bits[0, 0] == 0x7e and bits[1, 0] == 0
    both, one = feed.quantize(x, 128)
    assert one.shape == (1, 2) and one[0, 0] == scale[:, 0].max()


@pytest.mark.parametrize("name", ["silu", "gelu", "gelu_tanh"])
def test_gradients_are_differences(name):
    rng = np.random.default_rng(3)
    x, wg, wu, dy = rng.normal(size=(3, 5)), rng.normal(size=(4, 5)), rng.normal(size=(4, 5)), rng.normal(size=(3, 4))

    def loss(x, wg, wu):
        return (feed.gated(x, wg, wu, name, 0.0)["out"][0] * dy).sum()

    got = feed.gated_backward(x, wg, wu, dy, name, 0.0)
    for i, key in enumerate(("grad_x", "grad_w_gate", "grad_w_up")):
        arrays = [x, wg, wu]
        for at in np.ndindex(arrays[i].shape):
            moved = [[a.copy() for a in arrays] for _ in range(2)]
            moved[0][i][at] += 1e-5
            moved[1][i][at] -= 1e-5
            assert abs((loss(*moved[0]) - loss(*moved[1])) / 2e-5 - got[key][0][at]) < 1e-7


@pytest.mark.parametrize("name", ["silu", "gelu", "gelu_tanh"])
def test_the_bounds_on_second_derivatives_hold(name):
    g = np.linspace(-12, 12, 200001)
    slope, bend = feed.activation(name, g)[1:]
    assert np.abs(np.diff(slope) / np.diff(g)).max() < bend
