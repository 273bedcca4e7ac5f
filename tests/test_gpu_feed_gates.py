"""GPU parity of the feed-forward operators' activations to the leading digits of each value, small ones among them: gates far below zero, where the
activation is a small part of its gate."""
import numpy as np
import pytest

from oracle import feed
from tests.feed_util import GATES, rounded, within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    import paper_1802_06905_amd as cc
    assert torch.cuda.is_available(), "these tests need the GPU"
    return cc, torch


def gates(torch, name, dtype):
    """From where the value is about 1e-30 up to 12."""
    least = {"silu": -70.0, "gelu": -11.0, "gelu_tanh": -8.0}[name]
    g = np.concatenate((np.linspace(least, 12, 700), np.linspace(-8, -3, 101), [-5.0, -5.5, -1e-3, 1e-3, 0.0]))
    return rounded(torch, g[:, None], dtype)


@pytest.mark.parametrize("C", [1, 63, 64])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("name", GATES)
def test_small_values_of_the_activation(env, name, dtype, C):
    """gate = X W_gate' is the first channel as it is and up is 1 (the second channel): Out is the activation."""
    cc, torch = env
    g, t = gates(torch, name, dtype)
    T = len(g)
    x = torch.zeros((T, C + 1), dtype=t.dtype)
    x[:, :1], x[:, 1:2] = t, 1
    w = torch.zeros((2, C + 1), dtype=t.dtype)
    w[0, 0], w[1, 1] = 1, 1
    y = torch.full((T, 1), float("nan"), dtype=t.dtype, device="cuda")
    cc.cacnn_gated_forward((T, C + 1, 1, GATES.index(name)), int(dtype == "bf16"), x.cuda(), w[:1].cuda(), w[1:].cuda(), y)
    value, off, _, _ = feed.activation_steps(name, g)
    within(name, y.cpu().double().numpy(), value, off + feed.HALF_STEP[dtype] * (np.abs(value) + off))


@pytest.mark.parametrize("keep", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("name", GATES)
def test_small_slopes(env, name, dtype, keep):
    """With up and Out's gradient 1, X's gradient is act'(gate) in its first channel, which is gate's, and act(gate) in its second, which is up's."""
    cc, torch = env
    g, t = gates(torch, name, dtype)
    T = len(g)
    x = torch.cat((t, torch.ones_like(t)), 1).cuda()
    w = torch.eye(2, dtype=t.dtype, device="cuda")
    grad_x = torch.full((T, 2), float("nan"), dtype=t.dtype, device="cuda")
    where = (T, 2, 1, GATES.index(name))
    workspace = torch.empty(cc.cacnn_gated_workspace(where, int(dtype == "bf16")), dtype=torch.uint8, device="cuda")
    kept = {"gate": t.cuda(), "up": torch.ones_like(t).cuda()} if keep else {}
    cc.cacnn_gated_backward(where, int(dtype == "bf16"), x, w[:1].contiguous(), w[1:].contiguous(), torch.ones_like(t).cuda(), grad_x, None, None, workspace, **kept)
    act, act_off, slope, slope_off = feed.activation_steps(name, g)
    # (rounded to the arrays' type once: the sums that follow have one term)
    value, off = np.concatenate((slope, act), 1), np.concatenate((slope_off, act_off), 1)
    within(name, grad_x.cpu().double().numpy(), value, off + feed.HALF_STEP[dtype] * (np.abs(value) + off))
