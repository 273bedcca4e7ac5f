"""GPU parity of the feed-forward operators where every array has rows of another distance: each is read and written by its own."""
import numpy as np
import pytest

from oracle import feed
from tests.feed_util import Result, put, rounded, within
from tests.test_gpu_feed_kernels import normal

pytestmark = pytest.mark.gpu

# of X, the weights, Out (and its gradient), gate and up, X's gradient, the weights' gradients: whole 16 bytes, and not
PADS = [(16, 48, 32, 80, 64, 112), (1, 5, 2, 7, 3, 9), (16, 0, 1, 0, 8, 3)]


@pytest.fixture(scope="module")
def env():
    import torch
    import paper_1802_06905_amd as cc
    assert torch.cuda.is_available(), "these tests need the GPU"
    return cc, torch


@pytest.mark.parametrize("usual", [True, False])
@pytest.mark.parametrize("keep", [True, False])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pads", PADS)
@pytest.mark.parametrize("T,C,F", [(5, 64, 48), (140, 72, 200), (150, 77, 90), (60, 3, 33), (700, 320, 400)])
def test_a_distance_for_each_array(env, monkeypatch, T, C, F, pads, dtype, keep, usual):
    cc, torch = env
    if not usual:
        monkeypatch.setattr(cc.binding, "_native", None)
    rng = np.random.default_rng(T + C + F)
    (x, tx), (wg, tg), (wu, tu) = normal(torch, rng, dtype, T, C), normal(torch, rng, dtype, F, C, C ** -0.5), normal(torch, rng, dtype, F, C, C ** -0.5)
    dy, td = normal(torch, rng, dtype, T, F, 1e-2)
    code, half = int(dtype == "bf16"), feed.HALF_STEP[dtype]
    where = (T, C, F, cc.CACNN_GATE_SILU)
    x_, g_, u_ = put(torch, tx, pads[0]), put(torch, tg, pads[1]), put(torch, tu, pads[1])
    y, gate, up = Result(torch, T, F, tx.dtype, pads[2]), Result(torch, T, F, tx.dtype, pads[3]), Result(torch, T, F, tx.dtype, pads[3])
    cc.cacnn_gated_forward(where, code, x_, g_, u_, y.view, gate=gate.view, up=up.view)
    for (name, expect), r in zip(feed.gated(x, wg, wu, "silu", half).items(), (gate, up, y)):
        within(name, r.numpy(), *expect)
        r.check()
    grads = [Result(torch, rows, C, tx.dtype, pad) for rows, pad in ((T, pads[4]), (F, pads[5]), (F, pads[5]))]
    work = torch.empty(cc.cacnn_gated_workspace(where, code), dtype=torch.uint8, device="cuda")
    kept = {"gate": gate.view, "up": up.view} if keep else {}
    cc.cacnn_gated_backward(where, code, x_, g_, u_, put(torch, td, pads[2]), *(r.view for r in grads), work, **kept)
    expect = feed.gated_backward(x, wg, wu, dy, "silu", half, *((gate.numpy(), up.numpy()) if keep else ()))
    for (name, value), r in zip(expect.items(), grads):
        within(name, r.numpy(), *value)
        r.check()


@pytest.mark.parametrize("usual", [True, False])
@pytest.mark.parametrize("pads", PADS)
@pytest.mark.parametrize("T,C,K", [(5, 64, 48), (140, 208, 300), (150, 77, 90), (60, 7, 33)])
def test_a_distance_for_each_array_in_8_bits(env, monkeypatch, T, C, K, pads, usual):
    """Quantisation, product and gated projection."""
    cc, torch = env
    if not usual:
        monkeypatch.setattr(cc.binding, "_native", None)
    rng = np.random.default_rng(T + C + K)
    arrays = []
    for rows, block, pad_in, pad_out in ((T, 1, pads[2], pads[0]), (K, 128, pads[3], pads[1]), (K, 128, pads[3], pads[1])):
        _, t = rounded(torch, rng.normal(size=(rows, C)), "f32")
        q = Result(torch, rows, C, torch.uint8, pad_out)
        s = torch.zeros((-(-rows // block), -(-C // 128)), device="cuda")
        cc.cacnn_quantize((rows, C, block), 0, put(torch, t, pad_in), q.view, s)
        bits, scale = feed.quantize(t.numpy(), block)
        assert np.array_equal(q.view.cpu().numpy(), bits) and np.array_equal(s.cpu().double().numpy(), scale)
        q.check()
        arrays.append((q.view, s, feed.stands_for(bits, scale, block)))
    (xq, xs, x), (wq, ws, w), (vq, vs, v) = arrays
    y, h = Result(torch, T, K, torch.float32, pads[4]), Result(torch, T, K, torch.float32, pads[5])
    cc.cacnn_matmul_scaled((T, C, K), xq, xs, wq, ws, 0, y.view)
    cc.cacnn_gated_forward_scaled((T, C, K, cc.CACNN_GATE_GELU_TANH), xq, xs, wq, ws, vq, vs, 0, h.view)
    within("product", y.numpy(), *feed.matmul_scaled(x, w, 2.0 ** -24))
    within("gated", h.numpy(), *feed.gated(x, w, v, "gelu_tanh", 2.0 ** -24, sums=128 + -(-C // 128) + 2)["out"])
    y.check(), h.check()
