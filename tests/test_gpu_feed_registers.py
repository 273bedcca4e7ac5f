"""GPU parity of every kernel of the feed-forward products that brings operands to LDS through registers, against the 64-bit oracle (that each call launches the
kernel it is listed for is a test without a GPU)."""
import numpy as np
import pytest

from oracle import feed
from tests.feed_shapes import THROUGH_REGISTERS
from tests.feed_util import Result, put, rounded, within
from tests.test_gpu_feed_kernels import cut_off, normal, say, scaled

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    import paper_1802_06905_amd as cc
    assert torch.cuda.is_available(), "these tests need the GPU"
    return cc, torch


def listed(*calls):
    return [row for row in THROUGH_REGISTERS if row[1] in calls]


@pytest.mark.parametrize("kernel,call,out,T,C,K,pad,shift", listed("matmul", "scaled"))
def test_operands_in_8_bits(env, kernel, call, out, T, C, K, pad, shift):
    cc, torch = env
    say("[feed] through registers", kernel, call, out, T, C, K, pad, shift)
    rng = np.random.default_rng(T + C + K)
    x, xq, xs = scaled(torch, rng, T, C, 1)
    (w, wq, ws), (v, vq, vs) = (scaled(torch, rng, K, C, 128) for _ in range(2))
    # (so that gates are about 1)
    xs, x = xs / 4, x / 4
    y = Result(torch, T, K, getattr(torch, {"f32": "float32", "bf16": "bfloat16"}[out]), pad, shift)
    code = int(out == "bf16")
    cut = [cut_off(torch, x, a) if code else 0.0 for a in (w, v)]
    operands = [put(torch, xq, pad, shift), xs.cuda(), wq.cuda(), ws.cuda()]
    if call == "matmul":
        cc.cacnn_matmul_scaled((T, C, K), *operands, code, y.view)
        expect = feed.matmul_scaled(x, w, feed.HALF_STEP[out], cut[0])
    else:
        cc.cacnn_gated_forward_scaled((T, C, K, cc.CACNN_GATE_SILU), *operands, vq.cuda(), vs.cuda(), code, y.view)
        expect = feed.gated(x, w, v, "silu", feed.HALF_STEP[out], sums=128 + -(-C // 128) + 2, cut=cut)["out"]
    within("out", y.numpy(), *expect)
    y.check()


@pytest.mark.parametrize("kernel,call,dtype,T,C,F,pad,shift", listed("forward"))
def test_gated_projections(env, kernel, call, dtype, T, C, F, pad, shift):
    cc, torch = env
    say("[feed] through registers", kernel, call, dtype, T, C, F, pad, shift)
    rng = np.random.default_rng(T + C + F)
    (x, tx), (wg, tg), (wu, tu) = normal(torch, rng, dtype, T, C), normal(torch, rng, dtype, F, C, C ** -0.5), normal(torch, rng, dtype, F, C, C ** -0.5)
    y, g, u = (Result(torch, T, F, tx.dtype, pad, shift) for _ in range(3))
    cc.cacnn_gated_forward((T, C, F, cc.CACNN_GATE_GELU_TANH), int(dtype == "bf16"), put(torch, tx, pad, shift), tg.cuda(), tu.cuda(), y.view, gate=g.view, up=u.view)
    expect = feed.gated(x, wg, wu, "gelu_tanh", feed.HALF_STEP[dtype])
    for name, r in (("out", y), ("gate", g), ("up", u)):
        within(name, r.numpy(), *expect[name])
        r.check()


@pytest.mark.parametrize("kernel,call,dtype,T,C,F,pad,shift", listed("backward"))
def test_gradients(env, kernel, call, dtype, T, C, F, pad, shift):
    cc, torch = env
    say("[feed] through registers", kernel, call, dtype, T, C, F, pad, shift)
    rng = np.random.default_rng(T + C + F)
    (x, tx), (wg, tg), (wu, tu) = normal(torch, rng, dtype, T, C), normal(torch, rng, dtype, F, C, C ** -0.5), normal(torch, rng, dtype, F, C, C ** -0.5)
    (dy, td), (g, kept_g), (u, kept_u) = normal(torch, rng, dtype, T, F, 1e-2), normal(torch, rng, dtype, T, F), normal(torch, rng, dtype, T, F)
    gx, gg, gu = (Result(torch, *a.shape, tx.dtype, pad, shift) for a in (tx, tg, tu))
    where = (T, C, F, cc.CACNN_GATE_SILU)
    workspace = torch.empty(cc.cacnn_gated_workspace(where, int(dtype == "bf16")), dtype=torch.uint8, device="cuda")
    cc.cacnn_gated_backward(where, int(dtype == "bf16"), *(put(torch, a, pad, shift) for a in (tx, tg, tu)), td.cuda(), gx.view, gg.view, gu.view, workspace,
                            gate=kept_g.cuda(), up=kept_u.cuda())
    expect = feed.gated_backward(x, wg, wu, dy, "silu", feed.HALF_STEP[dtype], g, u)
    for name, r in (("grad_x", gx), ("grad_w_gate", gg), ("grad_w_up", gu)):
        within(name, r.numpy(), *expect[name])
        r.check()
