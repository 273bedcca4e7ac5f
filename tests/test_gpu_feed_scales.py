"""Scales at either end of fp32 in the 8-bit products: each block's sum, exact here, times fp32's product of its two scales, which may be subnormal, zero, infinite or
NaN."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

X_SCALES = [1e-40, 2.0 ** -126, 3e-30, 1 / 60, 1.0, 5e10, 2e30, np.inf, np.nan, 0.0, -1.5]
W_SCALES = [1e-40, 2.0 ** -126, 1e-25, 1.0, 3e20, 2.0 ** 110]


@pytest.fixture(scope="module")
def env():
    import torch
    import paper_1802_06905_amd as cc
    assert torch.cuda.is_available(), "these tests need the GPU"
    return cc, torch


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("T,C,K", [(44, 15, 640), (44, 300, 640), (44, 304, 640), (1100, 640, 700), (2210, 640, 3400)])
def test_any_scale(env, T, C, K, out):
    """Finite products of scales are at most 2e33, far from the largest number also times sums of 2^12, so that what is infinite is a product of scales."""
    cc, torch = env
    rng = np.random.default_rng(C)
    x, w = (rng.integers(-2, 3, size=s).astype(np.float32) for s in ((T, C), (K, C)))
    x[5] = 0
    blocks = -(-C // 128)
    xs = np.array(X_SCALES, np.float32)[np.arange(T) % len(X_SCALES)][:, None].repeat(blocks, 1)
    ws = rng.choice(np.array(W_SCALES, np.float32), size=(-(-K // 128), blocks))
    half_step = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}[out]
    value, size = np.zeros((T, K)), np.zeros((T, K))
    with np.errstate(all="ignore"):
        for b in range(blocks):
            part = np.s_[:, b * 128:(b + 1) * 128]
            block = x[part].astype(np.float64) @ w[part].astype(np.float64).T
            f = (xs[:, b][:, None] * ws[:, b].repeat(128)[:K][None]).astype(np.float32).astype(np.float64)
            value += f * block
            size += np.abs(f * block)
        # a rounding for each block, and one where waves' sums are added; half of the least subnormal number where they are as small as that
        bound = (blocks + 4) * (size * 2.0 ** -24 + 2.0 ** -150)
        bound += half_step * (np.abs(value) + bound) + (2.0 ** -150 if out == "f32" else 2.0 ** -134)
    t, code = {"f32": (torch.float32, 0), "bf16": (torch.bfloat16, 1)}[out]
    xq, wq = (torch.from_numpy(a).to(torch.float8_e4m3fn).cuda() for a in (x, w))
    y = torch.full((T, K), 5.0, dtype=t, device="cuda")
    cc.cacnn_matmul_scaled((T, C, K), xq, torch.from_numpy(xs).cuda(), wq, torch.from_numpy(ws).cuda(), code, y)
    got = y.cpu().double().numpy()
    finite = np.isfinite(value)
    assert np.array_equal(np.isnan(got), np.isnan(value)) and np.array_equal(got[np.isinf(value)], value[np.isinf(value)])
    off = np.abs(got[finite] - value[finite]) - bound[finite]
    assert off.max() <= 0, (off.max(), got[finite][off.argmax()], value[finite][off.argmax()], bound[finite][off.argmax()])
