"""GPU parity of each kernel of the feed-forward products on a shape that chooses it, results and gradients against the 64-bit oracle; addresses beyond
32 bits; the binding's two ways; calls at the same time."""
import ctypes

import numpy as np
import pytest

from oracle import feed
from tests.feed_util import Result, put, rounded, within

pytestmark = pytest.mark.gpu

GATED, PLAIN, RIGHT, BOTH = 0, 1, 2, 3                    # forms, and kernels, as the library numbers them
W32, W64_32, W64, DEEP, MIDDLE, LARGE, SMALL = range(7)
TYPES = {"f32": 0, "bf16": 1, "e4m3": 2, "e4m3 exact": 3}


@pytest.fixture(scope="module")
def env():
    import torch
    import paper_1802_06905_amd as cc
    assert torch.cuda.is_available(), "these tests need the GPU"
    return cc, torch


def kernel_of(cc, form, dtype, M, N, k, direct=True):
    call = cc.binding._lib.cacnn_internal_matmul_kernel
    call.argtypes = [ctypes.c_int] * 3 + [ctypes.c_int64] * 3
    return call(form, TYPES[dtype], int(direct), M, N, k)


def say(*what):
    print(*what, flush=True)


def cut_off(torch, x, w):
    """oracle's cut_off, on the device"""
    x, w = (torch.from_numpy(np.abs(np.pad(a, ((0, 0), (0, -a.shape[1] % 8))))).cuda() for a in (x, w))
    total = torch.zeros((x.shape[0], w.shape[0]), dtype=torch.float64, device="cuda")
    for k in range(0, x.shape[1], 8):
        largest = torch.zeros_like(total)
        for i in range(k, k + 8):
            torch.maximum(largest, torch.outer(x[:, i], w[:, i]), out=largest)
        total += largest
    return (total * 7 * 2.0 ** -13).cpu().numpy()


def scaled(torch, rng, rows, cols, block_rows):
    bits = feed.e4m3_bits(np.clip(rng.normal(size=(rows, cols)) * 60, -448, 448))
    scale = np.exp(rng.normal(size=(-(-rows // block_rows), -(-cols // 128)))).astype(np.float32) / 60
    return feed.stands_for(bits, scale, block_rows), torch.from_numpy(bits).view(torch.float8_e4m3fn), torch.from_numpy(scale)


# (kernel, T, C, K or F) for each form and type: shapes, sought at random, that choose the kernel and have five slabs of the contraction at least
SHAPES = {
    (PLAIN, "e4m3"): [(W32, 26, 672, 126), (W64_32, 465, 688, 547), (W64, 522, 656, 908), (DEEP, 1369, 672, 717), (MIDDLE, 2185, 656, 1796), (LARGE, 2325, 640, 3374)],
    (PLAIN, "e4m3 exact"): [(W32, 120, 656, 61), (W64_32, 633, 656, 392), (W64, 653, 640, 746), (DEEP, 1223, 640, 810), (MIDDLE, 1576, 640, 2496)],
    (GATED, "bf16"): [(W32, 75, 360, 84), (W64_32, 556, 360, 462), (DEEP, 732, 320, 700), (MIDDLE, 1154, 320, 1641), (LARGE, 2325, 320, 1675)],
    (GATED, "f32"): [(W32, 40, 184, 83), (W64_32, 420, 184, 617), (SMALL, 537, 160, 1055), (DEEP, 918, 176, 1135), (MIDDLE, 1685, 160, 1831)],
    (GATED, "e4m3"): [(W32, 28, 720, 99), (W64_32, 590, 640, 423), (DEEP, 710, 640, 705), (MIDDLE, 1548, 640, 1230), (LARGE, 1288, 656, 2973)],
    (GATED, "e4m3 exact"): [(W32, 24, 688, 66), (W64_32, 388, 640, 703), (DEEP, 800, 640, 609), (MIDDLE, 1424, 656, 1365)],
    (RIGHT, "bf16"): [(W32, 30, 192, 325), (W64_32, 408, 616, 324), (W64, 771, 616, 352), (DEEP, 1221, 856, 330), (MIDDLE, 2492, 1600, 327), (LARGE, 4176, 1968, 329)],
    (RIGHT, "f32"): [(W32, 42, 120, 214), (W64_32, 466, 624, 162), (W64, 589, 832, 168), (SMALL, 1216, 856, 162), (DEEP, 1250, 1632, 167), (MIDDLE, 3295, 1840, 166)],
    (BOTH, "bf16"): [(W32, 331, 64, 44), (W64_32, 355, 360, 363), (W64, 328, 528, 542), (DEEP, 326, 560, 911), (MIDDLE, 320, 1184, 1596), (LARGE, 320, 1720, 2309)],
    (BOTH, "f32"): [(W32, 202, 64, 65), (W64_32, 213, 376, 401), (W64, 186, 408, 577), (SMALL, 161, 664, 716), (DEEP, 168, 688, 1354), (MIDDLE, 176, 1416, 2062)],
}


def shapes(*forms):
    return [(form, dtype, *shape) for (form, dtype), all_ in SHAPES.items() if form in forms for shape in all_]


def normal(torch, rng, dtype, rows, cols, size=1.0):
    return rounded(torch, rng.normal(size=(rows, cols)) * size, dtype)


@pytest.mark.parametrize("form,dtype,kernel,T,C,K", shapes(PLAIN) + [s for s in shapes(GATED) if s[1].startswith("e4m3")])
def test_operands_in_8_bits(env, form, dtype, kernel, T, C, K):
    cc, torch = env
    assert kernel_of(cc, form, dtype, T, K, C) == kernel
    say("[feed] 8 bits", form, dtype, kernel, T, C, K)
    rng = np.random.default_rng(kernel)
    x, xq, xs = scaled(torch, rng, T, C, 1)
    (w, wq, ws), (v, vq, vs) = (scaled(torch, rng, K, C, 128) for _ in range(2))
    out = "bf16" if dtype == "e4m3" else "f32"
    y = Result(torch, T, K, torch.float32 if out == "f32" else torch.bfloat16)
    cut = [cut_off(torch, x, a) if out == "bf16" else 0.0 for a in (w, v)]
    if form == PLAIN:
        cc.cacnn_matmul_scaled((T, C, K), xq.cuda(), xs.cuda(), wq.cuda(), ws.cuda(), 0 if out == "f32" else 1, y.view)
        expect = feed.matmul_scaled(x, w, feed.HALF_STEP[out], cut[0])
    else:
        cc.cacnn_gated_forward_scaled((T, C, K, cc.CACNN_GATE_GELU_TANH), xq.cuda(), xs.cuda(), wq.cuda(), ws.cuda(), vq.cuda(), vs.cuda(), 0 if out == "f32" else 1, y.view)
        expect = feed.gated(x, w, v, "gelu_tanh", feed.HALF_STEP[out], sums=128 + -(-C // 128) + 2, cut=cut)["out"]
    within("out", y.numpy(), *expect)
    y.check()


@pytest.mark.parametrize("form,dtype,kernel,T,C,F", [s for s in shapes(GATED) if not s[1].startswith("e4m3")])
def test_gated_projections(env, form, dtype, kernel, T, C, F):
    cc, torch = env
    assert kernel_of(cc, form, dtype, T, F, C) == kernel
    say("[feed] gated", dtype, kernel, T, C, F)
    rng = np.random.default_rng(kernel)
    (x, tx), (wg, tg), (wu, tu) = normal(torch, rng, dtype, T, C), normal(torch, rng, dtype, F, C, C ** -0.5), normal(torch, rng, dtype, F, C, C ** -0.5)
    y, g, u = (Result(torch, T, F, tx.dtype) for _ in range(3))
    cc.cacnn_gated_forward((T, C, F, cc.CACNN_GATE_SILU), TYPES[dtype], tx.cuda(), tg.cuda(), tu.cuda(), y.view, gate=g.view, up=u.view)
    expect = feed.gated(x, wg, wu, "silu", feed.HALF_STEP[dtype])
    for name, r in (("out", y), ("gate", g), ("up", u)):
        within(name, r.numpy(), *expect[name])
        r.check()


@pytest.mark.parametrize("form,dtype,kernel,T,C,F", shapes(RIGHT, BOTH))
def test_gradients(env, form, dtype, kernel, T, C, F):
    cc, torch = env
    assert (kernel_of(cc, form, dtype, T, C, F) if form == RIGHT else kernel_of(cc, form, dtype, F, C, T)) == kernel
    say("[feed] gradients", form, dtype, kernel, T, C, F)
    rng = np.random.default_rng(kernel)
    (x, tx), (wg, tg), (wu, tu) = normal(torch, rng, dtype, T, C), normal(torch, rng, dtype, F, C, C ** -0.5), normal(torch, rng, dtype, F, C, C ** -0.5)
    dy, td = normal(torch, rng, dtype, T, F, 1e-2)
    gx, gg, gu = Result(torch, T, C, tx.dtype), Result(torch, F, C, tx.dtype), Result(torch, F, C, tx.dtype)
    where = (T, C, F, cc.CACNN_GATE_SILU)
    workspace = torch.empty(cc.cacnn_gated_workspace(where, TYPES[dtype]), dtype=torch.uint8, device="cuda")
    cc.cacnn_gated_backward(where, TYPES[dtype], tx.cuda(), tg.cuda(), tu.cuda(), td.cuda(), gx.view, gg.view, gu.view, workspace)
    expect = feed.gated_backward(x, wg, wu, dy, "silu", feed.HALF_STEP[dtype])
    for name, r in (("grad_x", gx), ("grad_w_gate", gg), ("grad_w_up", gu)):
        within(name, r.numpy(), *expect[name])
        r.check()


def test_64_by_128_tiles_through_registers(env):
    """Odd sizes in fp32 that take these tiles in both directions, on operands whose rows allow no load to LDS."""
    cc, torch = env
    T, C, F = 1267, 803, 625
    assert [kernel_of(cc, form, "f32", *sizes, False) for form, sizes in ((GATED, (T, F, C)), (RIGHT, (T, C, F)), (BOTH, (F, C, T)))] == [SMALL] * 3
    say("[feed] 64 x 128 tiles through registers", T, C, F)
    rng = np.random.default_rng(64)
    (x, tx), (wg, tg), (wu, tu) = normal(torch, rng, "f32", T, C), normal(torch, rng, "f32", F, C, C ** -0.5), normal(torch, rng, "f32", F, C, C ** -0.5)
    dy, td = normal(torch, rng, "f32", T, F, 1e-2)
    y, gx, gg, gu = (Result(torch, rows, cols, torch.float32) for rows, cols in ((T, F), (T, C), (F, C), (F, C)))
    where = (T, C, F, cc.CACNN_GATE_SILU)
    tx, tg, tu, td = (a.cuda() for a in (tx, tg, tu, td))
    cc.cacnn_gated_forward(where, 0, tx, tg, tu, y.view)
    workspace = torch.empty(cc.cacnn_gated_workspace(where, 0), dtype=torch.uint8, device="cuda")
    cc.cacnn_gated_backward(where, 0, tx, tg, tu, td, gx.view, gg.view, gu.view, workspace)
    within("out", y.numpy(), *feed.gated(x, wg, wu, "silu", feed.HALF_STEP["f32"])["out"])
    expect = feed.gated_backward(x, wg, wu, dy, "silu", feed.HALF_STEP["f32"])
    for name, r in (("grad_x", gx), ("grad_w_gate", gg), ("grad_w_up", gu)):
        within(name, r.numpy(), *expect[name])
    for r in (y, gx, gg, gu):
        r.check()


# ---- addresses beyond 32 bits: the last rows of a large array are what the same rows give alone
def test_offsets_beyond_32_bits(env):
    cc, torch = env
    T, C, F = 1_100_003, 2048, 72                       # X is 4.5 GB
    say("[feed] X of 4.5 GB")
    x = torch.empty((T, C), dtype=torch.bfloat16, device="cuda")
    for part in x.split(100_000):
        part.normal_()
    wg, wu = (torch.randn((F, C), device="cuda").mul_(C ** -0.5).bfloat16() for _ in range(2))
    y, gate, up = (torch.zeros((T, F), dtype=torch.bfloat16, device="cuda") for _ in range(3))
    cc.cacnn_gated_forward((T, C, F, 0), 1, x, wg, wu, y, gate=gate, up=up)
    n = 300
    alone = [torch.zeros((n, F), dtype=torch.bfloat16, device="cuda") for _ in range(3)]
    tail = x[-n:].clone()
    cc.cacnn_gated_forward((n, C, F, 0), 1, tail, wg, wu, alone[0], gate=alone[1], up=alone[2])
    # (other kernels, other orders of summation: half a step of bf16 each and what fp32 sums of 2048 products differ by)
    for a, b in zip((y, gate, up), alone):
        assert torch.allclose(a[-n:].float(), b.float(), rtol=2.0 ** -7, atol=1e-4)
    say("[feed] quantise 4.5 GB")
    q, s = torch.zeros((T, C), dtype=torch.uint8, device="cuda"), torch.zeros((T, C // 128), device="cuda")
    q1, s1 = torch.zeros((n, C), dtype=torch.uint8, device="cuda"), torch.zeros((n, C // 128), device="cuda")
    cc.cacnn_quantize((T, C, 1), 1, x, q, s)
    cc.cacnn_quantize((n, C, 1), 1, tail, q1, s1)
    assert torch.equal(q[-n:], q1) and torch.equal(s[-n:], s1)
    say("[feed] gradients over 4.5 GB")
    grad_out = torch.zeros((T, F), dtype=torch.bfloat16, device="cuda")
    grad_out[-n:] = torch.randn((n, F), device="cuda").bfloat16()      # only the last rows count
    results = []
    for rows, args in ((T, (x, grad_out, gate, up)), (n, (tail, grad_out[-n:].clone(), gate[-n:].clone(), up[-n:].clone()))):
        grads = [torch.zeros(z, dtype=torch.bfloat16, device="cuda") for z in ((rows, C), (F, C), (F, C))]
        workspace = torch.empty(cc.cacnn_gated_workspace((rows, C, F, 0), 1), dtype=torch.uint8, device="cuda")
        cc.cacnn_gated_backward((rows, C, F, 0), 1, args[0], wg, wu, args[1], *grads, workspace, gate=args[2], up=args[3])
        results.append((grads[0][-n:].float(), grads[1].float(), grads[2].float()))
    for a, b in zip(*results):
        assert torch.allclose(a, b, rtol=2.0 ** -7, atol=1e-2 * float(b.abs().max()) * 2.0 ** -7)


def test_both_ways_of_the_binding_give_the_same(env, monkeypatch):
    cc, torch = env
    T, C, F = 33, 200, 136
    rng = np.random.default_rng(1)
    x, wg, wu, dy = (rounded(torch, a, "bf16")[1].cuda() for a in (rng.normal(size=(T, C)), rng.normal(size=(F, C)), rng.normal(size=(F, C)), rng.normal(size=(T, F))))
    wide = put(torch, x.cpu(), pad=5)
    assert cc.binding._native is not None

    def run():
        r = {n: torch.zeros(s, dtype=torch.bfloat16, device="cuda") for n, s in
             {"y": (T, F), "gate": (T, F), "up": (T, F), "gx": (T, C), "gg": (F, C), "gu": (F, C), "h": (T, F), "z": (T, F)}.items()}
        q, s = torch.zeros((T, C), dtype=torch.float8_e4m3fn, device="cuda"), torch.zeros((T, 2), device="cuda")
        wq, ws = torch.zeros((F, C), dtype=torch.uint8, device="cuda"), torch.zeros((2, 2), device="cuda")
        cc.cacnn_gated_forward((T, C, F, 1), 1, wide, wg, wu, r["y"], gate=r["gate"], up=r["up"])
        work = torch.zeros(cc.cacnn_gated_workspace((T, C, F, 1), 1), dtype=torch.uint8, device="cuda")
        cc.cacnn_gated_backward((T, C, F, 1), 1, wide, wg, wu, dy, r["gx"], r["gg"], r["gu"], work, gate=r["gate"], up=r["up"])
        cc.cacnn_quantize((T, C, 1), 1, wide, q, s)
        cc.cacnn_quantize((F, C, 128), 1, wg, wq, ws)
        cc.cacnn_matmul_scaled((T, C, F), q, s, wq, ws, 1, r["z"])
        cc.cacnn_gated_forward_scaled((T, C, F, 0), q, s, wq, ws, wq, ws, 1, r["h"])
        return {**r, "q": q.view(torch.uint8), "s": s, "wq": wq, "ws": ws}

    taken = []
    for name in ("quantize", "matmul_scaled", "gated_forward", "gated_forward_scaled", "gated_backward"):
        assert getattr(cc.binding._native, name)() == -1
    monkeypatch.setattr(cc.binding, "_lib", _Refusing(cc.binding._lib, taken))
    native = run()
    assert not taken, "the module left a usual call to the longer way"
    monkeypatch.undo()
    monkeypatch.setattr(cc.binding, "_native", None)
    longer = run()
    for k in native:
        assert torch.equal(native[k], longer[k]) and native[k].any(), k


class _Refusing:
    """The library but for the operators' calls, which are noted."""
    def __init__(self, lib, taken):
        self.lib, self.taken = lib, taken

    def __getattr__(self, name):
        if name in ("cacnn_quantize", "cacnn_matmul_scaled", "cacnn_gated_forward", "cacnn_gated_forward_scaled", "cacnn_gated_backward"):
            self.taken.append(name)
        return getattr(self.lib, name)


def test_calls_on_several_streams_at_once(env):
    """Different problems and operators, one right behind the other on four streams, give what each gives alone."""
    cc, torch = env
    jobs = []
    for i, (T, C, F) in enumerate([(3, 1024, 512), (40, 264, 1000), (300, 512, 512), (1000, 136, 700)]):
        rng = np.random.default_rng(i)
        args = [rounded(torch, a, "bf16")[1].cuda() for a in (rng.normal(size=(T, C)), rng.normal(size=(F, C)), rng.normal(size=(F, C)), rng.normal(size=(T, F)))]
        def call(out, work, stream=None, where=(T, C, F, i % 3), args=args):
            cc.cacnn_gated_forward(where, 1, *args[:3], out[0], gate=out[1], up=out[2], stream=stream)
            cc.cacnn_gated_backward(where, 1, *args, *out[3:], work, gate=out[1], up=out[2], stream=stream)
        new = lambda: [torch.zeros(s, dtype=torch.bfloat16, device="cuda") for s in ((T, F), (T, F), (T, F), (T, C), (F, C), (F, C))]  # noqa: E731
        work = torch.zeros(cc.cacnn_gated_workspace((T, C, F, 0), 1), dtype=torch.uint8, device="cuda")
        alone = new()
        call(alone, work)
        jobs.append((call, new(), torch.zeros_like(work), torch.cuda.Stream(), alone))
    torch.cuda.synchronize()
    for _ in range(3):
        for call, out, work, stream, _ in jobs:
            call(out, work, stream)
    torch.cuda.synchronize()
    for _, out, _, _, alone in jobs:
        assert all(torch.equal(a, b) for a, b in zip(out, alone))
