"""GPU parity of the feed-forward operators against the 64-bit oracle, within bounds that count roundings (oracle/feed.py).  Operands lie inside
arrays of NaN and results inside arrays of a mark, so that what is read or written beside them shows."""
import numpy as np
import pytest

from tests.feed_util import GATES, Result, put, rounded, within
from oracle import feed

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    import paper_1802_06905_amd as cc
    assert torch.cuda.is_available(), "these tests need the GPU"
    return cc, torch


def code(cc, dtype):
    return cc.CACNN_F32 if dtype == "f32" else cc.CACNN_BF16_F32ACC


def typ(torch, dtype):
    return torch.float32 if dtype == "f32" else torch.bfloat16


def activations(rng, T, C):
    x = rng.normal(size=(T, C)) * np.exp(0.5 * rng.normal(size=C))
    if T > 2:
        x[2::5] = 0                                     # padding
    return x


# ---- quantisation
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,C,pad,shift", [(1, 1, 0, 0), (1, 4096, 0, 0), (3, 127, 0, 0), (2, 128, 8, 0), (130, 129, 0, 1), (257, 400, 3, 0),
                                           (128, 2056, 0, 0), (5, 2049, 7, 3), (300, 8, 0, 0)])
def test_quantize(env, T, C, pad, shift, dtype, block_rows):
    cc, torch = env
    rng = np.random.default_rng(T * 1000 + C)
    x, t = rounded(torch, activations(rng, T, C) * 10.0 ** rng.integers(-30, 30, size=(T, 1)), dtype)
    bits, scale = feed.quantize(x, block_rows)
    q = Result(torch, T, C, torch.uint8, pad, shift)
    s = Result(torch, *scale.shape, torch.float32)
    cc.cacnn_quantize((T, C, block_rows), code(cc, dtype), put(torch, t, pad, shift), q.view, s.view)
    assert np.array_equal(s.numpy(), scale)
    assert np.array_equal(q.view.cpu().numpy(), bits)
    q.check(), s.check()


@pytest.mark.parametrize("block_rows", [1, 128])
def test_quantize_borders_subnormals_and_what_is_not_finite(env, block_rows):
    """Every number in 8 bits, every middle between two and its neighbours; scales at either end of their range; NaN and infinities."""
    cc, torch = env
    v = feed.e4m3_values()[:127]
    middle = ((v[1:] + v[:-1]) / 2).astype(np.float32)
    x = np.concatenate((v, middle, np.nextafter(middle, np.float32(0)), np.nextafter(middle, np.float32(500)))).astype(np.float32)
    x = np.concatenate((x, -x))
    x = np.concatenate((x, np.full(-len(x) % 127, 448.0, np.float32))).reshape(-1, 127)
    x = np.concatenate((x, np.full((len(x), 1), 448.0, np.float32)), 1)         # every block's scale is 1
    wild = np.zeros((6, 128), np.float32)
    wild[0, :3], wild[1, :4], wild[2, :2] = (1e-45, -3e-39, 1e-40), (np.nan, 2.0, -np.inf, np.inf), (np.finfo(np.float32).max, -1.0)
    wild[3, 7], wild[4, :] = 448 * 1.0000001, np.nan
    for rows in (x, wild[:3] if block_rows == 1 else wild[1:2], wild):
        bits, scale = feed.quantize(rows, block_rows)
        q = torch.zeros(rows.shape, dtype=torch.uint8, device="cuda")
        s = torch.zeros(scale.shape, device="cuda")
        cc.cacnn_quantize((*rows.shape, block_rows), cc.CACNN_F32, torch.from_numpy(rows).cuda(), q, s)
        assert np.array_equal(s.cpu().numpy(), scale)
        got = q.cpu().numpy()
        nan = (bits & 0x7f) == 0x7f
        assert np.array_equal((got & 0x7f) == 0x7f, nan) and np.array_equal(got[~nan], bits[~nan])


# ---- the product of operands in 8 bits
def scaled(torch, rng, rows, cols, block_rows):
    """Random bytes and scales of no special form, and what they stand for."""
    bits = feed.e4m3_bits(np.clip(rng.normal(size=(rows, cols)) * 60, -448, 448))
    scale = np.exp(rng.normal(size=(-(-rows // block_rows), -(-cols // 128)))).astype(np.float32) / 60
    return feed.stands_for(bits, scale, block_rows), torch.from_numpy(bits).view(torch.float8_e4m3fn), torch.from_numpy(scale)


PRODUCTS = [  # T, C, K, pad, shift
    (1, 1, 1, 0, 0), (1, 128, 32, 0, 0), (1, 4096, 200, 0, 0), (2, 127, 129, 0, 0), (31, 1000, 65, 0, 0), (33, 256, 1111, 3, 0), (64, 1040, 96, 0, 0),
    (65, 129, 128, 0, 1), (128, 512, 256, 16, 0), (130, 272, 260, 0, 0), (517, 100, 333, 0, 5), (300, 2048, 384, 0, 0), (700, 384, 640, 0, 16), (40, 15, 300, 1, 0), (200, 16, 70, 0, 3),
]


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("T,C,K,pad,shift", PRODUCTS)
def test_matmul_scaled(env, T, C, K, pad, shift, out):
    cc, torch = env
    rng = np.random.default_rng(T + 7 * C + 13 * K)
    x, xq, xs = scaled(torch, rng, T, C, 1)
    w, wq, ws = scaled(torch, rng, K, C, 128)
    y = Result(torch, T, K, typ(torch, out), pad, shift)
    cc.cacnn_matmul_scaled((T, C, K), put(torch, xq, pad, shift), xs.cuda(), put(torch, wq, pad, shift), ws.cuda(), code(cc, out), y.view)
    within("out", y.numpy(), *feed.matmul_scaled(x, w, feed.HALF_STEP[out], feed.cut_off(x, w) if out == "bf16" else 0.0))
    y.check()


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("T", [2, 300])
def test_every_8_bit_number(env, T, out):
    """Each of the 254 finite numbers, subnormal ones among them, times one: bf16 holds them all."""
    cc, torch = env
    x = torch.arange(254, dtype=torch.uint8)
    x = torch.where(x < 127, x, x + 1).view(2, 127).repeat(T // 2, 1)
    w = torch.where(torch.eye(127, dtype=torch.bool), 0x38, 0).to(torch.uint8)      # 0x38 is 1
    y = torch.zeros((T, 127), dtype=typ(torch, out), device="cuda")
    one = lambda n: torch.ones((n, 1), device="cuda")  # noqa: E731
    cc.cacnn_matmul_scaled((T, 127, 127), x.cuda(), one(T), w.cuda(), one(1), code(cc, out), y)
    assert np.array_equal(y.cpu().double().numpy(), feed.e4m3_values()[x.numpy()])


def test_a_nan_stays_in_its_row_and_column(env):
    cc, torch = env
    rng = np.random.default_rng(5)
    T, C, K = 40, 300, 70
    _, xq, xs = scaled(torch, rng, T, C, 1)
    _, wq, ws = scaled(torch, rng, K, C, 128)
    xq.view(torch.uint8)[7, 299] = 0x7f
    wq.view(torch.uint8)[69, 0] = 0xff
    y = torch.zeros((T, K), device="cuda")
    cc.cacnn_matmul_scaled((T, C, K), xq.cuda(), xs.cuda(), wq.cuda(), ws.cuda(), cc.CACNN_F32, y)
    nan = torch.isnan(y).cpu().numpy()
    expect = np.zeros((T, K), bool)
    expect[7, :], expect[:, 69] = True, True
    assert np.array_equal(nan, expect)


@pytest.mark.parametrize("gate", GATES)
@pytest.mark.parametrize("T,C,F,pad,shift", [(1, 1, 1, 0, 0), (1, 1024, 100, 0, 0), (16, 512, 128, 0, 0), (33, 130, 200, 3, 0), (64, 1040, 96, 0, 0), (150, 300, 333, 0, 1),
                                             (260, 640, 256, 0, 0), (600, 256, 512, 16, 0)])
def test_gated_forward_scaled(env, T, C, F, pad, shift, gate):
    cc, torch = env
    rng = np.random.default_rng(T + 7 * C + 13 * F)
    x, xq, xs = scaled(torch, rng, T, C, 1)
    xs, x = xs / C ** 0.5, x / C ** 0.5
    x = feed.stands_for(xq.view(torch.uint8).numpy(), xs.numpy(), 1)
    wg, gq, gs = scaled(torch, rng, F, C, 128)
    wu, uq, us = scaled(torch, rng, F, C, 128)
    out = ("f32", "bf16")[T % 2]
    y = Result(torch, T, F, typ(torch, out), pad, shift)
    cc.cacnn_gated_forward_scaled((T, C, F, GATES.index(gate)), put(torch, xq, pad, shift), xs.cuda(), put(torch, gq, pad, shift), gs.cuda(),
                                  put(torch, uq, pad, shift), us.cuda(), code(cc, out), y.view)
    cut = [feed.cut_off(x, w) if out == "bf16" else 0.0 for w in (wg, wu)]
    within("out", y.numpy(), *feed.gated(x, wg, wu, gate, feed.HALF_STEP[out], sums=128 + -(-C // 128) + 2, cut=cut)["out"])
    y.check()


# ---- the gated projection and its gradients
SHAPES = [  # T, C, F, pad, shift
    (1, 1, 1, 0, 0), (1, 1024, 96, 0, 0), (2, 7, 65, 0, 0), (17, 512, 128, 0, 0), (32, 1000, 72, 8, 0), (33, 129, 200, 3, 0), (64, 264, 320, 0, 0),
    (65, 64, 33, 0, 1), (129, 255, 130, 0, 0), (256, 512, 256, 0, 8), (300, 1032, 200, 0, 0), (640, 320, 704, 0, 0),
    (200, 64, 96, 0, 1), (150, 3, 40, 0, 0), (3, 5, 1000, 2, 1),
]


def problem(torch, dtype, T, C, F, seed):
    rng = np.random.default_rng(seed)
    x, wg, wu = activations(rng, T, C), rng.normal(size=(F, C)) / C ** 0.5, rng.normal(size=(F, C)) / C ** 0.5
    return [rounded(torch, a, dtype) for a in (x, wg, wu, rng.normal(size=(T, F)) * 1e-2)]


@pytest.mark.parametrize("gate", GATES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,C,F,pad,shift", SHAPES)
def test_gated_forward(env, T, C, F, pad, shift, dtype, gate):
    cc, torch = env
    (x, tx), (wg, tg), (wu, tu), _ = problem(torch, dtype, T, C, F, T + C + F)
    y, g, u = (Result(torch, T, F, typ(torch, dtype), pad, shift) for _ in range(3))
    args = [put(torch, t, pad, shift) for t in (tx, tg, tu)]
    where = (T, C, F, GATES.index(gate))
    cc.cacnn_gated_forward(where, code(cc, dtype), *args, y.view, gate=g.view, up=u.view)
    expect = feed.gated(x, wg, wu, gate, feed.HALF_STEP[dtype])
    for name, r in (("out", y), ("gate", g), ("up", u)):
        within(name, r.numpy(), *expect[name])
        r.check()
    alone = Result(torch, T, F, typ(torch, dtype), pad, shift)
    cc.cacnn_gated_forward(where, code(cc, dtype), *args, alone.view)
    assert torch.equal(alone.flat, y.flat)


@pytest.mark.parametrize("keep", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,C,F,pad,shift", SHAPES)
def test_gated_backward(env, T, C, F, pad, shift, dtype, keep):
    cc, torch = env
    gate = GATES[(T + F) % 3]
    (x, tx), (wg, tg), (wu, tu), (dy, td) = problem(torch, dtype, T, C, F, T + C + F + 1)
    g, u = (rounded(torch, x @ w.T, dtype) for w in (wg, wu))
    gx = Result(torch, T, C, typ(torch, dtype), pad, shift)
    gg, gu = (Result(torch, F, C, typ(torch, dtype), pad, shift) for _ in range(2))
    where = (T, C, F, GATES.index(gate))
    size = cc.cacnn_gated_workspace(where, code(cc, dtype))
    workspace = torch.full((size + 64,), 0xff, dtype=torch.uint8, device="cuda")
    kept = {"gate": put(torch, g[1], pad, shift), "up": put(torch, u[1], pad, shift)} if keep else {}
    cc.cacnn_gated_backward(where, code(cc, dtype), *[put(torch, t, pad, shift) for t in (tx, tg, tu, td)], gx.view, gg.view, gu.view, workspace[:size], **kept)
    expect = feed.gated_backward(x, wg, wu, dy, gate, feed.HALF_STEP[dtype], *((g[0], u[0]) if keep else ()))
    for name, r in (("grad_x", gx), ("grad_w_gate", gg), ("grad_w_up", gu)):
        within(name, r.numpy(), *expect[name])
        r.check()
    assert bool((workspace[size:] == 0xff).all())


def test_gradients_that_are_not_wanted(env):
    cc, torch = env
    T, C, F = 70, 96, 136
    args = [t.cuda() for _, t in problem(torch, "bf16", T, C, F, 3)]
    where = (T, C, F, cc.CACNN_GATE_SILU)
    workspace = torch.empty(cc.cacnn_gated_workspace(where, 1), dtype=torch.uint8, device="cuda")
    new = lambda r, c: torch.full((r, c), 5.0, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    x, g, u = new(T, C), new(F, C), new(F, C)
    cc.cacnn_gated_backward(where, 1, *args, x, g, u, workspace)
    x2, g2, u2 = new(T, C), new(F, C), new(F, C)
    cc.cacnn_gated_backward(where, 1, *args, x2, None, None, workspace)
    cc.cacnn_gated_backward(where, 1, *args, None, g2, u2, workspace)
    assert torch.equal(x, x2) and torch.equal(g, g2) and torch.equal(u, u2)


@pytest.mark.parametrize("C,F", [(72, 40), (3, 40)])
def test_no_tokens(env, C, F):
    cc, torch = env
    empty = lambda n, t=torch.bfloat16: torch.empty((0, n), dtype=t, device="cuda")  # noqa: E731
    w = torch.randn((F, C), device="cuda").bfloat16()
    g, u = torch.full_like(w, 3), torch.full_like(w, 3)
    where = (0, C, F, cc.CACNN_GATE_SILU)
    cc.cacnn_gated_forward(where, 1, empty(C), w, w, empty(F), gate=empty(F), up=empty(F))
    assert cc.cacnn_gated_workspace(where, 1) == 0
    cc.cacnn_gated_backward(where, 1, empty(C), w, w, empty(F), empty(C), g, u, torch.empty(0, dtype=torch.uint8, device="cuda"))
    assert not g.any() and not u.any()
    byte = torch.uint8
    cc.cacnn_quantize((0, C, 1), 1, empty(C), empty(C, byte), empty(1, torch.float32))
    wq = torch.zeros((F, C), dtype=byte, device="cuda")
    cc.cacnn_matmul_scaled((0, C, F), empty(C, byte), empty(1, torch.float32), wq, torch.ones((1, 1), device="cuda"), 0, empty(F, torch.float32))


def test_infinities_and_nan_stay_in_their_tokens(env):
    """A token of NaN, one of infinities: other tokens' results, and the gradient of the other tokens, are what they are without."""
    cc, torch = env
    T, C, F = 45, 136, 72
    (_, x), (_, wg), (_, wu), (_, dy) = problem(torch, "bf16", T, C, F, 9)
    x, wg, wu, dy = (t.cuda() for t in (x, wg, wu, dy))
    where = (T, C, F, cc.CACNN_GATE_GELU_TANH)
    bad = x.clone()
    bad[11, 5], bad[30] = float("nan"), float("inf")
    workspace = torch.empty(cc.cacnn_gated_workspace(where, 1), dtype=torch.uint8, device="cuda")
    results = []
    for data in (x, bad):
        y, gx = torch.zeros((T, F), dtype=torch.bfloat16, device="cuda"), torch.zeros((T, C), dtype=torch.bfloat16, device="cuda")
        cc.cacnn_gated_forward(where, 1, data, wg, wu, y)
        cc.cacnn_gated_backward(where, 1, data, wg, wu, dy, gx, None, None, workspace)
        results.append((y, gx))
    rest = [t for t in range(T) if t not in (11, 30)]
    for a, b in zip(*results):
        assert torch.equal(a[rest], b[rest]) and torch.isnan(b[11]).all() and not torch.isfinite(b[30]).all()


def test_far_gates(env):
    """Gates far from zero: act(g) is g or nothing, and the slopes are 1 or 0, without NaN from infinities on the way."""
    cc, torch = env
    g = torch.tensor([[1e20, -1e20, 3e38, -3e38, 100.0, -100.0, 0.0, -0.0]], device="cuda").t().contiguous()
    T = g.shape[0]
    one = torch.ones((1, 1), device="cuda")
    for gate in range(3):
        where = (T, 1, 1, gate)
        workspace = torch.empty(cc.cacnn_gated_workspace(where, 0), dtype=torch.uint8, device="cuda")
        gx, gg, gu = torch.zeros_like(g), torch.zeros((1, 1), device="cuda"), torch.zeros((1, 1), device="cuda")
        cc.cacnn_gated_backward(where, 0, torch.zeros_like(g), one, torch.zeros_like(one), torch.ones_like(g), gx, gg, gu, workspace, gate=g, up=torch.ones_like(g))
        assert torch.equal(gx.cpu().flatten(), torch.tensor([1.0, 0, 1, 0, 1, 0, 0.5, 0.5]))
        y = torch.zeros_like(g)
        cc.cacnn_gated_forward(where, 0, g, one, one / g[0, 0], y)
        expect = torch.where(g > 0, g, 0) * (g * (one / g[0, 0]))
        assert torch.allclose(y, expect, rtol=1e-5, atol=1e-30)


# ---- together, on streams, in graphs
def test_a_block_in_8_bits(env):
    """Serving: quantise the tokens, gated projection, quantise, project back; against the same in 64 bits on the kernels' own 8-bit operands."""
    cc, torch = env
    T, C, F = 37, 384, 520
    rng = np.random.default_rng(11)
    _, x = rounded(torch, activations(rng, T, C), "bf16")
    w = [rounded(torch, rng.normal(size=s) / s[1] ** 0.5, "bf16")[1].cuda() for s in ((F, C), (F, C), (C, F))]

    def eight(t, rows):
        q = torch.empty(t.shape, dtype=torch.float8_e4m3fn, device="cuda")
        s = torch.empty((-(-t.shape[0] // rows), -(-t.shape[1] // 128)), device="cuda")
        cc.cacnn_quantize((*t.shape, rows), 1, t, q, s)
        return q, s, feed.stands_for(q.view(torch.uint8).cpu().numpy(), s.cpu().numpy(), rows)

    xq, xs, x64 = eight(x.cuda(), 1)
    (gq, gs, g64), (uq, us, u64), (dq, ds, d64) = (eight(t, 128) for t in w)
    h = torch.empty((T, F), dtype=torch.bfloat16, device="cuda")
    cc.cacnn_gated_forward_scaled((T, C, F, cc.CACNN_GATE_SILU), xq, xs, gq, gs, uq, us, cc.CACNN_BF16_F32ACC, h)
    cut = [feed.cut_off(x64, w) for w in (g64, u64)]
    value, bound = feed.gated(x64, g64, u64, "silu", 2.0 ** -8, sums=128 + 3 + 2, cut=cut)["out"]
    within("hidden", h.cpu().double().numpy(), value, bound)
    hq, hs, h64 = eight(h, 1)
    y = torch.empty((T, C), device="cuda")
    cc.cacnn_matmul_scaled((T, F, C), hq, hs, dq, ds, cc.CACNN_F32, y)
    within("out", y.cpu().double().numpy(), *feed.matmul_scaled(h64, d64, 2.0 ** -24))


def test_a_training_step_moves_against_its_gradient(env):
    """Forward that keeps its products, backward from them: the change of the loss along each gradient is its square, by differences in 64 bits."""
    cc, torch = env
    T, C, F = 50, 72, 88
    (x, tx), (wg, tg), (wu, tu), (dy, td) = problem(torch, "f32", T, C, F, 21)
    x_, g_, u_, d_ = (t.cuda() for t in (tx, tg, tu, td))
    y, gate, up = (torch.empty((T, F), device="cuda") for _ in range(3))
    where = (T, C, F, cc.CACNN_GATE_GELU)
    cc.cacnn_gated_forward(where, 0, x_, g_, u_, y, gate=gate, up=up)
    grads = [torch.empty_like(t) for t in (x_, g_, u_)]
    workspace = torch.empty(cc.cacnn_gated_workspace(where, 0), dtype=torch.uint8, device="cuda")
    cc.cacnn_gated_backward(where, 0, x_, g_, u_, d_, *grads, workspace, gate=gate, up=up)
    step = 1e-4

    def loss(i, sign):
        arrays = [x, wg, wu]
        arrays[i] = arrays[i] + sign * step * grads[i].cpu().double().numpy()
        return (feed.gated(*arrays, "gelu", 0.0)["out"][0] * dy).sum()

    for i, grad in enumerate(grads):
        square = float((grad.double() ** 2).sum())
        # (differences are off by the third derivative times step^2 |grad|^3, and the gradient by its 32-bit roundings)
        assert abs((loss(i, 1) - loss(i, -1)) / (2 * step) - square) < 1e-4 * square


@pytest.mark.parametrize("T", [3, 200])
def test_graphs_and_streams(env, T):
    """Every operator on a side stream, and captured into a graph that is replayed between eager calls on new inputs, gives the eager call's bits."""
    cc, torch = env
    C, F = 264, 200
    data = [problem(torch, "bf16", T, C, F, s) for s in (1, 2, 3)]
    fixed = [t.cuda() for _, t in data[0]]
    where = (T, C, F, cc.CACNN_GATE_SILU)
    new = lambda r, c, t=torch.bfloat16: torch.zeros((r, c), dtype=t, device="cuda")  # noqa: E731

    def results():
        return {"h": new(T, F), "gate": new(T, F), "up": new(T, F), "gx": new(T, C), "gg": new(F, C), "gu": new(F, C), "q": new(T, F, torch.uint8),
                "s": new(T, -(-F // 128), torch.float32), "y": new(T, C), "wq": new(C, F, torch.uint8), "ws": new(-(-C // 128), -(-F // 128), torch.float32),
                "work": torch.zeros(cc.cacnn_gated_workspace(where, 1), dtype=torch.uint8, device="cuda")}

    def step(args, r, stream=None):
        x, wg, wu, dy = args
        cc.cacnn_gated_forward(where, 1, x, wg, wu, r["h"], gate=r["gate"], up=r["up"], stream=stream)
        cc.cacnn_quantize((T, F, 1), 1, r["h"], r["q"], r["s"], stream=stream)
        cc.cacnn_quantize((C, F, 128), 1, wg.t().contiguous() if stream is None else fixed_t, r["wq"], r["ws"], stream=stream)
        cc.cacnn_matmul_scaled((T, F, C), r["q"], r["s"], r["wq"], r["ws"], 1, r["y"], stream=stream)
        cc.cacnn_gated_backward(where, 1, x, wg, wu, dy, r["gx"], r["gg"], r["gu"], r["work"], gate=r["gate"], up=r["up"], stream=stream)

    fixed_t = fixed[1].t().contiguous()
    eager, aside, replayed = results(), results(), results()
    step(fixed, eager)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    step(fixed, aside, side)
    torch.cuda.current_stream().wait_stream(side)
    for k in eager:
        assert torch.equal(eager[k], aside[k]), k

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(fixed, replayed)
    for d in data:
        for dst, (_, t) in zip(fixed, d):
            dst.copy_(t)
        expect = results()
        step(fixed, expect)
        torch.cuda.synchronize()
        for _ in range(2):
            graph.replay()
            torch.cuda.synchronize()
            for k in expect:
                assert torch.equal(expect[k], replayed[k]), k


def test_two_graphs_with_a_workspace_each_run_at_once(env):
    cc, torch = env
    T, C, F = 300, 256, 320
    where = (T, C, F, cc.CACNN_GATE_SILU)
    runs = []
    for seed in (4, 5):
        args = [t.cuda() for _, t in problem(torch, "bf16", T, C, F, seed)]
        out = [torch.zeros(s, dtype=torch.bfloat16, device="cuda") for s in ((T, C), (F, C), (F, C))]
        eager = [torch.zeros_like(o) for o in out]
        work = torch.zeros(cc.cacnn_gated_workspace(where, 1), dtype=torch.uint8, device="cuda")
        cc.cacnn_gated_backward(where, 1, *args, *eager, work)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            cc.cacnn_gated_backward(where, 1, *args, *out, work)
        runs.append((graph, torch.cuda.Stream(), out, eager, args, work))
    for _ in range(3):
        torch.cuda.synchronize()
        for graph, stream, *_ in runs:
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        for _, _, out, eager, *_ in runs:
            assert all(torch.equal(a, b) for a, b in zip(out, eager))


def test_rows_of_two_megabytes(env):
    """The longest rows, through registers (their first element is not at a multiple of 16 bytes) and straight to LDS; 3 tokens, gradients too."""
    cc, torch = env
    T, C, F = 3, 1 << 20, 24
    print("[feed] rows of 2 MB", flush=True)
    x, wg, wu = (torch.randn((n, C), device="cuda").mul_(C ** -0.25).bfloat16() for n in (T, F, F))
    dy = torch.randn((T, F), device="cuda").bfloat16()
    where = (T, C, F, cc.CACNN_GATE_SILU)
    results = []
    for shift in (0, 1):
        moved = []
        for t in (x, wg, wu):
            flat = torch.zeros(t.numel() + 8, dtype=t.dtype, device="cuda")
            flat[shift:shift + t.numel()].copy_(t.flatten())
            moved.append(flat[shift:shift + t.numel()].view(t.shape))
        y, gate, up = (torch.zeros((T, F), dtype=torch.bfloat16, device="cuda") for _ in range(3))
        cc.cacnn_gated_forward(where, 1, *moved, y, gate=gate, up=up)
        grads = [torch.zeros_like(t) for t in (x, wg, wu)]
        work = torch.empty(cc.cacnn_gated_workspace(where, 1), dtype=torch.uint8, device="cuda")
        cc.cacnn_gated_backward(where, 1, *moved, dy, *grads, work, gate=gate, up=up)
        results.append((y, gate, up, *grads))
    for a, b in zip(*results):
        # the same sums in the same order
        assert torch.equal(a, b)
    g = torch.zeros((T, F), dtype=torch.float64, device="cuda")
    for part in range(0, C, 1 << 16):
        g += x[:, part:part + (1 << 16)].double() @ wg[:, part:part + (1 << 16)].double().t().contiguous()
    # C + 1 roundings of the sum of magnitudes, about C * 2 / pi / C^(1/2), and half a step of bf16
    bound = (C + 1) * 2.0 ** -23 * C ** 0.5 * 0.7 + 2.0 ** -8 * g.abs()
    assert bool(((results[0][1].double() - g).abs() <= bound).all())
