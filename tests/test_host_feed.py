"""What the feed-forward entry points refuse, before a GPU is looked for (nothing runs)."""
import ctypes

import pytest
import torch

import paper_1802_06905_amd as cc
from paper_1802_06905_amd import binding

NULL, INVALID, UNSUPPORTED, LAUNCH, NO_DEVICE = 1, 2, 3, 4, 5
LIB = binding._lib
A = 1 << 20                                             # addresses that nothing reads


def quantize(T=4, C=256, rows=1, ld_x=0, ld_q=0, dtype=0, x=A, q=A, s=A):
    return LIB.cacnn_quantize(ctypes.byref(cc.QuantizeProblem(T, C, rows, ld_x, ld_q)), dtype, x, q, s, None)


def matmul(T=4, C=256, K=64, ld_x=0, ld_w=0, ld_out=0, x=A, xs=A, w=A, ws=A, out_dtype=1, out=A):
    return LIB.cacnn_matmul_scaled(ctypes.byref(cc.MatmulProblem(T, C, K, ld_x, ld_w, ld_out)), x, xs, w, ws, out_dtype, out, None)


def forward(T=4, C=256, F=64, act=0, dtype=1, x=A, wg=A, wu=A, out=A, gate=None, up=None, **ld):
    return LIB.cacnn_gated_forward(ctypes.byref(cc.GatedProblem(T, C, F, act, **ld)), dtype, x, wg, wu, out, gate, up, None)


def forward_scaled(T=4, C=256, F=64, act=0, x=A, xs=A, wg=A, gs=A, wu=A, us=A, out_dtype=1, out=A, **ld):
    return LIB.cacnn_gated_forward_scaled(ctypes.byref(cc.GatedProblem(T, C, F, act, **ld)), x, xs, wg, gs, wu, us, out_dtype, out, None)


def backward(T=4, C=256, F=64, act=0, dtype=1, x=A, wg=A, wu=A, gate=None, up=None, dy=A, gx=A, gg=A, gu=A, work=A, size=2 * 4 * 64 * 2, **ld):
    return LIB.cacnn_gated_backward(ctypes.byref(cc.GatedProblem(T, C, F, act, **ld)), dtype, x, wg, wu, gate, up, dy, gx, gg, gu, work, size, None)


BIG = (1 << 20) + 1
REFUSED = [
    (quantize, NULL, [dict(x=None), dict(q=None), dict(s=None)]),
    (quantize, UNSUPPORTED, [dict(dtype=2), dict(dtype=-1), dict(rows=2), dict(rows=0)]),
    (quantize, INVALID, [dict(T=-1), dict(T=1 << 31), dict(C=0), dict(C=BIG), dict(ld_x=255), dict(ld_q=BIG), dict(ld_x=-1), dict(x=A + 2), dict(s=A + 1)]),
    (matmul, NULL, [dict(x=None), dict(xs=None), dict(w=None), dict(ws=None), dict(out=None), dict(T=0, w=None)]),
    (matmul, UNSUPPORTED, [dict(out_dtype=2)]),
    (matmul, INVALID, [dict(T=-1), dict(C=0), dict(K=0), dict(K=BIG), dict(ld_x=255), dict(ld_w=255), dict(ld_out=63), dict(xs=A + 2), dict(ws=A + 1),
                       dict(out=A + 1), dict(T=(1 << 31) - 1, K=1 << 20)]),
    (forward, NULL, [dict(x=None), dict(wg=None), dict(wu=None), dict(out=None)]),
    (forward, UNSUPPORTED, [dict(dtype=2), dict(act=3), dict(act=-1)]),
    (forward, INVALID, [dict(T=-1), dict(C=0), dict(F=0), dict(F=BIG), dict(ld_x=255), dict(ld_w=-1), dict(ld_out=63), dict(gate=A), dict(up=A), dict(x=A + 1),
                        dict(gate=A + 1, up=A), dict(dtype=0, wg=A + 2), dict(gate=A, up=A, ld_pre=32), dict(T=(1 << 31) - 1, F=64, C=1 << 20), dict(F=1 << 20, C=1 << 20)]),
    (forward_scaled, NULL, [dict(x=None), dict(xs=None), dict(wg=None), dict(gs=None), dict(wu=None), dict(us=None), dict(out=None)]),
    (forward_scaled, UNSUPPORTED, [dict(out_dtype=2), dict(act=9)]),
    (forward_scaled, INVALID, [dict(C=0), dict(T=-5), dict(xs=A + 2), dict(us=A + 2), dict(out=A + 1), dict(ld_w=7)]),
    (backward, NULL, [dict(x=None), dict(wg=None), dict(wu=None), dict(dy=None), dict(work=None)]),
    (backward, UNSUPPORTED, [dict(dtype=2), dict(act=3)]),
    (backward, INVALID, [dict(gg=None), dict(gu=None), dict(gx=None, gg=None, gu=None), dict(gate=A), dict(size=2 * 4 * 64 * 2 - 1), dict(work=A + 8),
                         dict(dy=A + 1), dict(ld_grad_x=3), dict(ld_grad_w=3), dict(F=0), dict(dtype=0)]),
]


@pytest.mark.parametrize("call,status,changes", [(c, s, d) for c, s, all_ in REFUSED for d in all_], ids=lambda v: getattr(v, "__name__", str(v)))
def test_refusals(call, status, changes):
    assert call(**changes) == status


@pytest.mark.parametrize("call", [quantize, matmul, forward, forward_scaled, backward])
def test_a_good_call_without_a_gpu_says_so(call):
    if torch.cuda.is_available():
        pytest.skip("a GPU is there: the call would run")
    assert call() == NO_DEVICE
    assert call(T=0) == NO_DEVICE


def test_null_problems():
    assert LIB.cacnn_quantize(None, 0, A, A, A, None) == NULL
    assert LIB.cacnn_matmul_scaled(None, A, A, A, A, 0, A, None) == NULL
    assert LIB.cacnn_gated_forward(None, 0, A, A, A, A, None, None, None) == NULL
    assert LIB.cacnn_gated_workspace(None, 0, ctypes.byref(ctypes.c_size_t())) == NULL


def test_workspace():
    assert cc.cacnn_gated_workspace((4, 256, 64, 0), 1) == 2 * 4 * 64 * 2
    assert cc.cacnn_gated_workspace((5, 256, 65, 0), 0) == 2 * 5 * 128 * 4
    assert cc.cacnn_gated_workspace((1 << 20, 8, 1 << 16, 2), 1) == 2 << 37
    # rows of C elements that are no multiple of 16 bytes are copied where there are enough of them
    assert cc.cacnn_gated_workspace((500, 7, 65, 0), 0) == 2 * 500 * 128 * 4 + (500 + 2 * 65) * 64 * 4
    assert cc.cacnn_gated_workspace((500, 8, 65, 0), 0) == cc.cacnn_gated_workspace((500, 12, 65, 0), 0) == 2 * 500 * 128 * 4
    for bad, status in (((4, 0, 64, 0), INVALID), ((4, 8, 64, 7), UNSUPPORTED)):
        with pytest.raises(cc.CacnnError) as e:
            cc.cacnn_gated_workspace(bad, 1)
        assert e.value.status == status


class Device(torch.Tensor):
    """A tensor on the CPU that says it is on a GPU."""
    is_cuda = True
    where = torch.device("cuda", 0)

    @property
    def device(self):
        return self.where


def on(*shape, dtype=torch.bfloat16, device=0):
    t = torch.zeros(shape, dtype=dtype).as_subclass(Device)
    t.where = torch.device("cuda", device)
    return t


@pytest.fixture
def calls(monkeypatch):
    """The library's answers are 0 and its calls are noted."""
    noted = []

    class Library:
        def __getattr__(self, name):
            if not name.startswith(("cacnn_gated", "cacnn_quantize", "cacnn_matmul")):
                return getattr(LIB, name)

            def call(problem, *args):
                noted.append((name, problem._obj, args))
                return 0
            return call
    monkeypatch.setattr(binding, "_lib", Library())
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(binding, "_stream_handle", lambda s: 77 if s is None else s)
    return noted


def good(**changes):
    args = dict(x=on(4, 256), w_gate=on(64, 256), w_up=on(64, 256), out=on(4, 64), gate=None, up=None)
    args.update(changes)
    return args


def test_strides_come_from_the_tensors(calls):
    wide = on(4, 300)[:, :256]
    cc.cacnn_gated_forward((4, 256, 64, 1), 1, **good(x=wide, gate=on(4, 64), up=on(4, 64)))
    (name, p, args), = calls
    assert name == "cacnn_gated_forward" and (p.ld_x, p.ld_w, p.ld_out, p.ld_pre) == (300, 256, 64, 64) and args[-1] == 77
    # a single row's stride is nobody's, and a problem's own stride has to be the tensor's
    cc.cacnn_gated_forward((1, 256, 64, 0), 1, **good(x=on(4, 300)[:1, :256], out=on(1, 64)))
    assert calls[-1][1].ld_x == 0
    said = cc.GatedProblem(4, 256, 64, 0, ld_x=300)
    cc.cacnn_gated_forward(said, 1, **good(x=wide))
    with pytest.raises(ValueError, match="the problem says 300"):
        cc.cacnn_gated_forward(said, 1, **good())
    assert said.ld_w == 0 and len(calls) == 3


BAD = [
    (dict(x=on(4, 255)), "x is"), (dict(x=on(5, 256)), "x is"), (dict(x=on(4, 256, dtype=torch.float16)), "float16"), (dict(w_up=on(64, 256, dtype=torch.float32)), "float32"),
    (dict(x=on(256, 4).t()), "contiguous"), (dict(out=on(1, 64).expand(4, 64)), "overlap"), (dict(w_up=on(64, 300)[:, :256]), "elements apart"),
    (dict(w_up=on(64, 256, device=1)), "on cuda:1"), (dict(gate=on(4, 64), up=on(4, 70)[:, :64]), "elements apart"), (dict(x=torch.zeros(4, 256, dtype=torch.bfloat16)), "device"),
]


@pytest.mark.parametrize("changes,message", BAD, ids=[m for _, m in BAD])
def test_tensors_that_do_not_fit(calls, changes, message):
    with pytest.raises(ValueError, match=message):
        cc.cacnn_gated_forward((4, 256, 64, 0), 1, **good(**changes))
    assert not calls


def test_more_that_does_not_fit(calls):
    with pytest.raises(TypeError):
        cc.cacnn_gated_forward((4, 256, 64, 0), 1, **good(x=5))
    with pytest.raises(cc.CacnnError):
        cc.cacnn_gated_forward((4, 256, 64, 0), 9, **good())
    with pytest.raises(ValueError, match="contiguous"):
        cc.cacnn_quantize((4, 256, 1), 1, on(4, 256), on(4, 256, dtype=torch.uint8), on(4, 3, dtype=torch.float32)[:, :2])
    with pytest.raises(cc.CacnnError):
        cc.cacnn_quantize((4, 256, 0), 1, on(4, 256), on(4, 256, dtype=torch.uint8), on(4, 2, dtype=torch.float32))
    with pytest.raises(ValueError, match="w_scale is"):
        cc.cacnn_matmul_scaled((4, 256, 130), on(4, 256, dtype=torch.uint8), on(4, 2, dtype=torch.float32), on(130, 256, dtype=torch.uint8),
                               on(1, 2, dtype=torch.float32), 0, on(4, 130, dtype=torch.float32))
    grads = dict(x=on(4, 256), w_gate=on(64, 256), w_up=on(64, 256), grad_out=on(4, 64), grad_x=on(4, 256), grad_w_gate=None, grad_w_up=None)
    with pytest.raises(ValueError, match="workspace"):
        cc.cacnn_gated_backward((4, 256, 64, 0), 1, **grads, workspace=torch.zeros(4096, dtype=torch.uint8))
    for work in (on(64, 64, dtype=torch.uint8).t(), None, 4096):
        with pytest.raises(ValueError, match="workspace"):
            cc.cacnn_gated_backward((4, 256, 64, 0), 1, **grads, workspace=work)
    assert not calls


# ---- which kernel a product runs on
W32, W64_32, W64, DEEP, MIDDLE, LARGE, SMALL = range(7)


def kernel(form, dtype, M, N, k, direct=1):
    LIB.cacnn_internal_matmul_kernel.argtypes = [ctypes.c_int] * 3 + [ctypes.c_int64] * 3
    return LIB.cacnn_internal_matmul_kernel(form, dtype, direct, M, N, k)


def test_a_kernel_for_every_size():
    """Few rows are divided among waves, many rows take the large tiles, and nothing asks for a kernel that the type or its operands have not."""
    plain, e4m3 = 1, 2
    assert [kernel(plain, e4m3, T, 4096, 4096) for T in (1, 32, 256, 1024, 2048, 8192)] == [W32, W32, W64, DEEP, MIDDLE, LARGE]
    assert [kernel(0, 1, T, 8192, 4096) for T in (1, 64, 256, 8192)] == [W32, W64_32, DEEP, LARGE]
    for form in range(4):
        for dtype in range(4):
            for M in (1, 7, 100, 1000, 10000, (1 << 31) - 1):
                for N in (1, 100, 5000, 1 << 20):
                    for k in (0, 1, 100, 10000):
                        for direct in (0, 1):
                            chosen = kernel(form, dtype, M, N, k, direct)
                            assert chosen not in (DEEP, LARGE) or direct
                            assert chosen != LARGE or dtype in (1, 2)
                            assert chosen != SMALL or dtype == 0
                            assert form != 0 or chosen != W64


def test_the_module_leaves_what_is_not_usual():
    if binding._native is None:
        pytest.skip("the module was not built")
    t = torch.zeros((4, 256), dtype=torch.bfloat16)
    for args in ((), (1,) * 6, ((4, 256, 1), 1, t, t, t, None), ((4, 256), 1, t, t, t, None), (cc.QuantizeProblem(4, 256, 1), 1, t, t, t, None),
                 ((0, 256, 1), 1, t, t, t, None), ((4, 256, 1), 7, t, t, t, None), ((4, 256, 3), 1, t, t, t, None), ((1 << 40, 256, 1), 1, t, t, t, None)):
        assert binding._native.quantize(*args) == -1
