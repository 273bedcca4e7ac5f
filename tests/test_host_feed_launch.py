"""What the feed-forward operators hand to the runtime, with a stand-in for the runtime (tests/hip_stand_in.cpp): nothing runs, no GPU is needed."""
import os
import subprocess
import sys

import pytest

import paper_1802_06905_amd as cc

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# (in a process of its own: the stand-in has to be there before the library looks for the runtime)
PRELUDE = r'''
import ctypes, random, re, sys
hip = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
lib = ctypes.CDLL(sys.argv[2])
hip.stand_in_launches.restype = ctypes.c_char_p
V, I = ctypes.c_void_p, ctypes.c_int
A = 1 << 20                                          # addresses that nothing reads
OK, INVALID = 0, 2
def struct(*n): return ctypes.byref((ctypes.c_int64 * len(n))(*n))
def kernels(): return hip.stand_in_launches().decode().split()
def matmul(T, C, K, out, ld=(0, 0, 0), x=A, w=A): return lib.cacnn_matmul_scaled(struct(T, C, K, *ld), V(x), V(A), V(w), V(A), I(out), V(A), V(0))
def scaled(T, C, F, out, act=0, ld=(0,) * 6, x=A, wg=A, wu=A):
    return lib.cacnn_gated_forward_scaled(struct(T, C, F, act, *ld), V(x), V(A), V(wg), V(A), V(wu), V(A), I(out), V(A), V(0))
def forward(T, C, F, dtype, act=0, ld=(0,) * 6, x=A, wg=A, wu=A):
    return lib.cacnn_gated_forward(struct(T, C, F, act, *ld), I(dtype), V(x), V(wg), V(wu), V(A), V(0), V(0), V(0))
def backward(T, C, F, dtype, keep=True, act=0, ld=(0,) * 6, x=A, wg=A, wu=A, grad_x=A, grad_w=A):
    p = struct(T, C, F, act, *ld)
    n = ctypes.c_size_t(0)
    rc = lib.cacnn_gated_workspace(p, I(dtype), ctypes.byref(n))
    kept = V(A if keep else 0)
    return rc or lib.cacnn_gated_backward(p, I(dtype), V(x), V(wg), V(wu), kept, kept, V(A), V(grad_x), V(grad_w), V(grad_w), V(A), n, V(0))
'''


@pytest.fixture(scope="module")
def run(tmp_path_factory):
    stand_in = str(tmp_path_factory.mktemp("stand_in") / "hip_stand_in.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-o", stand_in, os.path.join(ROOT, "tests", "hip_stand_in.cpp"), "-ldl"], check=True)

    def program(body):
        p = subprocess.run([sys.executable, "-c", PRELUDE + body, stand_in, cc.library_path()], capture_output=True, text=True, timeout=120)
        assert p.returncode == 0, p.stdout + p.stderr
        return p.stdout
    return program


def test_what_the_sizes_allow_can_be_launched(run):
    """Up to the limits on rows and columns no launch reaches 2^32 threads, whichever kernel would be the fastest: with few columns and short
    contractions that is one with small tiles."""
    run(r'''
for dtype in (0, 1):
    for T, C, F in ((1_100_000_000, 4, 1), (1_100_000_000, 64, 1), ((1 << 31) - 129, 8, 64), ((1 << 31) - 129, 64, 8)):
        for call in (lambda: forward(T, C, F, dtype), lambda: backward(T, C, F, dtype), lambda: backward(T, C, F, dtype, keep=False)):
            assert call() == OK, (dtype, T, C, F)
    for T, C, F in ((1, 1 << 20, 65535), (1, 65472, 1 << 20), (9, 1 << 14, 1 << 20)):      # the weights' gradients are the large ones
        rc = backward(T, C, F, dtype)
        assert rc == OK or (rc == INVALID and -(-2 * F // 128) * -(-C // 64) >= 1 << 24), (dtype, T, C, F, rc)
rng = random.Random(1)
taken = 0
for _ in range(4000):
    rows = int(2 ** rng.uniform(20, 31)) - 129
    cols, k = int(2 ** rng.uniform(0, 12)), int(2 ** rng.uniform(0, 20))
    dtype, out = rng.randint(0, 1), rng.randint(0, 1)
    for call in (lambda: matmul(rows, k, cols, out), lambda: scaled(rows, k, cols, out), lambda: forward(rows, k, cols, dtype),
                 lambda: backward(rows, k, cols, dtype), lambda: backward(rows, cols, k, dtype, keep=False), lambda: backward(cols, min(k, 1 << 12), min(rows, 1 << 20), dtype)):
        rc = call()
        assert rc in (OK, INVALID), (rows, cols, k, dtype, out, rc)
        taken += rc == OK
assert taken > 8000, taken
''')


PRODUCTS = r'''
def product(symbol):
    """The product's kernel that a symbol belongs to, with its template's arguments, or None."""
    m = re.search(r"matmul_(block|waves|short)_kernelI((?:L[ib]\d+E)+)", symbol)
    return m and m.group(1) + " " + ",".join(re.findall(r"L[ib](\d+)E", m.group(2)))
def launched(rc):
    assert rc == OK, rc
    return {product(k) for k in kernels()} - {None}
def listed(call, dtype, T, C, F, pad, shift):
    code, size = int(dtype == "bf16"), 1 if call in ("matmul", "scaled") else 2 if dtype == "bf16" else 4
    at = A + shift * size
    if call == "matmul": return launched(matmul(T, C, F, code, (C + pad, 0, 0), at))
    if call == "scaled": return launched(scaled(T, C, F, code, 0, (C + pad, 0, 0, 0, 0, 0), at))
    if call == "forward": return launched(forward(T, C, F, code, 0, (C + pad, 0, 0, 0, 0, 0), at))
    return launched(backward(T, C, F, code, True, 0, (C + pad, C + pad, 0, 0, C + pad, C + pad), at, at, at))
'''


def test_every_product_kernel_is_tested(run):
    """The calls listed for the kernels that bring operands through registers launch them, and those kernels, and the ones that the other tests on a GPU launch, are all
    that calls of many sizes, addresses and strides launch."""
    from tests import feed_shapes, test_gpu_feed, test_gpu_feed_kernels
    run(PRODUCTS + f"rows = {feed_shapes.THROUGH_REGISTERS!r}\nshapes = {test_gpu_feed_kernels.SHAPES!r}\nsmall = {test_gpu_feed.PRODUCTS + test_gpu_feed.SHAPES!r}\n" + r'''
tested = set()
for kernel, *call in rows:
    names = listed(*call)
    assert kernel in names and kernel.split(",")[-1] == "0", (kernel, call, names)
    tested.add(kernel)
for (form, dtype), all_ in shapes.items():
    for _, T, C, F in all_:
        if form == 1: tested |= listed("matmul", "bf16" if dtype == "e4m3" else "f32", T, C, F, 0, 0)
        elif dtype.startswith("e4m3"): tested |= listed("scaled", "bf16" if dtype == "e4m3" else "f32", T, C, F, 0, 0)
        else: tested |= listed("forward" if form == 0 else "backward", dtype, T, C, F, 0, 0)
for T, C, F, pad, shift in small:
    for dtype in ("f32", "bf16"):
        for call in ("matmul", "scaled", "forward"):
            tested |= listed(call, dtype, T, C, F, pad, shift)
rng = random.Random(5)
def size(high):
    n, kind = int(2 ** rng.uniform(0, high)), rng.random()
    return max(1, n if kind < 0.4 else n // 16 * 16 if kind < 0.7 else n // 128 * 128)
reached = set()
for _ in range(20000):
    T, C, F, dtype, pad = size(14), size(13.5), size(14), rng.randint(0, 1), int(rng.random() < 0.3)
    x, w = A + 4 * (rng.random() < 0.4), A + 4 * (rng.random() < 0.4)
    ld, ld_w = C + pad, C + pad * (rng.random() < 0.5)
    for rc in (matmul(T, C, F, dtype, (ld, 0, 0), x), scaled(T, C, F, dtype, 0, (ld, 0, 0, 0, 0, 0), x), forward(T, C, F, dtype, 0, (ld, 0, 0, 0, 0, 0), x),
               backward(T, C, F, dtype, rng.random() < 0.5, 0, (ld, ld_w, 0, 0, 0, 0), x, w, w)):
        reached |= launched(rc)
assert len(reached) > 90 and reached <= tested, sorted(reached - tested)
''')
