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
