"""Feed-forward operators in 64 bits, and how far a computation in the library's precision may be from them (plain numpy; shares no code with
the kernels).

A bound counts the roundings: `sums` additions in fp32 are off by at most sums * 2^-23 of the sum of magnitudes (2^-24 each where an addition rounds to
nearest, twice that where it cuts off), a rounding to bf16 by at most 2^-8 of the value, and the rest is carried through by derivatives.
"""
import math

import numpy as np

E4M3_MAX = 448.0
HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
_erf = np.vectorize(math.erf, otypes=[float])


def e4m3_values():
    """The 256 numbers that 8 bits stand for (sign, four bits of exponent with bias 7, three of fraction; 0x7f and 0xff NaN)."""
    out = np.empty(256)
    for b in range(256):
        sign, e, f = -1.0 if b & 0x80 else 1.0, (b >> 3) & 15, b & 7
        out[b] = sign * (f * 2.0 ** -9 if e == 0 else (8 + f) * 2.0 ** (e - 10))
        if b & 0x7f == 0x7f:
            out[b] = math.nan
    return out


def e4m3_bits(x):
    """The nearest 8-bit float of each |x| <= 448, ties to the even one, as its byte; NaN for what is not finite."""
    x = np.asarray(x, dtype=np.float64)
    positive = e4m3_values()[:127]
    a = np.where(np.isfinite(x), np.abs(x), 0.0)
    hi = np.clip(np.searchsorted(positive, a), 1, 126)
    lo = hi - 1
    to_lo, to_hi = a - positive[lo], positive[hi] - a
    bits = np.where((to_lo < to_hi) | ((to_lo == to_hi) & (lo % 2 == 0)), lo, hi)
    return np.where(np.isfinite(x), bits | np.where(np.signbit(x), 0x80, 0), 0x7f).astype(np.uint8)


def quantize(x, block_rows):
    """(bytes, scales) of x[T, C]."""
    T, C = x.shape
    bits = np.zeros((T, C), np.uint8)
    scale = np.ones((-(-T // block_rows), -(-C // 128)))
    for i in range(scale.shape[0]):
        for b in range(scale.shape[1]):
            part = np.s_[i * block_rows:(i + 1) * block_rows, b * 128:(b + 1) * 128]
            finite = np.abs(x[part][np.isfinite(x[part])]).astype(np.float64)
            largest = finite.max() if finite.size else 0.0
            power = 0
            if largest > 0:
                power = -126
                while largest > E4M3_MAX * 2.0 ** power:
                    power += 1
            scale[i, b] = 2.0 ** power
            with np.errstate(invalid="ignore"):
                bits[part] = e4m3_bits(x[part].astype(np.float64) / scale[i, b])
    return bits, scale


def stands_for(bits, scale, block_rows):
    values = e4m3_values()[bits]
    s = np.repeat(np.repeat(scale.astype(np.float64), block_rows, 0)[:bits.shape[0]], 128, 1)[:, :bits.shape[1]]
    return values * s


def cut_off(x, w):
    """What the 8-bit matrix instructions may lose of x @ w.T.  They add eight neighbouring products (of the 16 contraction indices that
    a lane holds in a piece, so of aligned groups of eight) keeping bits down to 2^-13 of the largest one's power of two: each of the other seven loses less than 2^-13 of
    the largest product, and there is one such loss for every group, carried through sums in fp32."""
    x, w = (np.abs(np.pad(a, ((0, 0), (0, -a.shape[1] % 8)))) for a in (x, w))
    total = np.zeros((x.shape[0], w.shape[0]))
    for k in range(0, x.shape[1], 8):
        largest = np.zeros_like(total)
        for i in range(k, k + 8):
            np.maximum(largest, np.outer(x[:, i], w[:, i]), out=largest)
        total += largest
    return total * 7 * 2.0 ** -13


def matmul_scaled(x, w, half_step, cut=0.0):
    """(Out, bound) for the values x[T, C], w[K, C] that 8 bits and scales stand for; cut: cut_off's array where the result is bf16."""
    out, size = x @ w.T, np.abs(x) @ np.abs(w).T
    # products are exact; 128 additions in a block, one of the block, and the roundings of two scales' product and of its product
    sums = 128 + -(-x.shape[1] // 128) + 2
    off = size * sums * 2.0 ** -23 + cut
    return out, off + half_step * (np.abs(out) + off)


def activation(name, g):
    """(act, act', a bound on |act''|)"""
    if name == "silu":
        with np.errstate(over="ignore"):
            s = 1 / (1 + np.exp(-g))
        return g * s, s + g * s * (1 - s), 0.5
    if name == "gelu":
        p = 0.5 * (1 + _erf(g / math.sqrt(2)))
        return g * p, p + g * np.exp(-g * g / 2) / math.sqrt(2 * math.pi), 0.8
    k = math.sqrt(2 / math.pi)
    t = np.tanh(k * (g + 0.044715 * g ** 3))
    return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * k * (1 + 3 * 0.044715 * g * g), 0.9


_erfc = np.vectorize(math.erfc, otypes=[float])


def activation_steps(name, g):
    """(act, how far its 32-bit steps may be, act', how far its may be), relative to the numbers that they multiply and add, so that a gate far below
    zero, whose act is small, has to be right in its leading digits too.  Counted: 2^-24 for a rounding or a constant's, an ulp for a power of two or a
    reciprocal, 16 for the tail of the normal distribution, and what a relative error r of its argument y makes of e^y: |y| r."""
    ulp, tiny = 2.0 ** -23, 2.0 ** -120
    if name == "gelu":
        share = 0.5 * _erfc(-g / math.sqrt(2))
        # d ln erfc(z) / d ln z is at most 2 z^2 + 1 in magnitude, z = x / sqrt 2 of two roundings
        off = share * (16 + g * g + 2) * ulp
        rest, rest_off = g * np.exp(-g * g / 2) / math.sqrt(2 * math.pi), (0.75 * g * g + 4) * ulp
    else:
        # share = 1 / (1 + e^-y)
        k = math.sqrt(8 / math.pi)
        y = g if name == "silu" else k * g * (1 + 0.044715 * g * g)
        bend = np.ones_like(g) if name == "silu" else k * (1 + 0.134145 * g * g)
        share = np.where(y < 0, np.exp(-np.abs(y)), 1.0) / (1 + np.exp(-np.abs(y)))
        other = np.where(y > 0, np.exp(-np.abs(y)), 1.0) / (1 + np.exp(-np.abs(y)))
        # y is of two roundings (with the constant that turns e into 2) or of nine, and counts by 1 - share
        off = share * ((1 if name == "silu" else 5) * np.abs(y) * other + 4) * ulp
        rest = g * share * other * bend
        rest_off = np.abs(rest) * 5 * ulp + np.abs(g) * bend * (off * np.abs(other - share) + share * ulp)
        return g * share, np.abs(g) * off + ulp * np.abs(g * share) + tiny, share + rest, off + rest_off + ulp * np.abs(share + rest) + tiny
    return g * share, np.abs(g) * off + ulp * np.abs(g * share) + tiny, share + rest, off + np.abs(rest) * rest_off + ulp * np.abs(share + rest) + tiny


def _off(g):
    """How far the activation's 32-bit steps may be, of 1 + |g|: a power of two of an argument that grows with g, a reciprocal, a few products."""
    return 2.0 ** -20 * (1 + np.abs(g)) ** 2


def gated(x, wg, wu, name, half_step, sums=None, cut=(0.0, 0.0)):
    """dict of (value, bound) of gate, up and out; sums and cut: as in matmul_scaled where the operands are in 8 bits."""
    sums = x.shape[1] + 1 if sums is None else sums
    g, u = x @ wg.T, x @ wu.T
    dg, du = (np.abs(x) @ np.abs(w).T * sums * 2.0 ** -23 + c for w, c in zip((wg, wu), cut))
    a, slope, bend = activation(name, g)
    da = (np.abs(slope) + bend * dg) * dg + _off(g) * np.minimum(1.0, np.abs(g))
    h = a * u
    dh = da * (np.abs(u) + du) + np.abs(a) * du
    return {"gate": (g, dg + half_step * np.abs(g)), "up": (u, du + half_step * np.abs(u)), "out": (h, dh + half_step * (np.abs(h) + dh))}


def gated_backward(x, wg, wu, dy, name, half_step, gate=None, up=None):
    """dict of (value, bound) of the gradients of x, w_gate and w_up."""
    C = x.shape[1]
    if gate is None:
        g, u = x @ wg.T, x @ wu.T
        dg, du = (np.abs(x) @ np.abs(w).T * (C + 1) * 2.0 ** -23 for w in (wg, wu))
    else:
        g, u = gate, up
        dg = du = np.zeros_like(g)
    a, slope, bend = activation(name, g)
    # act'' is bounded by `bend`, and act''' by a little more: 2 bend covers the slope's own error
    dslope = 2 * bend * dg + _off(g)
    da = (np.abs(slope) + bend * dg) * dg + _off(g) * np.minimum(1.0, np.abs(g))
    gg, gu = dy * u * slope, dy * a
    egg = np.abs(dy) * ((np.abs(u) + du) * dslope + du * np.abs(slope))
    egu = np.abs(dy) * da
    # rounded to the arrays' type, as operands of the products
    egg, egu = egg + half_step * (np.abs(gg) + egg), egu + half_step * (np.abs(gu) + egu)

    def product(pairs):
        value = sum(p @ q for p, _, q in pairs)
        n = sum(p.shape[1] for p, _, _ in pairs) + 1
        bound = sum(e @ np.abs(q) + (np.abs(p) + e) @ np.abs(q) * n * 2.0 ** -23 for p, e, q in pairs)
        return value, bound + half_step * (np.abs(value) + bound)

    return {"grad_x": product([(gg, egg, wg), (gu, egu, wu)]), "grad_w_gate": product([(gg.T, egg.T, x)]),
            "grad_w_up": product([(gu.T, egu.T, x)])}
