"""Rotary positions in extended precision, rounded to bf16 once."""
import numpy as np

EXT = np.longdouble


def values(bits):
    """bf16 bit patterns -> fp64"""
    return (bits.astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def to_bits(x):
    """fp64 values that are bf16 -> bit patterns"""
    return (x.astype(np.float32).view(np.uint32) >> 16).astype(np.uint16)


def turn(x, positions, freq, magnitude=1.0, interleaved=False, back=False):
    """[T, heads, d] -> the same, and what an error of the arithmetic is measured by (|x_a| + |x_b|) m, in extended precision."""
    t = (positions.astype(np.float64)[:, None] * freq).astype(EXT)  # (the fp64 product is the definition's angle)
    c, s = np.cos(t)[:, None] * EXT(magnitude), np.sin(t)[:, None] * EXT(magnitude)
    if back:
        s = -s
    n = freq.size
    y, size = x.astype(EXT), np.zeros(x.shape, EXT)
    a, b = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n))
    xa, xb = x[..., a].astype(EXT), x[..., b].astype(EXT)
    y[..., a], y[..., b] = xa * c - xb * s, xa * s + xb * c
    size[..., a] = size[..., b] = (abs(xa) + abs(xb)) * abs(EXT(magnitude))
    return y, size


def nearest(y):
    """Extended precision -> the nearest bf16 as fp64, ties to even, and the distance to the nearest border between two of them."""
    m, e = np.frexp(y)
    e = np.maximum(e, -125)  # (below 2^-126 the steps stay)
    scaled = np.ldexp(y, 8 - e)
    r = np.rint(scaled)
    return np.ldexp(r, e - 8).astype(np.float64), np.ldexp(abs(abs(scaled - r) - EXT(0.5)), e - 8)


def check(got_bits, y, size, what=""):
    """Bit for bit, but where the value is so near a border that fp64 cannot tell (three roundings of 2^-53 of the products each,
    and two of the angle's functions: below 2^-50 of |x_a| + |x_b|)."""
    want, room = nearest(y)
    got = values(got_bits)
    differ = got != want
    assert not np.any(differ & (room > size * EXT(2.0) ** -50)), f"{what}: {int(differ.sum())} of {got.size} values differ"
    return want


def codes(keys, W):
    """[T, Hkv, d] fp64 (of bf16), [Hkv, d, r] -> [T, Hkv, r / 32]"""
    bits = np.einsum("thd,hdr->thr", keys, W.astype(np.float64)) >= 0
    return np.packbits(bits, axis=2, bitorder="little").view(np.uint32)
