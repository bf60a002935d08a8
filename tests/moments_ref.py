"""The AdamW step with 8-bit moments in numpy (no test functions here): every
product, sum and root of the moments in IEEE fp32, so codes and scale bytes are
the kernels' bit for bit; the parameter in 64 bits.

A value is multiplied by INVERSE[byte], 2^-k, before it is rounded. On the device
these are the math library's powers, some half a unit in the last place low:
the GPU tests put them here (device_powers), after they are checked to be within
that of the powers themselves."""
from __future__ import annotations

import numpy as np

BLOCK = 32
U32 = 2.0 ** -24
M64 = (1 << 64) - 1

# The 256 e4m3 numbers by their bits: sign, 4 exponent bits of bias 7, 3 fraction
# bits; exponent 0 holds the subnormals, all ones the only NaN.
_b = np.arange(256)
_e, _f = (_b >> 3) & 15, _b & 7
E4M3 = np.where(_e == 0, _f / 8.0 * 2.0 ** -6, (1 + _f / 8.0) * 2.0 ** (_e - 7.0))
E4M3[(_b & 0x7F) == 0x7F] = np.nan
E4M3 = np.where(_b & 0x80, -E4M3, E4M3)


INVERSE = np.exp2(127.0 - np.arange(256)).astype(np.float32)


def device_powers(torch):
    """INVERSE as torch.ldexp has it on the device: within half a unit in the last
    place of 2^-k, never above it."""
    k = 127 - torch.arange(255, dtype=torch.int32, device="cuda")
    got = torch.ldexp(torch.ones(255, device="cuda"), k).cpu().numpy()
    want = np.exp2(127.0 - np.arange(255))
    assert (got <= want).all() and (got >= want * (1 - 2.0 ** -24)).all()
    INVERSE[:255] = got


def words(number, seed):
    """The random words of value numbers (uint64 array)."""
    z = (seed * 0x9E3779B97F4A7C15 + 0x632BE59BD9B4E019) & M64
    z = ((z ^ (z >> 29)) * 0xD6E8FEB86659FD93) & M64
    z ^= z >> 32
    k0, k1 = np.uint32(z & 0xFFFFFFFF), np.uint32(z >> 32)
    number = np.asarray(number, np.uint64)
    lo, hi = (number & np.uint64(0xFFFFFFFF)).astype(np.uint32), (number >> np.uint64(32)).astype(np.uint32)
    with np.errstate(over="ignore"):
        h = (lo ^ k0) * np.uint32(0x9E3779B1)
        h ^= h >> np.uint32(15)
        h = (h + k1 + hi * np.uint32(0x85EBCA77)) * np.uint32(0xC2B2AE3D)
    return h ^ (h >> np.uint32(16))


def blocks(n):
    return -(-n // BLOCK)


def scale_of(byte, n):
    """2^k of each of n values (last axis), from their blocks' scale bytes."""
    return np.repeat(np.exp2(byte.astype(np.float64) - 127), BLOCK, -1)[..., :n]


def decode(codes, byte):
    return E4M3[codes] * scale_of(byte, codes.shape[-1])


def encode(x, part, keep):
    """(codes, scale bytes) of fp32 x [.., n]; part: R / 2^20 of each value."""
    n = x.shape[-1]
    a = np.abs(x).astype(np.float64)
    pad = np.zeros(x.shape[:-1] + (blocks(n) * BLOCK,))
    pad[..., :n] = a
    top = pad.reshape(x.shape[:-1] + (-1, BLOCK)).max(-1)
    f, e = np.frexp(top)  # top = f 2^e, f in [1/2, 1): at most 448 2^k = 7/8 2^(k + 9)
    k = np.where(top == 0, -127, np.maximum(e - 9 + (f > 0.875), -127))
    byte = (k + 127).astype(np.uint8)
    with np.errstate(under="ignore"):
        y = np.abs(x) * np.repeat(INVERSE[byte], BLOCK, -1)[..., :n]
    y = y.astype(np.float64)
    exp = np.maximum(np.frexp(y)[1] - 1, -6)
    step = np.exp2(exp - 3.0)
    q = np.floor(y / step + part) * step
    if keep:
        q = np.where((q == 0) & (a > 0), 2.0 ** -9, q)
    at = np.searchsorted(E4M3[:0x7F], q)
    assert np.array_equal(E4M3[at], q), "not an e4m3 number"
    return (at + 0x80 * np.signbit(x)).astype(np.uint8), byte


def step8(p, g, m, v, ms, vs, hyper, number, seed):
    """One step on values [.., n]: fp32 p and g (scaled), code and scale bytes.
    Returns p in 64 bits, its bound, and the new codes and scales; `left` where
    the new second moment is not finite."""
    lr, b1, b2, eps, wd, step = hyper
    f = np.float32
    lr, b1, b2, eps, wd = f(lr), f(b1), f(b2), f(eps), f(wd)
    c1, c2 = f(1) - b1, f(1) - b2
    m0, r0 = decode(m, ms).astype(f), decode(v, vs).astype(f)
    with np.errstate(over="ignore", invalid="ignore"):
        m1 = m0 * b1 + g * c1
        v1 = (r0 * r0) * b2 + (g * c2) * g
    left = ~np.isfinite(v1)
    v1 = np.where(left, f(0), v1)
    m1, r1 = np.where(left, m0, m1), np.where(left, r0, np.sqrt(v1))
    p1, bound = parameter(p, np.where(left, f(0), g), m0, v1, m1, hyper)
    p1, bound = np.where(left, p, p1), np.where(left, 0.0, bound)
    w = words(number, seed)
    m8, ms8 = encode(m1, (w >> np.uint32(12)) / 2.0 ** 20, False)
    v8, vs8 = encode(r1, (w & np.uint32(0xFFFFF)) / 2.0 ** 20, True)
    return p1, bound, m8, v8, ms8, vs8, left


def parameter(p, g, m0, v1, m1, hyper):
    """The new parameter in 64 bits from the new moments, and how far fp32 may be
    off: one half step of the result; the update's own roundings (the moments'
    three each, the corrections', the root's, the sum's, the quotient's and the
    decay's: under 16 half steps) relative to its parts before they cancel."""
    lr, b1, b2, eps, wd = (float(np.float32(x)) for x in hyper[:5])
    step = hyper[5]
    p, g, m0, v1, m1 = (np.asarray(x, np.float64) for x in (p, g, m0, v1, m1))
    i1, i2 = 1 / (1 - b1 ** step), 1 / (1 - b2 ** step)
    den = np.sqrt(v1 * i2) + eps
    new = p - lr * (m1 * i1 / den + wd * p)
    parts = (b1 * np.abs(m0) + (1 - b1) * np.abs(g)) * i1 / den + np.abs(wd * p)
    return new, 1.01 * U32 * (np.abs(new) + np.abs(p) + 16 * lr * parts) + 1e-45
