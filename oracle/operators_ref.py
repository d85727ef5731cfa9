"""Float64 NumPy definitions of the operators beside the projected step: AdamW
with fp32 or 8-bit moments, the gradient norm, MXFP4 quantisation and packed
operands.  Test infrastructure only."""

from __future__ import annotations

import numpy as np

BLOCK = 256
E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


# ---------------------------------------------------------------- AdamW
def adamw(p, g, m, v, t, lr, beta1, beta2, eps, wd):
    """(p, m, v) after one step; all float64."""
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    with np.errstate(invalid="ignore", divide="ignore"):
        upd = (m / (1 - beta1 ** t)) / (np.sqrt(v / (1 - beta2 ** t)) + eps)
    return p * (1 - lr * wd) - lr * upd, m, v


def mix32(x):
    x = np.asarray(x, dtype=np.uint32).copy()
    with np.errstate(over="ignore"):
        x ^= x >> np.uint32(16)
        x *= np.uint32(0x85EBCA6B)
        x ^= x >> np.uint32(13)
        x *= np.uint32(0xC2B2AE35)
        x ^= x >> np.uint32(16)
    return x


def random_bits(n, seed, ident, t, first=0):
    """32 bits of each of n entries from `first` on (below 2^32 entries)."""
    k = mix32(mix32(seed & 0xFFFFFFFF) ^ np.uint32(seed >> 32))
    k = mix32(mix32(k ^ np.uint32(ident)) ^ np.uint32(t & 0xFFFFFFFF))
    i = np.arange(first, first + n, dtype=np.uint64)
    return mix32((i & np.uint64(0xFFFFFFFF)).astype(np.uint32) ^ mix32(k ^ (i >> np.uint64(32)).astype(np.uint32)))


def decode8(codes, scales, signed):
    """Values of 8-bit moments: 3 mantissa bits, largest exponent 0."""
    codes = np.asarray(codes).astype(np.int64)
    mag = codes & 127 if signed else codes
    emin = -14 if signed else -30
    e = mag >> 3
    y = np.where(e == 0, (mag & 7) * 2.0 ** (emin - 3), (8 + (mag & 7)) * 2.0 ** (np.maximum(e, 1) - 1 + emin - 3))
    if signed:
        y = np.where(codes & 128, -y, y)
    return y * np.repeat(np.asarray(scales, dtype=np.float64), BLOCK)[:len(codes)]


def code_position(x, signed):
    """Real-valued position of |x| on the code axis of its block, and the scales."""
    n = len(x)
    full = np.zeros(-(-n // BLOCK) * BLOCK)
    full[:n] = np.abs(x)
    top = full.reshape(-1, BLOCK).max(axis=1)
    scale = np.where(top < 2.0 ** -100, 0.0, top / 1.875)
    with np.errstate(invalid="ignore", divide="ignore"):
        y = np.where(np.repeat(scale, BLOCK)[:n] > 0, np.abs(x) / np.repeat(scale, BLOCK)[:n], 0.0)
    emin = -14 if signed else -30
    with np.errstate(divide="ignore"):
        e = np.maximum(np.floor(np.log2(np.maximum(y, 1e-300))), emin)
    return (e - emin) * 8 + y * 2.0 ** (3 - e), scale


# ---------------------------------------------------------------- MXFP4
def quantize(x):
    """(codes with the sign in bit 3, scale bytes) of x by rows in blocks of 32."""
    x = np.asarray(x, dtype=np.float64)
    m, k = x.shape
    kb = -(-k // 32)
    full = np.zeros((m, kb * 32))
    full[:, :k] = x
    b = full.reshape(m, kb, 32)
    top = np.abs(b).max(axis=2)
    bad = ~np.isfinite(b).all(axis=2)
    e = np.full(top.shape, -127.0)
    fine = ~bad & (top > 0)
    e[fine] = np.maximum(np.ceil(np.log2(top[fine] / 6)), -127)
    # log2 is rounded: settle at the smallest power that holds the block
    for _ in range(2):
        e = np.where(fine & (top > 6 * 2.0 ** e), e + 1, e)
        e = np.where(fine & (e > -127) & (top <= 6 * 2.0 ** (e - 1)), e - 1, e)
    with np.errstate(invalid="ignore"):
        a = np.abs(b) / 2.0 ** e[:, :, None]
    mid = (E2M1[1:] + E2M1[:-1]) / 2
    code = np.searchsorted(mid, a)                  # mid[i-1] < a <= mid[i]
    tie = (code < 7) & (a == mid[np.minimum(code, 6)])
    code = np.where(tie & (code % 2 == 1), code + 1, code)
    code = code | (np.signbit(b).astype(np.int64) << 3)
    return code.reshape(m, kb * 32), np.where(bad, 255, e + 127).astype(np.int64)


def values(code, scale, cols):
    m = code.shape[0]
    v = E2M1[code & 7] * np.where(code & 8, -1.0, 1.0)
    s = np.where(scale == 255, np.nan, 2.0 ** (scale - 127.0))
    return (v.reshape(m, -1, 32) * s[:, :, None]).reshape(m, -1)[:, :cols]


def pack(code, scale):
    """The bytes q and sf of an operand."""
    q = (code[:, 0::2] | code[:, 1::2] << 4).astype(np.uint8)
    m, kb = scale.shape
    ct = -(-kb // 4)
    sf = np.full(-(-m // 128) * ct * 512, 127, dtype=np.uint8)
    i, b = np.meshgrid(np.arange(m), np.arange(kb), indexing="ij")
    sf[(i // 128 * ct + b // 4) * 512 + i % 32 * 16 + i % 128 // 32 * 4 + b % 4] = scale
    return q.reshape(-1), sf


def operand(x):
    """(q, sf, values) of a matrix."""
    x = np.asarray(x, dtype=np.float64)
    code, scale = quantize(x)
    return pack(code, scale) + (values(code, scale, x.shape[1]),)
