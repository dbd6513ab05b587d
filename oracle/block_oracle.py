"""fp64 oracle of the operators between the linear layers (test infrastructure): norm with the residual's
addition and dropout, its backward pass, counter-based dropout, rotary positions, and matrix products in
8-bit floating point with power-of-two block scales.  Plain numpy from the definitions; bf16 inputs arrive
widened."""
from __future__ import annotations

import numpy as np


# ------------------------------------------------------------------ Philox-4x32-10 and the mask
def philox(c, key):
    """One call on counters c [n, 4] and a key of two words (Salmon, Moraes, Dror, Shaw 2011)."""
    c = [np.asarray(c[:, i], dtype=np.uint64) for i in range(4)]
    k0, k1 = int(key[0]), int(key[1])
    low, sh = np.uint64(0xFFFFFFFF), np.uint64(32)
    for _ in range(10):
        p0, p1 = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(p1 >> sh) ^ c[1] ^ np.uint64(k0), p1 & low, (p0 >> sh) ^ c[3] ^ np.uint64(k1), p0 & low]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return np.stack(c, axis=1).astype(np.uint32)


def keep_mask(n, p, seed, offset):
    groups = (n + 7) // 8
    c = np.zeros((groups, 4), dtype=np.uint64)
    i = np.arange(groups, dtype=np.uint64)
    c[:, 0], c[:, 1] = i & np.uint64(0xFFFFFFFF), i >> np.uint64(32)
    c[:, 2], c[:, 3] = offset & 0xFFFFFFFF, offset >> 32
    w = philox(c, (seed & 0xFFFFFFFF, seed >> 32))
    bits = np.stack([w & 0xFFFF, w >> 16], axis=2).reshape(-1)[:n]
    return bits >= round(p * 65536)


def drop(x, dropout):
    """x over its flat index, under a mask (p, seed, offset) or None."""
    x = np.asarray(x, dtype=np.float64)
    if dropout is None or round(dropout[0] * 65536) == 0:
        return x
    p, seed, offset = dropout
    r = round(p * 65536)
    scale = 65536.0 / (65536 - r) if r < 65536 else 0.0
    return np.where(keep_mask(x.size, p, seed, offset).reshape(x.shape), x * scale, 0.0)


# ------------------------------------------------------------------ norm
def add_rmsnorm(x, gain, residual=None, eps=1e-5, dropout=None):
    """(h, y, rstd) of rows along the last axis."""
    h = drop(x, dropout)
    if residual is not None:
        h = h + np.asarray(residual, dtype=np.float64)
    rstd = 1.0 / np.sqrt(np.mean(h * h, axis=-1) + eps)
    return h, h * rstd[..., None] * np.asarray(gain, dtype=np.float64), rstd


def add_rmsnorm_backward(dy, h, rstd, gain, dh_residual=None, dropout=None):
    """dy, h [B, T, d]: (dh, dx, n [B], S [d])."""
    dy, h, gain = (np.asarray(v, dtype=np.float64) for v in (dy, h, gain))
    r = np.asarray(rstd, dtype=np.float64)[..., None]
    hat = h * r
    u = dy * gain
    dh = r * (u - hat * np.mean(u * hat, axis=-1, keepdims=True))
    if dh_residual is not None:
        dh = dh + np.asarray(dh_residual, dtype=np.float64)
    g = np.sum(dy * hat, axis=1)
    return dh, drop(dh, dropout), np.sum(g * g, axis=-1), np.sum(g, axis=0)


# ------------------------------------------------------------------ rotary positions
def rope_frequencies(rot_dim, base=10000.0, scaling="none", factor=1.0, context=0.0, low=1.0, high=32.0):
    """Radians a position for each of rot_dim / 2 pairs."""
    if scaling == "ntk" and rot_dim > 2:
        base = base * factor ** (rot_dim / (rot_dim - 2))
    w = np.array([base ** (-2.0 * j / rot_dim) for j in range(rot_dim // 2)])
    if scaling == "linear":
        w = w / factor
    if scaling == "by_parts":
        u = np.minimum(1.0, np.maximum(0.0, (w * context / (2 * np.pi) - low) / (high - low)))
        w = u * w + (1 - u) * w / factor
    return w


def rope(x, positions, w, magnitude=1.0, interleaved=False, inverse=False):
    """x [B, T, H, D], positions [B, T], w radians a position."""
    x = np.array(x, dtype=np.float64)
    n = len(w)
    angle = np.asarray(positions, dtype=np.float64)[..., None, None] * w * (-1.0 if inverse else 1.0)
    c, s = magnitude * np.cos(angle), magnitude * np.sin(angle)
    ia, ib = (np.arange(0, 2 * n, 2), np.arange(1, 2 * n, 2)) if interleaved else (np.arange(n), np.arange(n, 2 * n))
    a, b = x[..., ia].copy(), x[..., ib].copy()
    x[..., ia], x[..., ib] = a * c - b * s, a * s + b * c
    return x


# ------------------------------------------------------------------ 8 bits
def scale_exponent(amax):
    """The smallest whole e >= -127 with amax <= 448 2^e (0 for a block of zeros)."""
    amax = np.asarray(amax, dtype=np.float64)
    m, k = np.frexp(amax)                       # amax = m 2^k, m in [0.5, 1); 448 = 0.875 2^9
    e = np.maximum(k - 9 + (m > 0.875), -127)
    return np.where(amax > 0, e, 0)


def to_e4m3(v):
    """Nearest number of the format (3 bits of fraction, smallest normal 2^-6, largest 448), ties to even."""
    v = np.asarray(v, dtype=np.float64)
    _, k = np.frexp(np.abs(v))
    step = np.ldexp(1.0, np.maximum(k - 1, -6) - 3)
    return np.round(v / step) * step            # numpy rounds halves to even


def _blocks(x, r, c):
    R, K = x.shape
    p = np.zeros((-(-R // r) * r, -(-K // c) * c))
    p[:R, :K] = x
    return p.reshape(p.shape[0] // r, r, p.shape[1] // c, c)


def quantise(x, block_rows):
    """(e4m3 values [R, K], exponents [R / block_rows, K / 128]) of finite x."""
    x = np.asarray(x, dtype=np.float64)
    b = _blocks(x, block_rows, 128)
    e = scale_exponent(np.abs(b).max(axis=(1, 3)))
    q = to_e4m3(b * np.ldexp(1.0, -e)[:, None, :, None]).reshape(b.shape[0] * block_rows, -1)
    return q[: x.shape[0], : x.shape[1]], e


def widen(q, e, block_rows):
    """The values that 8-bit numbers and their exponents stand for."""
    s = np.ldexp(1.0, e)
    s = np.repeat(np.repeat(s, block_rows, axis=0), 128, axis=1)
    return np.asarray(q, dtype=np.float64) * s[: q.shape[0], : q.shape[1]]
