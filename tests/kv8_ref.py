"""Plain 64-bit forms of rotary positions and of the 8-bit cache (numpy)."""
import numpy as np
import torch

from tests.attn_ref import UNIT

DT = {"bf16": torch.bfloat16, "fp16": torch.float16}
TOP = {"bf16": 1.875 * 2.0 ** 127, "fp16": 1.875 * 2.0 ** 15}


def _codes():
    """Values of the 127 codes without sign that are numbers."""
    c = np.arange(127)
    e, m = c >> 3, c & 7
    return np.where(e > 0, (8 + m) * 2.0 ** (e - 10.0), m * 2.0 ** -9)


VALUES = _codes()


def turn(x, pos, freq, axis=None, interleaved=False, inverse=False):
    """x [n][heads][dim] turned; pos [axes][n]: outputs and a bound on |kernel - out|.

    The bound.  The kernel's angle is the same 64-bit product, its sine and cosine are off by a few
    2^-53 and the two products and their sum by 2^-52 of |a| + |b|: together below 2^-49 (|a| +
    |b|).  Then one rounding to fp32 (2^-24) and one to the element type (u), of which fp16 has an
    absolute step of 2^-24, half of it, below its normal range."""
    x = np.asarray(x, np.float64)
    half = len(freq)
    axis = np.zeros(half, int) if axis is None else np.asarray(axis)
    pos = np.atleast_2d(np.asarray(pos, np.float64))
    at = np.where((axis >= 0) & (axis < len(pos)), axis, len(pos))
    phi = np.concatenate([pos, np.zeros((1, pos.shape[1]))])[at].T * np.asarray(freq)  # [n][half]
    c, s = np.cos(phi)[:, None], np.sin(phi)[:, None] * (-1 if inverse else 1)
    ia = np.arange(half) * 2 if interleaved else np.arange(half)
    ib = ia + 1 if interleaved else ia + half
    a, b = x[..., ia], x[..., ib]
    y, wide = x.copy(), np.zeros_like(x)
    y[..., ia], y[..., ib] = a * c - b * s, b * c + a * s
    wide[..., ia] = wide[..., ib] = np.abs(a) + np.abs(b)
    return y, wide


def turn_bound(y, wide, kind):
    return np.where(wide > 0, (UNIT[kind] + 2.0 ** -23) * np.abs(y) + 2.0 ** -49 * wide
                    + (2.0 ** -25 if kind == "fp16" else 0.0), 0.0)


def quantise(x, kind):
    """Codes (bytes) and exponent bytes of rows [...][dim] of element-type values in 64 bits."""
    x = np.asarray(x, np.float64)
    fine = np.isfinite(x)
    a = np.where(fine, np.minimum(np.abs(x), TOP[kind]), 0.0)
    scales = 2.0 ** np.arange(-126, 128)
    e = np.searchsorted(scales * 448.0, a.max(-1))  # the first with max <= 448 scale
    y = a / scales[e][..., None]
    up = np.clip(np.searchsorted(VALUES, y), 1, 126)
    over = (y - VALUES[up - 1]) - (VALUES[up] - y)  # exact: few bits
    code = np.where((over > 0) | ((over == 0) & (up % 2 == 0)), up, up - 1)
    code = np.where(fine, code, 127) | np.where(np.signbit(x), 128, 0)
    return code.astype(np.uint8), (e + 1).astype(np.uint8)


def held(code, byte):
    """Values of codes [...][dim] with the exponent bytes of their rows."""
    code = np.asarray(code).astype(int)
    v = np.append(VALUES, np.nan)[code & 127] * 2.0 ** (np.asarray(byte).astype(int)[..., None] - 127.0)
    return np.where(code & 128, -v, v)


def rows_of_a_range(rng, n, dim, kind):
    """Rows that meet what a quantiser can get wrong: ordinary ones, wide ranges, largest elements next to and at
    448 times a power of two, ties between codes, zeros, the smallest and largest numbers."""
    x = rng.standard_normal((n, dim)) * 2.0 ** rng.integers(-100 if kind == "bf16" else -18, 100 if kind == "bf16" else 12,
                                                            (n, 1))
    wide = rng.random(n) < 0.3
    x[wide] *= 2.0 ** rng.integers(-14, 1, (wide.sum(), dim))
    for i in range(n):
        k = rng.integers(0, 9)
        p = 2.0 ** rng.integers(-10, 8)
        if k == 0:
            x[i] = 0.0 if rng.random() < 0.5 else -0.0
        elif k == 1:  # the border of the scale
            x[i] = np.clip(x[i] / np.abs(x[i]).max(), -1, 1) * p
            x[i, rng.integers(dim)] = (1.75 + rng.integers(-1, 2) * 2.0 ** -7) * p * (1 if rng.random() < 0.5 else -1)
        elif k == 2:  # halfway between codes, largest and subnormal ones among them
            step = rng.integers(0, 126, dim)
            x[i] = (VALUES[step] + VALUES[step + 1]) / 2 * p * np.where(rng.random(dim) < 0.5, 1, -1)
            x[i, 0] = 448 * p if p < 100 else 1.0
        elif k == 3:
            x[i] = 2.0 ** (-133 if kind == "bf16" else -24) * rng.integers(-200, 201, dim)
        elif k == 4:
            x[i, rng.integers(dim, size=2)] = torch.finfo(DT[kind]).max * np.array([1, -1.0])
    return torch.from_numpy(np.clip(x, -torch.finfo(DT[kind]).max, torch.finfo(DT[kind]).max)).to(DT[kind])
