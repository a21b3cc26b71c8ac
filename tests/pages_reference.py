"""Plain fp64 statements of the rotary positions and of rows in pages, with the tolerance of a rotation. Test infrastructure only."""
import math

import numpy as np

U_F32 = 2.0 ** -24
UNIT = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11, "fp32": 2.0 ** -24}
LEAST = {"bf16": 2.0 ** -134, "fp16": 2.0 ** -25, "fp32": 2.0 ** -150}     # half a step of the subnormals


def angles(turns, pos):
    """pos [...] of any size, turns: whole numbers of 2^-64 turns -> radians [..., pairs], exact but for fp64's rounding of the result."""
    with np.errstate(over="ignore"):
        phase = np.asarray(pos, np.int64)[..., None].astype(np.uint64) * np.asarray(turns, np.uint64)
    return phase.view(np.int64).astype(np.float64) * (2 * math.pi / 2.0 ** 64)


def rotate(x, angle, interleaved, factor=1.0, transpose=False):
    """x fp64 [..., heads, dims], angle [..., pairs] -> rotated, and the sum of magnitudes that rounding goes by."""
    half = angle.shape[-1]
    c, s = np.cos(angle)[..., None, :] * factor, np.sin(angle)[..., None, :] * factor
    if transpose:
        s = -s
    a, b = (x[..., 0:2 * half:2], x[..., 1:2 * half:2]) if interleaved else (x[..., :half], x[..., half:2 * half])
    y, mag = x.copy(), np.zeros_like(x)
    ya, yb, m = a * c - b * s, b * c + a * s, (np.abs(a) + np.abs(b)) * abs(factor)
    if interleaved:
        y[..., 0:2 * half:2], y[..., 1:2 * half:2] = ya, yb
        mag[..., 0:2 * half:2] = mag[..., 1:2 * half:2] = m
    else:
        y[..., :half], y[..., half:2 * half] = ya, yb
        mag[..., :half] = mag[..., half:2 * half] = m
    return y, mag


def rotation_tolerance(y, mag, dtype):
    """What the kernels may be off. In units of u = 2^-24, relative to (|a| + |b|) factor: the angle (at most pi/4, relative u: below 1, and
    the whole multiple of 2^-64 turns it stands for is the test's own) and cos and sin of it (a series with one rounding of a value below
    1 that matters: below 1), the factor's product 1, the product's rounding 1: 4 in all; u |y| for the last one; then the type's."""
    wide = 4 * U_F32 * mag + U_F32 * np.abs(y)
    fixed = np.where(mag > 0, wide * (1 + 2 * UNIT[dtype]), 0)
    return fixed + np.where(mag > 0, (0 if dtype == "fp32" else UNIT[dtype]) * np.abs(y) + LEAST[dtype], 0)


def pool_rows(table, page, rows):
    """(page, slot) of rows of one sequence."""
    rows = np.asarray(rows)
    return np.asarray(table)[rows // page], rows % page
