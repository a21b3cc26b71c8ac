"""Plain fp64 statement of the key/value stores (row formats, decode attention over own rows and a shared prefix), written from
the definitions in gkv.h with numpy and Python's exact fractions' arithmetic where rounding decides. Test infrastructure only.

Tolerances of the attention are derived here as well (`attend` returns them with the values), from the roundings the kernels
make: u = half a step of a type relative to a value (bf16 2^-8, fp16 2^-11, fp32 2^-24)."""
import math

import numpy as np

D = 128
SCALES = {"bf16": 0, "e4m3": 1, "int8": 1, "int4": 4}
U_BF16, U_F16, U_F32 = 2.0 ** -8, 2.0 ** -11, 2.0 ** -24


def bf16_value(bits):
    return (np.asarray(bits, np.uint32) << 16).view(np.float32).astype(np.float64)


def round_bf16(x):
    """fp64 -> nearest bf16 value (ties to even), normal range and subnormals."""
    x = np.asarray(x, np.float64)
    m, e = np.frexp(x)
    step = np.ldexp(1.0, np.maximum(e - 8, -133))
    return np.rint(x / step) * step


def scale_of(amax, fmt):
    if not np.isfinite(amax):
        return np.nan
    least = 2.0 ** -126
    if fmt == "e4m3":
        s = least
        if amax > 448 * least:
            e = math.floor(math.log2(amax)) - 10      # below the answer; exact comparisons from here
            while amax > 448 * math.ldexp(1.0, e):
                e += 1
            s = math.ldexp(1.0, e)
        return s
    return max(float(round_bf16(amax / (127 if fmt == "int8" else 7))), least)


def encode(x, fmt):
    """fp64 rows [..., 128] -> (codes as numbers [..., 128], scales [..., groups])."""
    x = np.asarray(x, np.float64)
    ng = SCALES[fmt]
    flat = x.reshape(-1, ng, D // ng)
    amax = np.abs(flat).max(-1)                       # NaN and infinity come through
    s = np.array([[scale_of(a, fmt) for a in row] for row in amax])
    with np.errstate(invalid="ignore"):
        y = flat / s[..., None]                       # 8 bits over 8 bits: fp64 keeps ties apart from the rest
        if fmt == "e4m3":
            step = np.exp2(np.floor(np.log2(np.maximum(np.abs(y), 2.0 ** -6))) - 3)
            c = np.rint(y / step) * step
        else:
            c = np.rint(y)
    c = np.where(np.isfinite(s)[..., None], c, 0.0)
    return c.reshape(x.shape), s.reshape(x.shape[:-1] + (ng,))


def values(codes, scales, fmt):
    if fmt == "bf16":
        return codes
    ng = SCALES[fmt]
    return (codes.reshape(codes.shape[:-1] + (ng, D // ng)) * scales[..., None]).reshape(codes.shape)


def pack(codes, fmt):
    """Codes as numbers -> the store's bytes."""
    if fmt == "int8":
        return codes.astype(np.int8).view(np.uint8)
    if fmt == "int4":
        u = (codes + 8).astype(np.uint8)
        out = np.zeros(codes.shape[:-1] + (64,), np.uint8)
        for e in range(D):
            g, q, i = e // 32, e % 32 // 4, e % 4
            word = 4 * q + g
            out[..., 2 * word + i // 2] |= u[..., e] << (4 * (i % 2))
        return out
    # e4m3: sign, exponent (bias 7), 3 bits
    a = np.abs(codes)
    m, e = np.frexp(a)
    normal = a >= 2.0 ** -6
    exp = np.where(normal, e - 1 + 7, 0)
    man = np.where(normal, np.rint((m * 2 - 1) * 8), np.rint(a * 2.0 ** 9))
    return (np.where(np.signbit(codes), 128, 0) + exp * 8 + man).astype(np.uint8)


def attend(q, k, v, kp=None, vp=None, weight_unit=U_F16, code_bound=None):
    """One (sequence, KV head): q [g][128], own k, v [n][128], prefix kp, vp [m][128]. Returns out, lse and their tolerances.

    The kernels' roundings, relative to a weight p_t: u of the type in which weights enter the product (prefix rows and bf16
    rows: bf16, others: fp16); the logit is off by dz = (128 + 12) u32 (sum |q_i k_i| scale) for the products' fp32 sums and
    scalings and by 8 u32 (max |z| log2 e + 130) for the subtraction of the reference and the added log2 of a scale, the
    exponential by 2^-21. A weight is off by twice that in the quotient (numerator and sum). Outputs are rounded to bf16.
    fp16 weights are lifted so that the largest is at least 2^6: below 2^-14 they are off by up to 2^-25, 2^-31 of the largest,
    times the largest value times the number of keys, in units of the largest weight."""
    n = len(k)
    K = k if kp is None else np.concatenate([k, kp])
    V = v if vp is None else np.concatenate([v, vp])
    g = q.shape[0]
    if len(K) == 0:
        return np.zeros((g, D)), np.full(g, -np.inf), np.zeros((g, D)), np.zeros(g)
    sc = 1 / math.sqrt(D)
    z = q @ K.T * sc
    mag = (np.abs(q) @ np.abs(K).T * sc).max(-1)
    top = z.max(-1, keepdims=True)
    e = np.exp(z - top)
    l = e.sum(-1, keepdims=True)
    p = e / l
    out, lse = p @ V, (top + np.log(l))[:, 0]
    dz = 140 * U_F32 * mag + 8 * U_F32 * (np.abs(z).max(-1) * 1.4427 + 130) + 2.0 ** -21
    unit = np.full(len(K), weight_unit)
    if kp is not None:
        unit[n:] = U_BF16
    a = np.abs(V)
    tol = (p * unit) @ a + (2 * dz[:, None] + 2.0 ** -15) * (p @ a) + U_BF16 * np.abs(out) * (1 + U_BF16)
    if n and weight_unit == U_F16:
        tol = tol + (n * 2.0 ** -31 * (p[:, :n] * np.abs(V[:n]).max(-1)).max(-1))[:, None]
    return out, lse, tol + 1e-30, dz + len(K) * U_F32 + 2.0 ** -20 * np.maximum(1, np.abs(lse))
