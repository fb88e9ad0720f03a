"""Plain 64-bit forms of the 8-bit cache, of attention over it and of the
rotary positions, in numpy, from their definitions."""
import math

import numpy as np

BLK = 64
TOP = {"int8": 127.0, "e4m3": 448.0}


def bf16(x):
    """Rounded to bf16 (nearest, ties to even), as fp32."""
    u = np.ascontiguousarray(x, dtype=np.float32).view(np.uint32).astype(np.uint64)
    r = ((u + 0x7FFF + ((u >> 16) & 1)) >> 16 << 16).astype(np.uint32)
    return r.view(np.float32)


def round_e4m3(y):
    """64-bit values of magnitude at most 448 to the nearest e4m3 value, ties to even."""
    a = np.abs(y)
    step = 2.0 ** (np.floor(np.log2(np.maximum(a, 2.0 ** -6))) - 3)
    return np.sign(y) * np.rint(a / step) * step


def quantise(x, fmt):
    """A block [64, d] -> (code values, fp32 scale).  Q x / eff in 64 bits: both are
    bf16 values times small whole numbers, so a quotient that is a midpoint is
    formed exactly and no other one is near enough to one to be moved there."""
    Q = TOP[fmt]
    x = np.asarray(x, dtype=np.float64)
    eff = min(max(np.abs(x).max(), Q * 2.0 ** -60), Q * 2.0 ** 60)
    y = np.clip(Q * x / eff, -Q, Q)
    return (np.rint(y) if fmt == "int8" else round_e4m3(y)), np.float32(np.float32(eff) / np.float32(Q))


def open_scale(x):
    """The open block's scale entry for its rows [r, d]."""
    top = float(np.abs(x).max()) if x.size else 0.0
    e = math.floor(math.log2(top)) - 14 if top > 0 else -60
    return np.float32(2.0 ** max(e, -60))


def read_back(x, fmt):
    """Rows [n, d] (bf16 values) of one side of a unit as the cache holds them, in 64 bits."""
    x = np.asarray(x, dtype=np.float64)
    out = x.copy()
    for j in range(len(x) // BLK):
        c, s = quantise(x[j * BLK:(j + 1) * BLK], fmt)
        out[j * BLK:(j + 1) * BLK] = c * np.float64(s)
    return out


def attend(q, K, V, scale, end):
    """One query over the first `end` rows; zeros if there are none.  Also returns
    the sum over channels of |scale q K| at its largest, which bounds how far
    the logits may be off."""
    end = max(min(end, len(K)), 0)
    if end == 0:
        return np.zeros(K.shape[1]), 0.0
    q = np.asarray(q, dtype=np.float64)
    s = (K[:end] @ q) * scale
    p = np.exp(s - s.max())
    return (p / p.sum()) @ V[:end], float((np.abs(K[:end]) @ np.abs(q)).max()) * scale


def tolerance(end, d, reach, vmax, out_fp32):
    """How far an output may be off, from the roundings on its way.  A logit is a
    sum of d products of exact factors in fp32 (d additions, the products
    themselves exact or rounded once) times a factor of three roundings:
    (d + 4) 2^-23 of its absolute sum `reach` (2^-23, should the matrix cores
    truncate).  Weights: e^(2 of that) - 1, and 8 steps of 2^-23 for the exponential,
    its argument and the running maxima; the exponent's argument, at most 2 reach
    log2(e) + 128, is rounded to 2^-24 of itself.  Sums: additions within a block
    are 64 deep, across blocks end / 64.  All relative to the largest |V| (the
    output is an average of values).  With bf16 outputs weights are rounded to fp16
    (2^-11) and the output to bf16 (2^-8)."""
    u = 2.0 ** -23
    logit = (d + 4) * u * reach + (2 * reach * 1.45 + 128) * 2.0 ** -24
    rel = 2 * math.expm1(logit) + (8 + 64 + end / 64 + 16) * u
    if not out_fp32:
        rel += 2.0 ** -11 + 2.0 ** -8
    return rel * vmax + 1e-30


def rope(x, pos, rot, freq, axis, adjacent, inverse, scale):
    """x [n, d], pos [3, n] -> rotated, in 64 bits."""
    x = np.asarray(x, dtype=np.float64)
    out = x.copy()
    for i in range(rot // 2):
        a = pos[axis[i]].astype(np.float64) * freq[i]
        c, s = np.cos(a), np.sin(a) * (-1 if inverse else 1)
        p, q = (2 * i, 2 * i + 1) if adjacent else (i, i + rot // 2)
        out[:, p] = scale * (x[:, p] * c - x[:, q] * s)
        out[:, q] = scale * (x[:, q] * c + x[:, p] * s)
    return out


def rope_axes(rot, sections, interleaved):
    if not interleaved:
        return [0] * sections[0] + [1] * sections[1] + [2] * sections[2]
    return [1 if i % 3 == 1 and i < 3 * sections[1] else 2 if i % 3 == 2 and i < 3 * sections[2] else 0
            for i in range(rot // 2)]
