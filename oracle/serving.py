"""The operators around the prefill (include/mmi_cache.h) in plain numpy, fp64:
rotary positions, the codes of the paged cache and the attention of drafted
tokens over cached ones. Written from the definitions, one row at a time where
that is the definition."""
from __future__ import annotations

import math

import numpy as np

D, GROUP = 128, 32
TOP = {"fp8": 448.0, "int8": 127.0, "fp4": 6.0}
MOST = {"fp8": 1.875 * 2.0 ** 127, "int8": 127 * 2.0 ** 121, "fp4": 1.5 * 2.0 ** 127}     # what stays below 2^128


# ------------------------------------------------------------------ rotary positions
def frequencies(rot_dim, theta=10000.0, scaling="none", factor=1.0, orig_len=0.0, beta_fast=32.0, beta_slow=1.0):
    """Radians a position of the rot_dim / 2 pairs."""
    if scaling == "ntk":
        theta = theta * factor ** (rot_dim / (rot_dim - 2))
    out = []
    for i in range(rot_dim // 2):
        f = theta ** (-2.0 * i / rot_dim)
        if scaling == "linear":
            f /= factor
        if scaling == "parts":
            turns = orig_len * f / (2 * math.pi)
            keep = min(max((turns - beta_slow) / (beta_fast - beta_slow), 0.0), 1.0)
            f = f * keep + f / factor * (1 - keep)
        out.append(f)
    return np.array(out)


def pairs(rot_dim, layout):
    """Channels of the first and of the second entry of every pair."""
    i = np.arange(rot_dim // 2)
    return (i, i + rot_dim // 2) if layout == "half" else (2 * i, 2 * i + 1)


def rope(x, pos, freq, layout="half", m=1.0, inverse=False, sections=(0, 0, 0)):
    """x [S, H, 128] turned; pos [S], or [3, S] with sections."""
    pos = np.asarray(pos, np.float64).reshape(-1, x.shape[0])
    axis = np.repeat(np.arange(3), sections) if any(sections) else np.zeros(len(freq), int)
    y = np.array(x, np.float64)
    a, b = pairs(2 * len(freq), layout)
    for s in range(x.shape[0]):
        angle = pos[axis, s] * freq * (-1 if inverse else 1)
        c, n = m * np.cos(angle), m * np.sin(angle)
        y[s][:, a] = x[s][:, a] * c - x[s][:, b] * n
        y[s][:, b] = x[s][:, b] * c + x[s][:, a] * n
    return y


# ------------------------------------------------------------------ the cache
def grid(kind):
    """Every finite value of the type's codes, by code."""
    if kind == "int8":
        return np.array([c if c < 128 else c - 256 for c in range(256)], np.float64)
    bits, mant, bias = (8, 3, 7) if kind == "fp8" else (4, 1, 1)
    out = []
    for c in range(1 << bits):
        sign = -1.0 if c >> (bits - 1) else 1.0
        e, f = (c >> mant) & ((1 << (bits - 1 - mant)) - 1), c & ((1 << mant) - 1)
        v = f * 2.0 ** (1 - bias - mant) if e == 0 else (1 + f / (1 << mant)) * 2.0 ** (e - bias)
        if kind == "fp8" and c & 127 == 127:
            v = math.nan                           # E4M3's only non-finite codes
        out.append(sign * v)
    return np.array(out)


def exponent(amax, kind):
    """Smallest e >= -126 with amax <= M 2^e."""
    e = -126
    if amax > 0:
        e = max(e, math.frexp(amax)[1] - math.frexp(TOP[kind])[1] - 1)
        while amax > TOP[kind] * 2.0 ** e:
            e += 1
    return e


def quantise(row, kind):
    """(codes [128], scale bytes [4]) of one row."""
    g = grid(kind)
    usable = np.flatnonzero(np.isfinite(g) & (np.abs(g) <= TOP[kind]))
    codes, scales = np.zeros(D, np.int64), np.zeros(4, np.int64)
    for s in range(4):
        x = np.asarray(row[s * GROUP:(s + 1) * GROUP], np.float64)
        if not np.isfinite(x).all():
            scales[s] = 255
            continue
        x = np.clip(x, -MOST[kind], MOST[kind])
        e = exponent(np.abs(x).max(), kind)
        scales[s] = e + 127
        for i, v in enumerate(x / 2.0 ** e):
            far = np.abs(g[usable] - v)
            near = usable[far == far.min()]
            # a tie goes to the even code; among the two zeros the sign decides
            near = [c for c in near if c % 2 == 0] if len({abs(g[c]) for c in near}) > 1 else list(near)
            near = [c for c in near if (np.signbit(g[c]) or (kind != "int8" and c >> (7 if kind == "fp8" else 3)))
                    == np.signbit(v)] or near
            codes[s * GROUP + i] = near[0]
    return codes, scales


def value(codes, scales, kind):
    """What codes [..., 128] and scale bytes [..., 4] stand for."""
    g = grid(kind)
    s = np.where(np.asarray(scales) == 255, np.nan, np.exp2(np.asarray(scales, np.float64) - 127))
    return g[np.asarray(codes)] * np.repeat(s, GROUP, -1)


# ------------------------------------------------------------------ drafted tokens
def attend(q, k, v, sees, scale=D ** -0.5):
    """One row: q [128], k and v [n, 128], sees [n]. Returns (o, lse, spread, score bound): spread = the mean
    of |v - o| under the row's weights (what rounding the weights can move o by, per relative error), score
    bound = the largest sum of |q k| scale, per unit of relative error of the scores' products."""
    at = np.flatnonzero(sees)
    if len(at) == 0:
        return np.zeros(D), -np.inf, np.zeros(D), 0.0
    with np.errstate(all="ignore"):
        z = k[at] @ q * scale
        top = z.max()
        w = np.exp(z - top)
        total = w.sum()
        w = w / total
        o = w @ v[at]
        return o, top + np.log(total), w @ np.abs(v[at] - o), (np.abs(k[at]) @ np.abs(q)).max() * scale
