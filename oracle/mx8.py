"""The quantised cache's number format and the rotary options, from their definitions.

Format: a row of 128 values is four blocks of 32; a block's exponent e is the smallest integer >= -100
with max|y| 2^-e <= 448 (maximum over its finite values), and a value is held as y 2^-e rounded to the
nearest e4m3 number, ties to the even fraction.  e4m3: (-1)^s 2^(x-7) (1 + f/8) for x = 1..15 except
x = 15, f = 7 (NaN), (-1)^s 2^-6 f/8 for x = 0.  The nearest number is searched in the list of all of them.

Rotation: pairs (x_2j, x_2j+1) or (x_j, x_j+rot/2) of the first rot dimensions; binary32 products and
sums emulated in float64 (oracle.rope).  Tables: angles, cos and sin in float64, rounded once.

Test infrastructure: nothing in the library imports this module.
"""
from __future__ import annotations

import math

import numpy as np

from .numerics import bf16_to_f64, f32_to_f64, round_f32

# the non-negative finite e4m3 numbers by code 0..126
E4M3 = np.array([(2.0 ** -6 * f / 8 if x == 0 else 2.0 ** (x - 7) * (1 + f / 8)) for x in range(16) for f in range(8)][:127])


def e4m3_code(z: np.ndarray) -> np.ndarray:
    """Code of the nearest e4m3 number (ties to even), |z| <= 448 or NaN (code 0x7f)."""
    z = np.asarray(z, np.float64)
    a = np.abs(np.where(np.isnan(z), 0.0, z))
    hi = np.minimum(np.searchsorted(E4M3, a, side="left"), 126)
    lo = np.maximum(hi - 1, 0)
    up, down = E4M3[hi] - a, a - E4M3[lo]
    code = np.where(up < down, hi, np.where(down < up, lo, np.where(hi % 2 == 0, hi, lo)))
    code = np.where(E4M3[hi] == a, hi, code).astype(np.uint8)
    code = code | (np.signbit(z).astype(np.uint8) << 7)
    return np.where(np.isnan(z), np.uint8(0x7F), code)


def e4m3_value(code: np.ndarray) -> np.ndarray:
    mag = code & 0x7F
    v = np.where(mag == 0x7F, np.nan, E4M3[np.minimum(mag, 126)])
    return np.where(code & 0x80, -v, v)


def exponent(top: float) -> int:
    """The smallest integer e >= -100 with top 2^-e <= 448."""
    e = -100
    if top > 0:
        e = max(e, math.frexp(top)[1] - 10)
        while math.ldexp(top, -e) > 448:
            e += 1
    return e


def quantise(y: np.ndarray):
    """(codes [..., 128], scale bytes [..., 4]) of float64 y [..., 128]."""
    b = np.asarray(y, np.float64).reshape(-1, 32)
    fin = np.isfinite(b)
    top = np.where(fin, np.abs(b), 0.0).max(axis=1)
    uniq, inv = np.unique(top, return_inverse=True)
    e = np.array([exponent(float(t)) for t in uniq])[inv]
    codes = e4m3_code(np.where(fin, np.ldexp(np.where(fin, b, 0.0), -e[:, None]), np.nan))
    return codes.reshape(y.shape), (e + 127).astype(np.uint8).reshape(y.shape[:-1] + (4,))


def values(codes: np.ndarray, scale: np.ndarray) -> np.ndarray:
    v = e4m3_value(codes).reshape(codes.shape[:-1] + (4, 32))
    return (v * np.ldexp(1.0, scale.astype(int) - 127)[..., None]).reshape(codes.shape)


def rotate(x_bits: np.ndarray, cos32: np.ndarray, sin32: np.ndarray, half: bool) -> np.ndarray:
    """Rotated bf16 x [..., N, H, 128] as binary32 values (in float64); tables [N, rot / 2]."""
    x = bf16_to_f64(x_bits)
    pairs = cos32.shape[1]
    c, s = (f32_to_f64(t)[:, None, :] for t in (cos32, sin32))
    j = np.arange(pairs)
    a, b = (j, j + pairs) if half else (2 * j, 2 * j + 1)
    y = x.copy()
    y[..., a] = round_f32(round_f32(x[..., a] * c) - round_f32(x[..., b] * s))
    y[..., b] = round_f32(round_f32(x[..., a] * s) + round_f32(x[..., b] * c))
    return y


def frequencies(dims, theta=10000.0, scaling="none", factor=1.0, trained=0.0, turns=(32.0, 1.0)):
    """float64 angle per position of every pair, frame axis scaled, then rows, then columns."""
    out = []
    for axis, d in enumerate(dims):
        for k in range(d // 2):
            th = theta * factor ** (d / (d - 2.0)) if axis == 0 and scaling == "base" and d > 2 else theta
            w = th ** (-2.0 * k / d)
            if axis == 0 and scaling == "linear":
                w /= factor
            if axis == 0 and scaling == "parts":
                n = trained * w / (2 * math.pi)
                g = min(1.0, max(0.0, (n - turns[1]) / (turns[0] - turns[1])))
                w *= g + (1 - g) / factor
            out.append(w)
    return np.array(out)


def tables(start, frames, gh, gw, dims, amplitude=1.0, **kw):
    """float64 (cos, sin) [N, pairs] times the amplitude."""
    w = frequencies(dims, **kw)
    n = np.arange(frames * gh * gw)
    pos = np.stack([start + n // (gh * gw), n // gw % gh, n % gw], 1).astype(np.float64)
    axis = np.repeat([0, 1, 2], [d // 2 for d in dims])
    ang = pos[:, axis] * w
    return amplitude * np.cos(ang), amplitude * np.sin(ang)


def attention(q: np.ndarray, k: np.ndarray, v: np.ndarray):
    """float64 q [N, 128], k, v [M, 128]: out, natural log-sum-exp and sum_m p_m |v_m|, weights 2^(q k)."""
    s = q @ k.T
    top = s.max(axis=1, keepdims=True)
    p = np.exp2(s - top)
    total = p.sum(axis=1, keepdims=True)
    return (p / total) @ v, ((top + np.log2(total)) * math.log(2.0))[:, 0], (p / total) @ np.abs(v)
