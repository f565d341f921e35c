"""fp64 NumPy oracle of the operators around attention: e4m3 linear layers, rotary positions, the quantised K/V cache.

Written from the definitions, elementwise and with loops where a loop is plainest; shares no code with the library or with the measured cases.
Inputs are float64 arrays (holding bf16 values); scales and quotients that the definitions call fp32 are rounded to fp32 and
kept in float64.
"""
import math

import numpy as np


def f32(x):
    return np.asarray(x, np.float64).astype(np.float32).astype(np.float64)


def _magnitudes(exponents, mantissa_bits, bias, top):
    """All non-negative finite numbers of a small format, in order of their codes."""
    out = []
    for e in range(exponents):
        for m in range(1 << mantissa_bits):
            v = math.ldexp(m, 1 - bias - mantissa_bits) if e == 0 else math.ldexp((1 << mantissa_bits) + m, e - bias - mantissa_bits)
            if v <= top:
                out.append(v)
    return np.array(out)


E4M3 = _magnitudes(16, 3, 7, 448.0)        # codes 0 .. 126
E2M1 = _magnitudes(4, 1, 1, 6.0)           # codes 0 .. 7


def encode(y, table):
    """Index of the nearest magnitude of `table` (ties to the even code, saturating)."""
    a = np.minimum(np.abs(y), table[-1])
    hi = np.clip(np.searchsorted(table, a), 1, len(table) - 1)
    lo = hi - 1
    down, up = a - table[lo], table[hi] - a
    pick_up = (up < down) | ((up == down) & (hi % 2 == 0))
    return np.where(pick_up, hi, lo)


def e4m3_bytes(y):
    return np.where(np.isnan(y), 127, encode(y, E4M3) + 128 * np.signbit(y)).astype(np.uint8)


def e4m3_values(b):
    b = np.asarray(b)
    return np.append(E4M3, np.nan)[b & 127] * np.where(b >= 128, -1.0, 1.0)


def amax_of_numbers(x, axis=None):
    """Largest magnitude, NaNs left out (0 of nothing)."""
    return np.where(np.isnan(x), 0.0, np.abs(x)).max(axis)


def scale8(amax):
    return np.where(amax == 0, 1.0, f32(amax / 448.0))


def quantize_rows(x):
    """x [M,K] -> (bytes [M,K], scale [ceil(K/128), M])."""
    M, K = x.shape
    G = -(-K // 128)
    codes, scale = np.zeros((M, K), np.uint8), np.zeros((G, M))
    for g in range(G):
        part = x[:, 128 * g:128 * g + 128]
        scale[g] = scale8(amax_of_numbers(part, 1))
        with np.errstate(invalid="ignore"):               # (infinity / infinity: a NaN)
            codes[:, 128 * g:128 * g + 128] = e4m3_bytes(f32(part / scale[g][:, None]))
    return codes, scale


def quantize_tiles(w):
    """w [N,K] -> (bytes [N,K], scale [ceil(N/128), ceil(K/128)])."""
    N, K = w.shape
    codes, scale = np.zeros((N, K), np.uint8), np.zeros((-(-N // 128), -(-K // 128)))
    for J in range(scale.shape[0]):
        for g in range(scale.shape[1]):
            at = np.s_[128 * J:128 * J + 128, 128 * g:128 * g + 128]
            scale[J, g] = scale8(amax_of_numbers(w[at]))
            with np.errstate(invalid="ignore"):
                codes[at] = e4m3_bytes(f32(w[at] / scale[J, g]))
    return codes, scale


def activation(y, act):
    if act == "none":
        return y
    with np.errstate(over="ignore"):                      # (far to the negative side: y / infinity)
        # 0.5 y (1 + tanh u) = y / (1 + exp(-2u)), without the cancellation of 1 + tanh
        x = 2.0 * math.sqrt(2.0 / math.pi) * (y + 0.044715 * y ** 3) if act == "gelu" else y
        return y / (1.0 + np.exp(-x))


def linear(x8, x_scale, w8, w_scale, bias=None, act="none", residual=None):
    """(out, sum of the magnitudes of the product's terms), from codes and scales."""
    M, K = x8.shape
    x = e4m3_values(x8) * np.repeat(x_scale, 128, 0)[:K].T
    w = e4m3_values(w8) * np.repeat(np.repeat(w_scale, 128, 0)[:w8.shape[0]], 128, 1)[:, :K]
    y = x @ w.T
    if bias is not None:
        y = y + bias
    y = activation(y, act)
    return (y if residual is None else y + residual), np.abs(x) @ np.abs(w).T


def frequencies(axis_pairs, base=10000.0, scaling="none", factor=1.0, trained_length=1.0, beta_fast=32.0, beta_slow=1.0):
    """Radians per position of every pair."""
    out = []
    for P in axis_pairs:
        for j in range(P):
            b = base * factor ** (P / (P - 1)) if scaling == "ntk" and P > 1 else base
            theta = b ** (-j / P)
            if scaling == "linear":
                theta /= factor
            if scaling == "parts":
                turns = trained_length * theta / (2 * math.pi)
                g = min(1.0, max(0.0, (turns - beta_slow) / (beta_fast - beta_slow)))
                theta *= (1 - g) / factor + g
            out.append(theta)
    return np.array(out)


def rope(x, theta, positions, axis_pairs, rotary_dim, layout, factor=1.0, inverse=False):
    """x [B,H,N,d], positions [axes][B or 1][N]."""
    out = x.copy()
    B, _, N, _ = x.shape
    pair = 0
    for axis, P in enumerate(axis_pairs):
        for _ in range(P):
            first, second = (pair, pair + rotary_dim // 2) if layout == "half" else (2 * pair, 2 * pair + 1)
            for b in range(B):
                p = positions[axis][b if len(positions[axis]) > 1 else 0].astype(np.float64)
                c, s = np.cos(p * theta[pair]) * factor, np.sin(p * theta[pair]) * factor
                if inverse:
                    s = -s
                a, z = x[b, :, :, first], x[b, :, :, second]
                out[b, :, :, first] = a * c - z * s
                out[b, :, :, second] = z * c + a * s
            pair += 1
    return out


def cache_row(x, form):
    """One row [d] -> (code bytes, scale, sf bytes or None, values in fp64 before their rounding to bf16).  4-bit codes have no NaN: a row that
    holds one gets the scale NaN, codes and sf 0."""
    with np.errstate(invalid="ignore"):
        if form == "e4m3":
            scale = float(scale8(amax_of_numbers(x)))
            codes = e4m3_bytes(f32(x / scale))
            return codes, scale, None, f32(e4m3_values(codes) * scale)
        amax = np.abs(x).max()                            # (NaN if there is one)
        scale = 1.0 if amax == 0 else float(f32(amax / 2688.0))
        codes, sf = np.zeros(x.size, np.int64), np.zeros(x.size // 16, np.uint8)
        values = np.zeros(x.size)
        for i in range(sf.size):
            at = np.s_[16 * i:16 * i + 16]
            sf[i] = e4m3_bytes(f32(f32(np.abs(x[at]).max() / 6.0) / scale))
            unit = float(f32(e4m3_values(sf[i]) * scale))
            if unit > 0:
                y = f32(x[at] / unit)
                codes[at] = encode(y, E2M1) + 8 * np.signbit(y)
            elif np.isnan(unit):                          # (NaN, or infinite scales)
                sf[i] = 0
            values[at] = f32(E2M1[codes[at] & 7] * np.where(codes[at] >= 8, -1.0, 1.0) * e4m3_values(sf[i]) * scale)
    return (codes[0::2] + 16 * codes[1::2]).astype(np.uint8), scale, sf, values
