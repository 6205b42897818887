"""CPU oracle for the operators around attention in a transformer over the rows of a sparse tensor: rotary positions of several
axes, root-mean-square norm, rows in 8 bits with a power of two for each 128 elements, and the gated feed-forward block.

TEST INFRASTRUCTURE ONLY, like the rest of `oracle/`: plain numpy in float64, each function is the definition written out.
Pinned against torch's autograd and against differences in tests/test_block_oracle.py.
"""
from __future__ import annotations

import math

import numpy as np


# ---- rotary positions ------------------------------------------------------------------------------------------
def rope(x, pos, parts, base=10000.0, split=False, scale=1.0, back=False):
    """x [n][heads][dim], pos [n][axes]; every pair by itself."""
    x = np.asarray(x, np.float64)
    y, at = x.copy(), 0
    for a, part in enumerate(parts):
        for i in range(part // 2):
            angle = pos[:, a].astype(np.float64) * (scale * base ** (-2 * i / part)) * (-1 if back else 1)
            j, k = (at + i, at + i + part // 2) if split else (at + 2 * i, at + 2 * i + 1)
            c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
            y[:, :, j], y[:, :, k] = x[:, :, j] * c - x[:, :, k] * s, x[:, :, j] * s + x[:, :, k] * c
        at += part
    return y


# ---- root-mean-square norm -------------------------------------------------------------------------------------
def rms_fwd(h, gamma, eps):
    """Returns (y, rstd)."""
    h = np.asarray(h, np.float64)
    rstd = 1 / np.sqrt((h * h).mean(axis=1) + eps)
    return h * rstd[:, None] * gamma, rstd


def rms_bwd(h, dy, gamma, rstd, dh=None):
    """Returns (dx, dgamma)."""
    hat = np.asarray(h, np.float64) * np.asarray(rstd, np.float64)[:, None]
    g = np.asarray(dy, np.float64) * gamma
    dx = np.asarray(rstd, np.float64)[:, None] * (g - hat * (g * hat).mean(axis=1)[:, None])
    return dx if dh is None else dx + dh, (dy * hat).sum(axis=0)


# ---- rows in 8 bits --------------------------------------------------------------------------------------------
def e4m3(code):
    """The values of codes: sign, 4 bits of exponent (bias 7), 3 of mantissa; 0x7f and 0xff are NaN."""
    code = np.asarray(code, np.uint8).astype(np.int64)
    e, m = (code >> 3) & 15, code & 7
    size = np.where(e > 0, (8 + m) * 2.0 ** (np.maximum(e, 1) - 10), m * 2.0 ** -9)
    return np.where((code & 127) == 127, np.nan, np.where(code >> 7, -size, size))


_SIZES = e4m3(np.arange(127, dtype=np.uint8))


def e4m3_codes(v):
    """The nearest code of every value of at most 448, to the even one between two."""
    size = np.abs(v)
    hi = np.searchsorted(_SIZES, size).clip(0, 126)
    lo = np.maximum(hi - 1, 0)
    up, down = _SIZES[hi] - size, size - _SIZES[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    return (code + 128 * np.signbit(v)).astype(np.uint8)


def q8_rows(x):
    """Returns (codes [n][128 * blocks], scales [n][blocks rounded up to 4]) as bytes."""
    x = np.asarray(x, np.float64)
    n, c = x.shape
    blocks = -(-c // 128)
    codes, scales = np.zeros((n, blocks * 128), np.uint8), np.full((n, -(-blocks // 4) * 4), 127, np.uint8)
    for b in range(blocks):
        v = x[:, 128 * b:128 * b + 128]
        for r in range(n):
            top = np.abs(v[r]).max()
            if not np.isfinite(top):
                scales[r, b] = 255
                continue
            if top == 0:
                codes[r, 128 * b:128 * b + v.shape[1]] = 128 * np.signbit(v[r])
                continue
            e = math.frexp(top / 448)[1]                      # top / 448 = m * 2^e, 0.5 <= m < 1 (rounding is mended below)
            while top <= 448 * 2.0 ** (e - 1):
                e -= 1
            while top > 448 * 2.0 ** e:
                e += 1
            e = max(-127, e)
            scales[r, b] = e + 127
            codes[r, 128 * b:128 * b + v.shape[1]] = e4m3_codes(v[r] / 2.0 ** e)
    return codes, scales


def q8_values(codes, scales):
    """What codes and scales stand for, [n][128 * blocks]."""
    n, wide = codes.shape
    e = scales[:, :wide // 128].astype(np.int64)
    times = np.where(e == 255, np.nan, 2.0 ** (np.minimum(e, 254) - 127))
    return (e4m3(codes).reshape(n, wide // 128, 128) * times[:, :, None]).reshape(n, wide)


# ---- gated feed-forward block ----------------------------------------------------------------------------------
_erf = np.vectorize(math.erf)


def gate(g, act):
    """act(g) and its derivative."""
    if act == "silu":
        p = 1 / (1 + np.exp(-g))
        return g * p, p * (1 + g * (1 - p))
    p = 0.5 * (1 + _erf(g / math.sqrt(2)))
    return g * p, p + g * np.exp(-g * g / 2) / math.sqrt(2 * math.pi)


def ffn_fwd(x, w_in, w_out, act):
    """Returns (y, g, u, h)."""
    gu = x @ w_in.T
    m = w_out.shape[1]
    g, u = gu[:, :m], gu[:, m:]
    h = gate(g, act)[0] * u
    return h @ w_out.T, g, u, h


def ffn_bwd(x, w_in, w_out, g, u, h, dy, act):
    """Returns (dx, dw_in, dw_out, [dg du])."""
    a, da = gate(g, act)
    dh = dy @ w_out
    dgu = np.concatenate([dh * u * da, dh * a], axis=1)
    return dgu @ w_in, dgu.T @ x, dy.T @ h, dgu
