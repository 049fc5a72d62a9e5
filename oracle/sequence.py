"""The operators on the rows of a sequence batch in 64 bits, from their definitions (numpy; no code of the library).

Beside each result of the recurrence stands how far a computation in 32 bits may be off: every term of a result is a product
of factors that are each off by a few roundings, so the sum of the terms' magnitudes, each times its number of roundings,
bounds the error in whatever order the terms are combined."""
from __future__ import annotations

import numpy as np

U32 = 2.0 ** -24              # half a step of fp32, relative
BLOCK = 32


def pack8(x):
    """(codes int8 [n, D], exps uint8 [n, ceil(D/32)]) of finite or non-finite values, by the definition of the format."""
    x = np.asarray(x, np.float64)
    n, D = x.shape
    nb = -(-D // BLOCK)
    codes, exps = np.zeros((n, D), np.int8), np.zeros((n, nb), np.uint8)
    for b in range(nb):
        v = x[:, b * BLOCK:(b + 1) * BLOCK]
        bad = ~np.isfinite(v).all(1)
        top = np.where(bad, 1.0, np.abs(np.where(np.isfinite(v), v, 0)).max(1))
        E = np.full(n, 1)
        for e in range(2, 255):           # the smallest E with which the largest value rounds to at most 127 (ties to even: 127.5 does not)
            E = np.where(top >= 127.5 * 2.0 ** (e - 1 - 133), e, E)
        q = np.clip(np.round(np.where(bad[:, None], 0, v) / 2.0 ** (E[:, None] - 133.0)), -127, 127)
        kept = np.where(np.isnan(v), -128, np.where(np.isinf(v), np.sign(np.where(np.isnan(v), 0, v)) * 127, 0))
        codes[:, b * BLOCK:(b + 1) * BLOCK] = np.where(bad[:, None], kept, q).astype(np.int8)
        exps[:, b] = np.where(bad, 255, E)
    return codes, exps


def unpack8(codes, exps):
    """The values that codes and exponents stand for (float64)."""
    D = codes.shape[1]
    E = np.repeat(exps.astype(np.int64), BLOCK, axis=1)[:, :D]
    c = codes.astype(np.float64)
    kept = np.where(c == -128, np.nan, np.where(c == 0, 0.0, np.copysign(np.inf, c)))
    return np.where(E == 255, kept, c * 2.0 ** (np.clip(E, 1, 254) - 133.0))


def norm_fwd(x, gamma, beta, eps):
    x = np.asarray(x, np.float64)
    mean = x.mean(1)
    rstd = 1 / np.sqrt(((x - mean[:, None]) ** 2).mean(1) + eps)
    return (x - mean[:, None]) * rstd[:, None] * gamma + beta, mean, rstd


def norm_bwd(dy, x, mean, rstd, gamma):
    dy, x = np.asarray(dy, np.float64), np.asarray(x, np.float64)
    u = (x - np.asarray(mean, np.float64)[:, None]) * np.asarray(rstd, np.float64)[:, None]
    g = dy * gamma
    dx = np.asarray(rstd, np.float64)[:, None] * (g - g.mean(1, keepdims=True) - u * (g * u).mean(1, keepdims=True))
    return dx, (dy * u).sum(0), dy.sum(0)


def gates(gate):
    """f and 1 - f, and the share of each that 32 bits may miss: |gate| roundings' worth from the exponent's product, a few more
    from the exponential, the sum, the reciprocal and the product."""
    g = np.asarray(gate, np.float64)
    with np.errstate(over="ignore"):
        f, o = 1 / (1 + np.exp(-g)), 1 / (1 + np.exp(g))
    return f, o, (np.where(np.isfinite(g), np.abs(g), 0) + 16) * U32


def scan_fwd(x, gate, offsets, h0=None):
    """(h [n, D], h_last [S, D], bound of h, bound of h_last)"""
    x = np.asarray(x, np.float64)
    f, o, e = gates(gate)
    S, D = len(offsets) - 1, x.shape[1]
    h, off = np.zeros_like(x), np.zeros_like(x)
    last, last_off = np.zeros((S, D)), np.zeros((S, D))
    for s in range(S):
        v = np.zeros(D) if h0 is None else np.asarray(h0[s], np.float64).copy()
        size, err = np.abs(v), np.zeros(D)                     # the terms' magnitudes summed, and what they may be off
        for t in range(offsets[s], offsets[s + 1]):
            v = f[t] * v + o[t] * x[t]
            grown = f[t] * size + o[t] * np.abs(x[t])
            err = f[t] * err + grown * e[t]
            size = grown
            h[t], off[t] = v, err
        last[s], last_off[s] = v, err
    return h, last, off, last_off


def scan_bwd(dh, dh_last, x, gate, h, offsets, h0=None):
    """(dx, dgate, dh0, bound of dx, bound of dgate, bound of dh0)"""
    dh, x, h = (np.asarray(a, np.float64) for a in (dh, x, h))
    f, o, e = gates(gate)
    S, D = len(offsets) - 1, x.shape[1]
    dx, dg, dx_off, dg_off = (np.zeros_like(x) for _ in range(4))
    first, first_off = np.zeros((S, D)), np.zeros((S, D))
    for s in range(S):
        back = np.zeros(D) if dh_last is None else np.asarray(dh_last[s], np.float64).copy()
        size, err = np.abs(back), np.zeros(D)
        for t in range(offsets[s + 1] - 1, offsets[s] - 1, -1):
            before = h[t - 1] if t > offsets[s] else (np.zeros(D) if h0 is None else np.asarray(h0[s], np.float64))
            G = dh[t] + back
            size = size + np.abs(dh[t])
            err = err + size * 2 * U32
            dx[t], dg[t] = o[t] * G, G * (before - x[t]) * f[t] * o[t]
            dx_off[t] = o[t] * (err + size * e[t])
            dg_off[t] = f[t] * o[t] * np.abs(before - x[t]) * (err + size * 2 * e[t])
            back, err, size = f[t] * G, f[t] * (err + size * e[t]), f[t] * size
        first[s], first_off[s] = back, err
    return dx, dg, first, dx_off, dg_off, first_off
