"""Operators around the residual stream in plain numpy float64: lookup and its gradient, rows in 8 bits, layer norm of such rows.

TEST INFRASTRUCTURE: textbook definitions, token by token and group by group.
"""
from __future__ import annotations

import numpy as np

F64 = np.float64
GROUP = 32
TOP = {"int8": 127.0, "e4m3": 448.0}


def embed_lookup(ids, table, scale=1.0, positions=None, pos_table=None):
    """x[t] = scale table[ids[t]] + pos_table[positions[t]]; a term whose index names no row is left out."""
    x = np.zeros((len(ids), table.shape[1]), F64)
    for t, v in enumerate(ids):
        if 0 <= v < len(table):
            x[t] = scale * table[v].astype(F64)
        if pos_table is not None:
            p = t % len(pos_table) if positions is None else positions[t]
            if 0 <= p < len(pos_table):
                x[t] += pos_table[p].astype(F64)
    return x


def embed_grad(ids, dx, V, scale=1.0):
    """(gradient [V, d], sums of magnitudes [V, d], how many tokens name each row [V])."""
    g, a, n = np.zeros((V, dx.shape[1]), F64), np.zeros((V, dx.shape[1]), F64), np.zeros(V, np.int64)
    for t, v in enumerate(ids):
        if 0 <= v < V:
            g[v] += scale * dx[t].astype(F64)
            a[v] += abs(scale) * np.abs(dx[t].astype(F64))
            n[v] += 1
    return g, a, n


def numbers(code):
    """What each of the 256 codes of a format stands for."""
    b = np.arange(256)
    if code == "int8":
        return np.where(b < 128, b, b - 256).astype(F64)
    sign, power, part = np.where(b < 128, 1.0, -1.0), b >> 3 & 15, (b & 7) / 8.0
    v = sign * np.where(power == 0, part * 2.0 ** -6, (1 + part) * 2.0 ** (power - 7.0))
    v[(b & 127) == 127] = np.nan
    return v


def _nearest(q, code):
    """Codes of the format's numbers nearest to q, of two the one whose last bit is 0; zeros keep their sign where the format has one."""
    if code == "int8":
        return np.rint(q).astype(np.int64).astype(np.uint8)
    table = numbers(code)[:127]                      # ascending from 0 to 448
    a = np.abs(q)
    hi = np.minimum(np.searchsorted(table, a), 126)
    lo = np.maximum(hi - 1, 0)
    up, down = table[hi] - a, a - table[lo]
    pick = np.where((down < up) | ((down == up) & (lo % 2 == 0)), lo, hi)
    return (pick + np.where(np.signbit(q), 128, 0)).astype(np.uint8)


def pack8(x, code):
    """codes [T, d] and scales [T, groups], as bytes."""
    x = np.asarray(x, F64)
    T, d = x.shape
    G = -(-d // GROUP)
    codes, scales = np.zeros((T, d), np.uint8), np.zeros((T, G), np.uint8)
    for g in range(G):
        part = x[:, g * GROUP:(g + 1) * GROUP]
        a = np.abs(part).max(1)
        fine = np.isfinite(a)
        e = np.full(T, -126)
        for t in np.nonzero(fine)[0]:
            while a[t] > TOP[code] * 2.0 ** e[t]:
                e[t] += max(1, int(np.log2(a[t] / TOP[code]) - e[t] - 1))
        q = np.where(fine[:, None], part, 0.0) * (2.0 ** -e.astype(F64))[:, None]
        codes[:, g * GROUP:(g + 1) * GROUP] = np.where(fine[:, None], _nearest(q, code), 0)
        scales[:, g] = np.where(fine, e + 127, 255)
    return codes, scales


def unpack8(codes, scales, code):
    two = np.where(scales == 255, np.nan, np.where(scales == 0, 0.0, 2.0 ** (scales.astype(F64) - 127)))
    return numbers(code)[codes] * np.repeat(two, GROUP, 1)[:, :codes.shape[1]]


def layernorm(v, gamma, beta, eps):
    """(y, mean, rstd)."""
    m = v.mean(1)
    r = 1.0 / np.sqrt(((v - m[:, None]) ** 2).mean(1) + eps)
    return gamma * ((v - m[:, None]) * r[:, None]) + beta, m, r


def layernorm_grad(dy, v, mean, rstd, gamma, res=None):
    """(dx, dgamma, dbeta, dres_sum)."""
    xh = (v - mean[:, None]) * rstd[:, None]
    g = dy * gamma
    dx = (g - g.mean(1, keepdims=True) - xh * (g * xh).mean(1, keepdims=True)) * rstd[:, None]
    if res is not None:
        dx = dx + res
    return dx, (dy * xh).sum(0), dy.sum(0), None if res is None else res.sum(0)
