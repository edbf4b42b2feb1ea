"""Oracle of the operators of a stage that is trained on packed documents, in 64 bits and from their definitions: norms of query and key heads with
rotary positions, causal attention over sequences that lie one behind the other, a stash in 8 bits.

Layouts as in oracle.operators: rows are tokens, heads are column blocks, H query heads share KV key heads.
"""
from __future__ import annotations

import math

import numpy as np

from . import operators as ops

BLOCK = 1024                                     # tokens of a column that share a scale


# ---- norms of query and key heads -------------------------------------------------------------------------------------
def _gains(gq, gk, H, KV):
    return np.concatenate([np.tile(gq, (H, 1)), np.tile(gk, (KV, 1))])


def _turn(x, angles, layout, back):
    """x [rows, heads, dh]; angles [rows, half]; pairs (i, i + half) or (2i, 2i + 1) as complex numbers."""
    half = angles.shape[1]
    a = np.arange(half) * (2 if layout else 1)
    b = a + (1 if layout else half)
    z = (x[..., a] + 1j * x[..., b]) * np.exp((-1j if back else 1j) * angles)[:, None]
    y = x.copy()
    y[..., a], y[..., b] = z.real, z.imag
    return y


def qk_norm(x, gq, gk, H, KV, eps, angles, layout=0):
    """x [rows, (H + KV) dh] -> y = R (x / sqrt(mean x^2 + eps) g)."""
    x = np.asarray(x, np.float64).reshape(len(x), H + KV, -1)
    n = x / np.sqrt((x * x).mean(axis=2, keepdims=True) + eps)
    return _turn(n * _gains(gq, gk, H, KV), angles, layout, False).reshape(len(x), -1)


def qk_norm_p1(dy, x, gq, gk, H, KV, eps, angles, layout=0):
    """-> dx, dg [2, dh]."""
    x, dy = (np.asarray(t, np.float64).reshape(len(x), H + KV, -1) for t in (x, dy))
    r = 1 / np.sqrt((x * x).mean(axis=2, keepdims=True) + eps)
    n, dz = x * r, _turn(dy, angles, layout, True)
    dn = dz * _gains(gq, gk, H, KV)
    dx = r * (dn - n * (dn * n).mean(axis=2, keepdims=True))
    dg = (dz * n).sum(axis=0)
    return dx.reshape(len(x), -1), np.stack([dg[:H].sum(axis=0), dg[H:].sum(axis=0)])


# ---- attention over packed sequences -----------------------------------------------------------------------------------
def packed_attention_fwd(qkv, starts, H, KV, dh):
    """-> out [rows, H dh], lse (natural) [H, rows]."""
    out, lse = np.zeros((len(qkv), H * dh)), np.full((H, len(qkv)), -np.inf)
    for a, b in zip(starts[:-1], starts[1:]):
        if b > a:
            out[a:b], l = ops.window_attention_fwd(qkv[a:b], b - a, H, KV, dh, b - a, 0)
            lse[:, a:b] = l[0]
    return out, lse


def packed_attention_p1(qkv, d_out, starts, H, KV, dh):
    d = np.zeros((len(qkv), (H + 2 * KV) * dh))
    for a, b in zip(starts[:-1], starts[1:]):
        if b > a:
            d[a:b] = ops.window_attention_p1(qkv[a:b], d_out[a:b], b - a, H, KV, dh, b - a, 0)
    return d


# ---- a stash in 8 bits --------------------------------------------------------------------------------------------------
def held(x):
    """What x [tokens, cols] is held as: value by value, without vector shortcuts for the scale."""
    x = np.asarray(x, np.float64)
    y = np.empty_like(x)
    for t in range(0, len(x), BLOCK):
        for c in range(x.shape[1]):
            v = x[t:t + BLOCK, c]
            if not np.all(np.isfinite(v)):
                y[t:t + BLOCK, c] = np.nan
                continue
            top, e = float(np.max(np.abs(v))), -126
            if top > 127 * 2.0 ** e:
                e = max(e, math.frexp(top)[1] - 8)
                while e < 121 and top > math.ldexp(127.0, e):
                    e += 1
            y[t:t + BLOCK, c] = np.clip(np.rint(v / math.ldexp(1.0, e)), -127, 127) * math.ldexp(1.0, e)
    return y


def stash8_dw(xs, dys):
    """The micro-batches of a set, each held by itself -> X^T dY, and for every element the sum of the blocks' magnitudes (of which fp32 loses a share)."""
    dw = size = 0.0
    for x, dy in zip(xs, dys):
        hx, hd = held(x), held(dy)
        for t in range(0, len(x), BLOCK):
            part = hx[t:t + BLOCK].T @ hd[t:t + BLOCK]
            dw, size = dw + part, size + np.abs(part)
    return dw, size
