"""Oracle of the operators for long contexts, the last stage and serving, in 64 bits and from their definitions.

Layouts as in oracle.ops: rows are tokens, sequence b in rows b*seq ..; heads are column blocks; H query heads share KV key heads,
the H/KV query heads of a key head following each other.
"""
from __future__ import annotations

import numpy as np


def _length(lengths, b, seq):
    return seq if lengths is None else int(min(max(lengths[b], 0), seq))


def seen(n, window, sinks):
    """[n, n] truth values: does query i see key j."""
    i, j = np.arange(n)[:, None], np.arange(n)[None, :]
    return (j <= i) & ((j > i - window) | (j < sinks))


# ---- sliding-window attention with sinks -----------------------------------------------------------------------------
def _softmax(q, k, window, sinks):
    s = q @ k.T / np.sqrt(q.shape[1])
    s = np.where(seen(len(q), window, sinks), s, -np.inf)
    m = s.max(axis=1, keepdims=True)
    e = np.exp(s - m)
    l = e.sum(axis=1, keepdims=True)
    return e / l, (m + np.log(l))[:, 0]


def _heads(qkv, rows, h, H, KV, dh):
    g = h // (H // KV)
    return [qkv[rows, c * dh:(c + 1) * dh] for c in (h, H + g, H + KV + g)]


def window_attention_fwd(qkv, seq, H, KV, dh, window, sinks, lengths=None):
    """-> out [rows, H dh], lse (natural) [batch, H, seq]."""
    nb = len(qkv) // seq
    out, lse = np.zeros((len(qkv), H * dh)), np.full((nb, H, seq), -np.inf)
    for b in range(nb):
        n = _length(lengths, b, seq)
        rows = slice(b * seq, b * seq + n)
        for h in range(H if n else 0):
            q, k, v = _heads(qkv, rows, h, H, KV, dh)
            p, lse[b, h, :n] = _softmax(q, k, window, sinks)
            out[rows, h * dh:(h + 1) * dh] = p @ v
    return out, lse


def window_attention_p1(qkv, d_out, seq, H, KV, dh, window, sinks, lengths=None):
    """-> dqkv: dS = P (dP - rowsum(dP P)); the gradients of shared heads add up."""
    d = np.zeros((len(qkv), (H + 2 * KV) * dh))
    for b in range(len(qkv) // seq):
        n = _length(lengths, b, seq)
        rows = slice(b * seq, b * seq + n)
        for h in range(H if n else 0):
            q, k, v = _heads(qkv, rows, h, H, KV, dh)
            dq, dk, dv = _heads(d, rows, h, H, KV, dh)
            do = d_out[rows, h * dh:(h + 1) * dh]
            p, _ = _softmax(q, k, window, sinks)
            dp = do @ v.T
            ds = p * (dp - (dp * p).sum(axis=1, keepdims=True)) / np.sqrt(dh)
            dq += ds @ k
            dk += ds.T @ q
            dv += p.T @ do
    return d


# ---- the cache of a batch of sequences, token by token --------------------------------------------------------------------
def cache_row(p, capacity, sinks):
    return p if p < sinks else sinks + (p - sinks) % (capacity - sinks)


def window_decode(q, k_tokens, v_tokens, H, KV, dh, window, sinks, capacity):
    """One sequence: q [H dh] of its last token over all of its tokens [n, KV dh] -> out [H dh], lse [H].  Of the tokens behind the
    sinks only the last capacity - sinks are still there."""
    n = len(k_tokens)
    at = [p for p in range(n) if p < sinks or p >= n - min(window, capacity - sinks)]
    out, lse = np.zeros(H * dh), np.full(H, -np.inf)
    for h in range(H if n else 0):
        g = h // (H // KV)
        s = k_tokens[at, g * dh:(g + 1) * dh] @ q[h * dh:(h + 1) * dh] / np.sqrt(dh)
        e = np.exp(s - s.max())
        out[h * dh:(h + 1) * dh] = e @ v_tokens[at, g * dh:(g + 1) * dh] / e.sum()
        lse[h] = s.max() + np.log(e.sum())
    return out, lse


# ---- rotary positions -------------------------------------------------------------------------------------------------------
def rotary_theta(rot_dim, base, scaling="plain", factor=1.0, low=1.0, high=32.0, original=4096.0):
    i = np.arange(rot_dim // 2)
    if scaling == "base":
        base = base * factor ** (rot_dim / (rot_dim - 2))
    theta = base ** (-2.0 * i / rot_dim)
    if scaling == "linear":
        theta = theta / factor
    if scaling == "ramp":
        g = np.clip((original * theta / (2 * np.pi) - low) / (high - low), 0.0, 1.0)
        theta = theta * ((1 - g) / factor + g)
    return theta


def rotary(x, heads, dh, theta, positions, interleaved=False, backward=False, magnitude=1.0):
    """x [rows, heads dh]; every pair of columns as a vector of the plane, turned by position * theta."""
    y = np.array(x[:, :heads * dh], dtype=np.float64)
    half = len(theta)
    for h in range(heads):
        for i in range(half):
            a, b = (h * dh + 2 * i, h * dh + 2 * i + 1) if interleaved else (h * dh + i, h * dh + half + i)
            ang = np.asarray(positions, np.float64) * theta[i] * (-1.0 if backward else 1.0)
            c, s = magnitude * np.cos(ang), magnitude * np.sin(ang)
            y[:, a], y[:, b] = x[:, a] * c - x[:, b] * s, x[:, a] * s + x[:, b] * c
    return y


# ---- log probabilities --------------------------------------------------------------------------------------------------------
def logprobs(x, targets):
    """-> logp, entropy, lse of rows of logits."""
    logp, entropy, lse = np.zeros(len(x)), np.zeros(len(x)), np.full(len(x), -np.inf)
    for r, row in enumerate(x):
        there = row > -np.inf
        if there.any():
            m = row.max()
            lse[r] = m + np.log(np.exp(row[there] - m).sum())
            lp = row[there] - lse[r]
            entropy[r] = -(np.exp(lp) * lp).sum()
        if 0 <= targets[r] < len(row):
            logp[r] = row[targets[r]] - lse[r] if there.any() else -np.inf
    return logp, entropy, lse


def top(row, k):
    """The k largest of a row in order, ties by the lower index."""
    return sorted(range(len(row)), key=lambda i: (-row[i], i))[:k]


def logprobs_p1(x, targets, d_logp, d_entropy):
    d = np.zeros(x.shape)
    _, entropy, lse = logprobs(x, targets)
    for r, row in enumerate(x):
        if not (row > -np.inf).any():
            continue
        given = 0 <= targets[r] < len(row)
        lp = row - lse[r]
        p = np.exp(lp)
        d[r] = -p * (d_logp[r] if given else 0.0) - d_entropy[r] * p * np.where(p > 0, np.where(p > 0, lp, 0.0) + entropy[r], 0.0)
        if given:
            d[r, targets[r]] += d_logp[r]
    return d


# ---- the norm over gradient tensors, and clipping ------------------------------------------------------------------------------
def grad_clip(grads, max_norm):
    norm = np.sqrt(sum(float((g.astype(np.float64) ** 2).sum()) for g in grads))
    c = max_norm / norm if np.isfinite(norm) and norm > max_norm else 1.0
    return norm, [g.astype(np.float64) * c for g in grads]
