"""Oracle: the operators of one attention layer around the cache.

Test infrastructure only: rotary positions, the score rules (tanh cap, bias by
distance, documents, prefix, window, padding), attention of whole prompts and of
one token under them, and the prompt's importance.  Everything in fp64 from the
operands as stored.
"""
from __future__ import annotations

import math

import numpy as np


def rotary_frequencies(rot_dim, base=10000.0, scaling="none", factor=1.0, original_length=4096.0, low=1.0, high=None):
    """(radians per position of every pair, factor on rotated channels)."""
    p = np.arange(rot_dim // 2, dtype=np.float64)
    if scaling == "ntk":
        base = base * factor ** (rot_dim / (rot_dim - 2.0))
    w = base ** (-2.0 * p / rot_dim)
    if scaling == "linear":
        return w / factor, 1.0
    if scaling == "bands":
        turns = original_length * w / (2 * math.pi)
        keep = np.clip((turns - low) / ((4.0 if high is None else high) - low), 0, 1)
        return keep * w + (1 - keep) * w / factor, 1.0
    if scaling == "yarn":
        def at(n):
            return rot_dim * math.log(original_length / (2 * math.pi * n)) / (2 * math.log(base))
        first = max(0.0, math.floor(at(32.0 if high is None else high)))
        last = min(rot_dim - 1.0, math.ceil(at(low)))
        keep = 1 - np.clip((p - first) / max(last - first, 0.001), 0, 1)
        return keep * w + (1 - keep) * w / factor, 0.1 * math.log(factor) + 1.0
    return w, 1.0


def rotary(x, positions, w, magnitude=1.0, interleaved=False):
    """x [B, H, T, 128]; positions int [B, T]; w radians per position [rot / 2] -> fp64."""
    y = np.array(x, dtype=np.float64)
    r = 2 * len(w)
    angle = np.asarray(positions, dtype=np.float64)[:, None, :, None] * w
    c, s = np.cos(angle) * magnitude, np.sin(angle) * magnitude
    ia, ib = (slice(0, r, 2), slice(1, r, 2)) if interleaved else (slice(0, r // 2), slice(r // 2, r))
    a, b = y[..., ia].copy(), y[..., ib].copy()
    y[..., ia], y[..., ib] = a * c - b * s, b * c + a * s
    return y


def visible(T, documents=None, prefix=0, window=0):
    """bool [T, T]: query i sees key j."""
    m = np.zeros((T, T), dtype=bool)
    for i in range(T):
        a, z = 0, T
        if documents is not None:
            if documents[i] < 0:
                continue
            a = z = i
            while a > 0 and documents[a - 1] == documents[i]:
                a -= 1
            while z < T and documents[z] == documents[i]:
                z += 1
        for j in range(a, z):
            m[i, j] = (j <= i or j < prefix) and (not window or j > i - window)
    return m


def rule_scores(dots, scale, cap=0.0, slope=0.0, distance=None):
    """Scores of raw dot products (fp64) under a cap and a bias by distance."""
    s = np.asarray(dots, dtype=np.float64) * scale
    if cap:
        s = cap * np.tanh(s / cap)
    return s - slope * np.abs(distance) if slope else s


def masked_softmax(s, seen):
    """(p, lse) of each row over the keys seen; a row that sees nothing: 0 and -inf."""
    s = np.where(seen, s, -np.inf)
    m = s.max(axis=-1, keepdims=True)
    m = np.where(np.isfinite(m), m, 0.0)
    e = np.where(seen, np.exp(s - m), 0.0)
    total = e.sum(axis=-1, keepdims=True)
    with np.errstate(divide="ignore"):
        return e / np.where(total == 0, 1, total), (m + np.log(total))[..., 0]


def prompt_attention(q, k, v, seen, scale, cap=0.0, slopes=None):
    """q [G, T, D] of one KV head's query heads; k, v [T, D]; seen [T, T].

    Returns (out [G, T, D], lse [G, T], p [G, T, T]); rows of k and v that a query does
    not see do not enter its results, whatever they hold."""
    q, k, v = (np.asarray(x, dtype=np.float64) for x in (q, k, v))
    G, T, _ = q.shape
    i, j = np.arange(T)[:, None], np.arange(T)[None, :]
    with np.errstate(invalid="ignore"):
        s = np.stack([rule_scores(q[g] @ k.T, scale, cap, 0.0 if slopes is None else float(slopes[g]), i - j)
                      for g in range(G)])
    p, lse = masked_softmax(s, seen[None])
    used = seen.any(axis=0)
    clean = np.where((used & np.isfinite(v).all(axis=1))[:, None], v, 0.0)
    return p @ clean, lse, p


def decode_attention(cache, q16, scale, begin, cap=0.0, slopes=None, window=0, balance=None):
    """One token's attention over an OracleCache under score rules.

    q16 fp16 [H, G, D]; begin int [H] (first visible position of each head's sequence);
    slopes [H, G] or None; returns (o, p) fp64 [H, G, D], [H, G, L]."""
    L = cache.length
    o = np.zeros((cache.n_heads, cache.G, cache.d))
    p = np.zeros((cache.n_heads, cache.G, L))
    pos = np.arange(L)
    for h in range(cache.n_heads):
        k, v = (x.astype(np.float64) for x in cache.values(h))
        q = np.asarray(q16[h], np.float16).astype(np.float32)
        if balance is not None:
            q = q / np.asarray(balance[h], np.float32)
        seen = pos >= begin[h]
        if window:
            seen &= pos > L - 1 - window
        if not cache.lo_bits:
            seen &= cache.is_hi[h, :L]
        for g in range(cache.G):
            s = rule_scores(k @ q[g].astype(np.float64), scale, cap, 0.0 if slopes is None else float(slopes[h, g]),
                            L - 1 - pos)
            p[h, g], _ = masked_softmax(s, seen)
            o[h, g] = p[h, g] @ np.where(seen[:, None], v, 0.0)
    return o, p
