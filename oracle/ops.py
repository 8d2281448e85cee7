"""CPU oracle for the operators around the cache's attention, in float64: norm
and rotation of head rows, and attention with capped, biased or masked scores.

TEST INFRASTRUCTURE ONLY (see ``oracle.attention``).  It shares no code with
the HIP path.

Definitions.  A head's row x (head_dim D, weight w, position t):

    y = x * w / sqrt(mean(x^2) + eps)            (w None: y = x)
    pair i < r/2 of y, (y_i, y_{i + r/2}) or (y_{2i}, y_{2i+1}), as a complex
    number, times magnitude * exp(1j * t * f_i)

A query row of head h at position p over tokens t of its sequence:

    s_t = cap * tanh(scale * <q, K_t> / cap) - slope_h * |p - t|
    out = softmax of s over lo <= t < hi, times V; zeros where that is empty.
"""

from __future__ import annotations

import numpy as np

from .attention import gather_sequence


def head_rows(x, weight, eps, positions, freqs, magnitude, interleaved):
    """Rows x [n][heads][D] (float64) normed and turned to positions [n]."""
    y = np.array(x, dtype=np.float64)
    if weight is not None:
        y = y * np.asarray(weight, np.float64) / np.sqrt((y * y).mean(axis=-1, keepdims=True) + eps)
    half = len(freqs)
    if half:
        turn = magnitude * np.exp(1j * np.asarray(positions, np.float64)[:, None] * np.asarray(freqs, np.float64))
        first = slice(0, 2 * half, 2) if interleaved else slice(0, half)
        second = slice(1, 2 * half, 2) if interleaved else slice(half, 2 * half)
        pair = (y[..., first] + 1j * y[..., second]) * turn[:, None, :]
        y[..., first], y[..., second] = pair.real, pair.imag
    return y


def biased_rows(q, k, v, scale, cap, slopes, pos, lo, hi):
    """Query rows q [R][D] of one KV head over K, V [n][D]; slopes, pos, lo, hi [R].
    Hidden tokens are left out, whatever they hold."""
    out = np.zeros((q.shape[0], v.shape[1]))
    for r in range(q.shape[0]):
        a, b = max(int(lo[r]), 0), min(int(hi[r]), k.shape[0])
        if b <= a:
            continue
        with np.errstate(all="ignore"):
            s = scale * (k[a:b] @ q[r])
            if cap:
                s = cap * np.tanh(s / cap)
            s = s - slopes[r] * np.abs(pos[r] - np.arange(a, b))
            w = np.exp(s - s.max())
            out[r] = (w / w.sum()) @ v[a:b]
    return out


def biased_attention(q, q_start, k_pool, v_pool, block_tables, context_lens, scale, cap=0.0, slopes=None, window=0,
                     first=None, prefix=None):
    """out float64 [total][Hq][D] of chunks q (float64 [total][Hq][D]) over pools of bf16 bits."""
    total, hq, d = q.shape
    hkv = k_pool.shape[1]
    group = hq // hkv
    out = np.zeros((total, hq, d))
    slopes = np.zeros(hq) if slopes is None else np.asarray(slopes, np.float64)
    for b in range(len(q_start) - 1):
        n, start, length = int(context_lens[b]), int(q_start[b]), int(q_start[b + 1]) - int(q_start[b])
        K, V = gather_sequence(k_pool, v_pool, block_tables[b], n)
        rows = np.arange(start, start + length)
        pos = n - length + np.arange(length)
        lo = np.zeros(length, int) if first is None else np.asarray(first)[rows]
        if window:
            lo = np.maximum(lo, pos - window + 1)
        hi = pos + 1 if prefix is None else np.maximum(pos + 1, min(int(prefix[b]), n))
        for h in range(hq):
            g = h // group
            out[rows, h] = biased_rows(q[rows, h], K[g], V[g], scale, cap, np.full(length, slopes[h]), pos, lo, hi)
    return out
