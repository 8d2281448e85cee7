"""CPU oracle for the operators that choose tokens of a paged context, in float64:
attention of drafted trees, bounds of blocks and the choice by them, attention over
chosen blocks, attention weights per token, and the choice and move of the tokens
that stay.

TEST INFRASTRUCTURE ONLY (see ``oracle.attention``).  It shares no code with the HIP
path.
"""

from __future__ import annotations

from fractions import Fraction

import numpy as np

from .attention import bf16_to_f64, gather_sequence

BLOCK = 16


def path(parents, i):
    """Node i of a tree and its ancestors, ascending; a parent that is not below its node is the root's."""
    out = [i]
    while 0 <= parents[out[-1]] < out[-1]:
        out.append(int(parents[out[-1]]))
    return out[::-1]


def rows_over(q, k, v, scale, cap=0.0):
    """Outputs and weights of query rows q [R][D] over K, V [n][D] (n may be 0)."""
    if k.shape[0] == 0:
        return np.zeros((q.shape[0], v.shape[1])), np.zeros((q.shape[0], 0))
    with np.errstate(all="ignore"):
        s = scale * (q @ k.T)
        if cap:
            s = cap * np.tanh(s / cap)
        w = np.exp(s - s.max(axis=1, keepdims=True))
        w /= w.sum(axis=1, keepdims=True)
        return w @ v, w


def tree_attention(q, q_start, parents, k_pool, v_pool, tables, ctx, scale, cap=0.0):
    """out [total][Hq][D] of nodes q (float64 [total][Hq][D])."""
    out = np.zeros(q.shape)
    hkv = k_pool.shape[1]
    group = q.shape[1] // hkv
    for b in range(len(q_start) - 1):
        start, n, length = int(q_start[b]), int(ctx[b]), int(q_start[b + 1] - q_start[b])
        K, V = gather_sequence(k_pool, v_pool, tables[b], n)
        for i in range(length):
            seen = list(range(n - length)) + [n - length + j for j in path(parents[start:start + length], i)]
            for g in range(hkv):
                h = slice(g * group, (g + 1) * group)
                out[start + i, h] = rows_over(q[start + i, h], K[g][seen], V[g][seen], scale, cap)[0]
    return out


def block_bounds(k_rows):
    """[2][D] least and greatest of key rows [n][D], NaN left out."""
    with np.errstate(all="ignore"):
        return np.stack([np.fmin.reduce(k_rows, axis=0, initial=np.inf), np.fmax.reduce(k_rows, axis=0, initial=-np.inf)])


def block_score(q_heads, bounds):
    """Exact score of a block: rationals, so that no order of sums matters.  q_heads [G][D], bounds [2][D], finite."""
    total = Fraction(0)
    for q in q_heads:
        for x, lo, hi in zip(q, bounds[0], bounds[1]):
            total += max(Fraction(x) * Fraction(lo), Fraction(x) * Fraction(hi))
    return total


def select_blocks(scores, first, last, most):
    """Places of a sequence's chosen blocks, ascending; scores: of all its blocks."""
    n = len(scores)
    if n <= most:
        return list(range(n))
    free = sorted(range(first, n - last), key=lambda j: (-scores[j], j))[:most - first - last]
    return sorted(list(range(first)) + free + list(range(n - last, n)))


def selected_attention(q, selected, k_pool, v_pool, tables, ctx, scale):
    """out [B][Hq][D] over the listed blocks [B][Hkv][k]; entries that name no block are passed over."""
    out = np.zeros(q.shape)
    hkv = k_pool.shape[1]
    group = q.shape[1] // hkv
    for b in range(q.shape[0]):
        n = int(ctx[b])
        K, V = gather_sequence(k_pool, v_pool, tables[b], n)
        for g in range(hkv):
            t = [t for j in selected[b, g] if 0 <= j < (n + BLOCK - 1) // BLOCK for t in range(BLOCK * j, min(n, BLOCK * j + BLOCK))]
            h = slice(g * group, (g + 1) * group)
            out[b, h] = rows_over(q[b, h], K[g][t], V[g][t], scale)[0]
    return out


def decode_weights(q, k_pool, v_pool, tables, ctx, scale):
    """(out [B][Hq][D], list of the weights [n_b] summed over the heads)."""
    out, weights = np.zeros(q.shape), []
    hkv = k_pool.shape[1]
    group = q.shape[1] // hkv
    for b in range(q.shape[0]):
        n = int(ctx[b])
        K, V = gather_sequence(k_pool, v_pool, tables[b], n)
        total = np.zeros(n)
        for g in range(hkv):
            h = slice(g * group, (g + 1) * group)
            out[b, h], w = rows_over(q[b, h], K[g], V[g], scale)
            total += w.sum(axis=0)
        weights.append(total)
    return out, weights


def keep_heaviest(totals, first, recent, keep):
    """Kept tokens behind the first ones, as token - first, ascending; totals [n] of one sequence."""
    n = len(totals)
    first = min(max(first, 0), n)
    end = max(first, n - recent)
    want = min(max(keep - first - (n - end), 0), end - first)
    free = sorted(range(first, end), key=lambda t: (not np.isnan(totals[t]), -totals[t] if not np.isnan(totals[t]) else 0, t))
    return [t - first for t in sorted(free[:want])] + [t - first for t in range(end, n)]


def compact(pool, table, to, first, kept):
    """The pool after the move of one sequence's kept tokens."""
    out = pool.copy()
    for j, t in enumerate(kept):
        s, d = first + int(t), first + j
        out[to[d // BLOCK], :, d % BLOCK] = pool[table[s // BLOCK], :, s % BLOCK]
    return out
