"""Oracles of the operators around the verification step: page plans, rotary positions, token log probabilities.

TEST INFRASTRUCTURE ONLY.  Definitions written out in plain Python and float64 NumPy; nothing is shared with the product.
"""
from __future__ import annotations

import numpy as np


def cache_plan(held, want, table, free, count, page, max_rows):
    """Block tables and slots from request lengths, request by request and page by page.  max_rows None: rows are not wanted.
    Returns dict(table, free, count, seq_lens, row_start, positions, slots, info)."""
    table, free = np.array(table), np.array(free)
    width = table.shape[1] if table.ndim == 2 else 0
    pages = lambda n: -(-n // page)
    fits = lambda h, w: h >= 0 and w >= 0 and pages(h) <= width and pages(w) <= width
    stack = [int(x) for x in free[:count]]
    lens = [int(h) for h in held]
    freed = 0
    for b, (h, w) in enumerate(zip(held, want)):
        if fits(h, w) and w < h:
            for i in range(pages(w), pages(h)):
                stack.append(int(table[b, i]))
                freed += 1
            lens[b] = int(w)
    pushed = list(stack)
    row_start, positions, slots, taken, refused, dry = [], [], [], 0, 0, False
    for b, (h, w) in enumerate(zip(held, want)):
        row_start.append(len(positions))
        if not fits(h, w):
            refused += int(h != w)
            continue
        if w <= h:
            continue
        need = pages(w) - pages(h)
        dry = dry or need > len(stack) or (max_rows is not None and len(positions) + w - h > max_rows)
        if dry:
            refused += 1
            continue
        for i in range(pages(h), pages(w)):
            table[b, i] = stack.pop()
            taken += 1
        for t in range(h, w):
            positions.append(t)
            slots.append(int(table[b, t // page]) * page + t % page)
        lens[b] = int(w)
    row_start.append(len(positions))
    for i in range(count, len(stack)):
        free[i] = stack[i]
    n = max_rows or 0
    return dict(table=table, free=free, count=len(stack), seq_lens=np.array(lens, np.int32), row_start=np.array(row_start, np.int32),
                positions=np.array((positions + [0] * n)[:n], np.int32), slots=np.array((slots + [-1] * n)[:n], np.int32),
                info=np.array([len(positions), taken, freed, refused], np.int32), pushed=pushed)


def rope_turn(x, positions, frequencies, rotary, interleaved, magnitude=1.0, back=False):
    """x [rows, heads, D] float64: the first `rotary` elements of every head turned by their angles (back: the transpose)."""
    x = np.array(x, dtype=np.float64)
    half = rotary // 2
    i = np.arange(half)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    angle = np.asarray(positions, np.float64)[:, None] * np.asarray(frequencies, np.float64)[None, :half]
    c, s = magnitude * np.cos(angle)[:, None, :], magnitude * np.sin(angle)[:, None, :] * (-1.0 if back else 1.0)
    first, second = x[..., a].copy(), x[..., b].copy()
    x[..., a] = first * c - second * s
    x[..., b] = second * c + first * s
    return x


def token_logprobs(logits, tokens, T, n_top=0):
    """float64 results of rows of logits (widened exactly); T a number or one per row.  Returns dict(logprob, lse, entropy, top_ids,
    top_logprobs)."""
    z = np.asarray(logits, np.float64)
    M, V = z.shape
    T = np.broadcast_to(np.asarray(T, np.float64), (M,))
    out = dict(logprob=np.zeros(M), lse=np.full(M, -np.inf), entropy=np.zeros(M), top_ids=np.full((M, n_top), -1, np.int32),
               top_logprobs=np.full((M, n_top), -np.inf))
    for m in range(M):
        x = z[m] / T[m]
        top = x.max()
        if top > -np.inf:
            e = np.exp(x - top)
            out["lse"][m] = top + np.log(e.sum())
            p = e / e.sum()
            out["entropy"][m] = -(p[p > 0] * (x[p > 0] - out["lse"][m])).sum()
        lp = x - out["lse"][m] if top > -np.inf else np.full(V, -np.inf)
        if tokens is not None and 0 <= tokens[m] < V:
            out["logprob"][m] = lp[tokens[m]]
        order = np.lexsort((np.arange(V), -z[m]))[:n_top]  # (-0.0 and 0.0 compare equal)
        out["top_ids"][m, :len(order)] = order
        out["top_logprobs"][m, :len(order)] = lp[order]
    return out


def token_logprobs_backward(logits, tokens, T, dlogprob, dentropy):
    """Gradient with respect to the logits of sum_m dlogprob[m] logprob[m] + dentropy[m] entropy[m], float64."""
    z = np.asarray(logits, np.float64)
    M, V = z.shape
    T = np.broadcast_to(np.asarray(T, np.float64), (M,))
    f = token_logprobs(z, tokens, T)
    g = np.zeros((M, V))
    for m in range(M):
        if f["lse"][m] == -np.inf:
            continue
        lp = z[m] / T[m] - f["lse"][m]
        p = np.exp(lp)
        known = tokens is not None and 0 <= tokens[m] < V
        gl = dlogprob[m] if dlogprob is not None and known else 0.0
        gh = dentropy[m] if dentropy is not None else 0.0
        g[m] = -gl * p
        g[m][p > 0] -= gh * p[p > 0] * (lp[p > 0] + f["entropy"][m])
        if known:
            g[m, tokens[m]] += gl
        g[m] /= T[m]
    return g
