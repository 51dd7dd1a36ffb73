"""64-bit restatement of the operators around a step's attention -- TEST INFRASTRUCTURE (see the package docstring).

Each function states the operator's definition one row, request or sequence at a time; nothing is shared with the CUDA sources.
"""
from __future__ import annotations

import math
from fractions import Fraction

import numpy as np

from . import bf16_bits_to_f64, gather_logical

PAGE = 16


def head_norm(x, weight, eps):
    """x: float64 [rows, heads, D]; weight: [D], [heads, D] or None."""
    y = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    return y if weight is None else y * np.asarray(weight, np.float64)


def verify(target, draft, tokens, parents, size, uniforms, draw):
    """target, draft: float64 [B, T, V] (draft None: certain).  Returns (path, path_lens, next_tokens).  Small vocabularies are computed in
    fractions, so that ties are decided as the definition says."""
    B, T, V = target.shape
    exact = (lambda x: np.array([Fraction(float(e)) for e in x], dtype=object)) if V <= 64 else (lambda x: x)  # noqa: E731
    tokens, parents, uniforms = np.asarray(tokens), np.asarray(parents), np.asarray(uniforms)
    number = (lambda x: Fraction(float(x))) if V <= 64 else float  # noqa: E731
    path, took, follows = np.full((B, T), -1, np.int64), np.zeros(B, np.int64), np.full(B, -1, np.int64)
    clean = lambda x: exact(np.where(x > 0, x, 0.0))  # noqa: E731  (NaN compares false)
    for b in range(B):
        t = min(int(size[b]), T)
        if t <= 0:
            continue
        now, way = 0, [0]
        r = clean(target[b, 0])
        q = None if draft is None else clean(draft[b, 0])
        for i in range(1, t):
            x = int(tokens[b, i])
            if parents[b, i] != now or not 0 <= x < V:
                continue
            if draft is None:
                q = exact(np.arange(V) == x)
            if number(uniforms[b, i]) * q[x] < r[x]:
                now = i
                way.append(i)
                r = clean(target[b, i])
                q = None if draft is None else clean(draft[b, i])
                continue
            left = np.maximum(r - q, 0 * r)
            if left.sum() > 0:
                r = left / left.sum()
            if draw == "distinct":
                q = q.copy()
                q[x] = 0 * q[x]
                q = q / q.sum() if q.sum() > 0 else q
        sums = np.cumsum(r)
        u = float(uniforms[b, 0])
        above = np.nonzero(sums > number(max(u if u == u else 0.0, 0.0)) * sums[-1])[0]
        some = np.nonzero(r > 0)[0]
        follows[b] = above[0] if len(above) else some[-1] if len(some) else -1
        path[b, :len(way)], took[b] = way, len(way)
    return path, took, follows


def extend(rows, old, new, table, counts, free_list, count, begin=0, max_rows=None):
    """In place on the table and the counts.  Returns (row_starts, new_lens, seq, slots, end, recorded)."""
    n, pages, begin = len(rows), len(counts), max(begin, 0)
    length = min(count, len(free_list))
    starts = np.concatenate([[0], np.cumsum(np.maximum(new, 0))]).astype(np.int64)
    room = math.inf if max_rows is None else max_rows
    seq, slots = (np.full(max_rows or 0, -1, np.int64) for _ in range(2))
    lens, recorded, lacking, end = np.array(old, np.int64), False, 0, begin
    granted = []
    for f in range(n):
        r, c, m = int(rows[f]), int(old[f]), int(new[f])
        if r < 0:
            continue
        bad = r >= table.shape[0] or list(rows).count(r) > 1 or c < 0 or m < 0 or c + m > table.shape[1] * PAGE or starts[f + 1] > room
        want = []
        if not bad and m > 0:
            for i in range(c // PAGE, (c + m - 1) // PAGE + 1):
                if table[r, i] < 0:
                    want.append(i)
                    bad |= i == c // PAGE and c % PAGE != 0
                else:
                    bad |= table[r, i] >= pages or counts[table[r, i]] != 1
        if bad:
            recorded = True
            continue
        lacking += len(want)
        if want and begin + lacking > length:
            continue
        granted.append((f, r, want, begin + lacking - len(want)))
    for f, r, want, at in granted:
        for k, i in enumerate(want):
            page = int(free_list[at + k])
            if 0 <= page < pages and counts[page] == 0:
                table[r, i], counts[page] = page, 1
            else:
                recorded = True
        if want:
            end = at + len(want)
        lens[f] = old[f] + new[f]
        if max_rows is not None:
            seq[starts[f]:starts[f + 1]] = r
            slots[starts[f]:starts[f + 1]] = np.arange(old[f], old[f] + max(int(new[f]), 0))
    return np.minimum(starts, room if max_rows is not None else starts[-1]).astype(np.int64), lens, seq, slots, end, recorded


def decode_attention(pool, Hq, Hkv, D, q, lens, table, window=0, scale=None):
    """q: uint16 [B, Hq, D].  Returns (out, lse, spread, bound) in float64, as draft.tree_attention."""
    B, G = q.shape[0], Hq // Hkv
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    out, spread = np.zeros((B, Hq, D)), np.zeros((B, Hq, D))
    lse, bound = np.full((B, Hq), -np.inf), np.zeros((B, Hq))
    qf = bf16_bits_to_f64(q)
    for b in range(B):
        n = int(lens[b])
        if n <= 0:
            continue
        k, v = gather_logical(pool, Hkv, PAGE, D, table[b], max(0, n - window) if window else 0, n)
        k, v = bf16_bits_to_f64(k), bf16_bits_to_f64(v)
        for h in range(Hq):
            kk, vv = k[:, h // G], v[:, h // G]
            x = kk @ qf[b, h] * scale
            top = x.max()
            p = np.exp(x - top)
            out[b, h] = p @ vv / p.sum()
            spread[b, h] = p @ np.abs(vv) / p.sum()
            lse[b, h] = top + math.log(p.sum())
            bound[b, h] = (np.abs(kk) @ np.abs(qf[b, h])).max() * scale
    return out, lse, spread, bound
