"""64-bit restatement of the drafted-token operators -- TEST INFRASTRUCTURE (see the package docstring).

Each function states the operator's definition row by row over bf16 bit patterns (uint16), with the layout helpers
of the package; nothing is shared with the CUDA sources.
"""
from __future__ import annotations

import math

import numpy as np

from . import bf16_bits_to_f64, gather_logical

PAGE = 16


def frequencies(rot, theta=10000.0, scaling="plain", factor=1.0, original=0.0, low=0.0, high=0.0):
    """Radians per position of each pair, one at a time."""
    out = []
    for i in range(rot // 2):
        f = theta ** (-2.0 * i / rot)
        if scaling == "linear":
            f /= factor
        elif scaling == "ntk":
            f = (theta * factor ** (rot / (rot - 2.0))) ** (-2.0 * i / rot)
        elif scaling == "bands":
            lo, hi = low or 1.0, high or 4.0
            wave = 2 * math.pi / f
            if wave > original / lo:
                f /= factor
            elif wave >= original / hi:
                s = (original / wave - lo) / (hi - lo)
                f = (1 - s) * f / factor + s * f
        elif scaling == "yarn":
            lo, hi = low or 1.0, high or 32.0
            at = lambda beta: rot * math.log(original / (beta * 2 * math.pi)) / (2 * math.log(theta))  # noqa: E731
            a, b = max(math.floor(at(hi)), 0), min(math.ceil(at(lo)), rot - 1)
            w = min(max((i - a) / max(b - a, 0.001), 0.0), 1.0)
            f = f / factor * w + f * (1 - w)
        out.append(f)
    return np.array(out)


def rotate(x, positions, freq, layout, amplitude=1.0):
    """x: float64 [rows, heads, D]."""
    y = x.copy()
    r = len(freq)
    for i in range(r):
        c, s = np.cos(positions * freq[i])[:, None] * amplitude, np.sin(positions * freq[i])[:, None] * amplitude
        j, k = (i, i + r) if layout == "half" else (2 * i, 2 * i + 1)
        y[:, :, j], y[:, :, k] = x[:, :, j] * c - x[:, :, k] * s, x[:, :, k] * c + x[:, :, j] * s
    return y


def tree_attention(pool, Hq, Hkv, D, q, mask, positions, ctx, size, table, window=0, scale=None):
    """q: uint16 [B, T, Hq, D].  Returns (out, lse, spread, bound) in float64: spread = sum_j p_j |V_j| per element and
    bound = the largest sum_d |q_d K_jd| * scale of a row, from which the tests derive their tolerances."""
    B, T, G = q.shape[0], q.shape[1], Hq // Hkv
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    out, spread = np.zeros((B, T, Hq, D)), np.zeros((B, T, Hq, D))
    lse, bound = np.full((B, T, Hq), -np.inf), np.zeros((B, T, Hq))
    qf = bf16_bits_to_f64(q)
    for b in range(B):
        c, t = int(ctx[b]), min(int(size[b]), T)
        if c < 0 or t <= 0:
            continue
        lo = max(0, c + 1 - window) if window else 0
        n = c + t
        k, v = gather_logical(pool, Hkv, PAGE, D, table[b], lo, n)
        k, v = bf16_bits_to_f64(k), bf16_bits_to_f64(v)
        where = np.concatenate([np.arange(lo, c), np.maximum(positions[b, :t], c)]).astype(np.int64)
        for i in range(t):
            seen = np.ones(n - lo, dtype=bool)
            for m in range(t):
                seen[c - lo + m] = (int(mask[b, i]) >> m) & 1
            if window:
                seen &= where > max(int(positions[b, i]), c) - window
            if not seen.any():
                continue
            for h in range(Hq):
                kk, vv = k[seen, h // G], v[seen, h // G]
                x = kk @ qf[b, i, h] * scale
                top = x.max()
                p = np.exp(x - top)
                out[b, i, h] = p @ vv / p.sum()
                spread[b, i, h] = p @ np.abs(vv) / p.sum()
                lse[b, i, h] = top + math.log(p.sum())
                bound[b, i, h] = (np.abs(kk) @ np.abs(qf[b, i, h])).max() * scale
    return out, lse, spread, bound


def commit(pool, Hkv, D, accepted, accepted_lens, ctx, table, nodes):
    """In place; returns the new lengths."""
    new = np.array(ctx, dtype=np.int32)
    for b in range(len(ctx)):
        c, m = int(ctx[b]), max(0, min(int(accepted_lens[b]), nodes))
        if c < 0:
            continue
        new[b] = c + m
        if m == 0:
            continue
        k, v = gather_logical(pool, Hkv, PAGE, D, table[b], c, c + int(max(accepted[b, :m])) + 1)
        pick = np.asarray(accepted[b, :m], dtype=np.int64)
        for i in range(m):
            _put_row(pool, Hkv, D, int(table[b, (c + i) // PAGE]), (c + i) % PAGE, k[pick[i]], v[pick[i]])
    return new


def _put_row(pool, Hkv, D, page, slot, k, v):
    d = np.arange(D)
    at = ((d // 8) ^ (slot & 7)) * 8 + d % 8
    for g in range(Hkv):
        for kv, x in ((0, k), (1, v)):
            pool[(((page * Hkv + g) * 2 + kv) * PAGE + slot) * D + at] = x[g]


def append_rows(pool, Hkv, D, seq, slots, table, k, v):
    """uint16 k, v [rows, Hkv, D] into slot slots[r] of sequence seq[r] (seq < 0: padding)."""
    for r in range(len(seq)):
        if seq[r] >= 0:
            _put_row(pool, Hkv, D, int(table[seq[r], slots[r] // PAGE]), int(slots[r] % PAGE), k[r], v[r])


def fork(pools, Hkv, D, src, dst, lens, new_pages, table, counts):
    """In place on the pools, the table and the counts."""
    width, parents = table.shape[1], table.copy()
    for f in range(len(src)):
        whole, rest = int(lens[f]) // PAGE, int(lens[f]) % PAGE
        row = np.full(width, -1, dtype=table.dtype)
        row[:whole] = parents[src[f], :whole]
        for p in row[:whole]:
            if p >= 0:
                counts[p] += 1
        if rest:
            row[whole] = new_pages[f]
            counts[new_pages[f]] = 1
            for pool in pools:
                pages = pool.reshape(-1, Hkv * 2, PAGE, D)
                pages[new_pages[f], :, :rest] = pages[parents[src[f], whole], :, :rest]
        table[dst[f]] = row


def release(rows, keep, table, counts):
    for f, r in enumerate(rows):
        first = 0 if keep is None or keep[f] <= 0 else -(-int(keep[f]) // PAGE)
        for i in range(first, table.shape[1]):
            if table[r, i] >= 0:
                counts[table[r, i]] -= 1
            table[r, i] = -1
