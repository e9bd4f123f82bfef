"""Plain NumPy oracle of the streaming attention operators, in 64 bits, from their definitions and row by row.

It shares no code with the GPU path. Tensors are float64 arrays that hold the storage values; a row only ever touches the
keys and values that it sees, so what others hold cannot reach it.
"""
import math

import numpy as np


def angles(pos, freq):
    """angle(t, j) = sum over a of pos[t, a] * freq[a, j]."""
    return np.asarray(pos, np.float64) @ np.asarray(freq, np.float64)


def partners(pairs, adjacent):
    """Index arrays (first, second) of the elements of each pair."""
    j = np.arange(pairs)
    return (2 * j, 2 * j + 1) if adjacent else (j, j + pairs)


def rotate(x, pos, freq, adjacent=False, inverse=False):
    """x: tokens x heads x dim."""
    a = angles(pos, freq)[:, None, :]
    c, s = np.cos(a), np.sin(a) * (-1.0 if inverse else 1.0)
    first, second = partners(freq.shape[1], adjacent)
    y = np.array(x, np.float64)
    u, w = y[..., first].copy(), y[..., second].copy()
    y[..., first] = u * c - w * s
    y[..., second] = w * c + u * s
    return y


def places(page_table, row_start, kv_len, page_size, pages):
    """(row, page, slot) of every new token that has a place in the cache."""
    out = []
    for b in range(len(kv_len)):
        n = int(row_start[b + 1]) - int(row_start[b])
        for i in range(n):
            at = int(kv_len[b]) - n + i
            if at < 0 or at // page_size >= page_table.shape[1]:
                continue
            page = int(page_table[b, at // page_size])
            if 0 <= page < pages:
                out.append((int(row_start[b]) + i, page, at % page_size))
    return out


def append(k_pages, v_pages, k, v, page_table, row_start, kv_len):
    """New pages (pages x heads x page_size x dim) with the tokens' keys and values (tokens x heads x dim) in place."""
    k_pages, v_pages = np.array(k_pages), np.array(v_pages)
    for row, page, slot in places(page_table, row_start, kv_len, k_pages.shape[2], k_pages.shape[0]):
        k_pages[page, :, slot] = k[row]
        v_pages[page, :, slot] = v[row]
    return k_pages, v_pages


def visible(n, length, i, causal, window):
    """range(lo, hi) of the tokens that new token i of n sees in a sequence of `length` tokens."""
    p = length - n + i
    hi = min(p + 1, length) if causal else length
    lo = 0 if window < 0 else max(0, (p if causal else length - n) - window)
    return range(lo, max(lo, hi))


def attend(q, k_pages, v_pages, page_table, row_start, kv_len, causal=True, window=-1, scale=None):
    """(out, lse, bounds): out tokens x heads x dim, lse tokens x heads; bounds holds for each row what an error bound needs: the
    weighted mean of |v|, the largest sum of |q k| * scale, the largest |score| and the number of keys."""
    tokens, heads, dim = q.shape
    kv_heads, page_size = k_pages.shape[1], k_pages.shape[2]
    scale = dim ** -0.5 if scale is None else scale
    out = np.zeros((tokens, heads, dim))
    lse = np.full((tokens, heads), -math.inf)
    weight = np.zeros((tokens, heads, dim))
    size, most, count = np.zeros((tokens, heads)), np.zeros((tokens, heads)), np.zeros((tokens, heads))
    for b in range(len(kv_len)):
        n, length = int(row_start[b + 1]) - int(row_start[b]), int(kv_len[b])
        for i in range(n):
            seen = np.array(visible(n, length, i, causal, window), np.int64)
            if seen.size == 0:
                continue
            page, slot, row = page_table[b, seen // page_size], seen % page_size, int(row_start[b]) + i
            for h in range(heads):
                keys = k_pages[page, h // (heads // kv_heads), slot]
                values = v_pages[page, h // (heads // kv_heads), slot]
                s = scale * (keys @ q[row, h])
                m = s.max()
                e = np.exp(s - m)
                out[row, h] = e @ values / e.sum()
                lse[row, h] = m + math.log(e.sum())
                with np.errstate(invalid="ignore"):
                    weight[row, h] = e @ np.abs(values) / e.sum()
                    size[row, h] = scale * (np.abs(keys) @ np.abs(q[row, h])).max()
                    most[row, h] = np.abs(s).max()
                count[row, h] = seen.size
    return out, lse, {"weight": weight, "size": size, "most": most, "count": count}
