"""Plain NumPy oracle of the cache in 4 bits, of accumulated attention weight and of eviction, from their definitions.

It shares no code with the GPU path. A cache in 4 bits is (codes, scales): uint8 ... x 16 * groups, float16 ... x groups x 2.
"""
import numpy as np

from .stream_attention_oracle import visible

GROUP, MOST = 32, np.float32(32768.0)


def pack(x):
    """(codes, scales) of float32 elements, ... x dim, group by group. Every step rounds as the format says."""
    x = np.asarray(x, np.float32)
    dim = x.shape[-1]
    groups = -(-dim // GROUP)
    codes = np.zeros(x.shape[:-1] + (16 * groups,), np.uint8)
    scales = np.zeros(x.shape[:-1] + (groups, 2), np.float16)
    for g in range(groups):
        part = x[..., g * GROUP:(g + 1) * GROUP]
        fine = np.isfinite(part).all(-1)
        y = np.where(fine[..., None], np.clip(part, -MOST, MOST), np.float32(0))
        low = y.min(-1).astype(np.float16)
        scale = np.maximum((y.max(-1) - low.astype(np.float32)) / np.float32(15), np.float32(0)).astype(np.float16)
        with np.errstate(divide="ignore", invalid="ignore"):
            c = np.rint((y - low.astype(np.float32)[..., None]) / scale.astype(np.float32)[..., None])
        c = np.where((scale > 0)[..., None], np.clip(c, 0, 15), 0).astype(np.uint8)
        for e in range(c.shape[-1]):
            codes[..., 16 * g + e // 2] |= (c[..., e] << (4 * (e % 2))).astype(np.uint8)
        scales[..., g, 0] = np.where(fine, scale, np.float16("nan"))
        scales[..., g, 1] = np.where(fine, low, np.float16("nan"))
    return codes, scales


def values(codes, scales, dim):
    """What codes stand for, as float64: minimum + code * scale is exact in 64 bits, and rounded once to fp16."""
    out = np.zeros(codes.shape[:-1] + (dim,))
    with np.errstate(over="ignore", invalid="ignore"):
        for e in range(dim):
            c = (codes[..., e // 2] >> (4 * (e % 2))) & 15
            pair = scales[..., e // GROUP, :].astype(np.float64)
            out[..., e] = (pair[..., 1] + c * pair[..., 0]).astype(np.float16)
    return out


def weigh(weights, q, lse, k_pages, page_table, row_start, kv_len, causal=True, window=-1, scale=None, decay=1.0):
    """(weights, size): the new weights (pages x kv_heads x page_size), and for each the sum over its rows of what a term's error is relative to:
    (term, term * largest sum of |q k| * scale, term * (|score| + |lse|))."""
    tokens, heads, dim = q.shape
    pages, kv_heads, page_size = k_pages.shape[:3]
    group, scale = heads // kv_heads, dim ** -0.5 if scale is None else scale
    out, size = np.array(weights, np.float64), np.zeros(weights.shape + (3,))
    for b in range(len(kv_len)):
        n, length = int(row_start[b + 1]) - int(row_start[b]), int(kv_len[b])
        if n == 0:
            continue
        got = np.zeros((kv_heads, length))
        much = np.zeros((kv_heads, length, 3))
        at = np.arange(length)
        page, slot = page_table[b, at // page_size], at % page_size
        for i in range(n):
            seen = np.array(visible(n, length, i, causal, window), np.int64)
            for h in range(heads if seen.size else 0):
                l = lse[int(row_start[b]) + i, h]  # noqa: E741
                if np.isneginf(l):
                    continue
                keys, row = k_pages[page[seen], h // group, slot[seen]], q[int(row_start[b]) + i, h]
                s = scale * (keys @ row)
                e = np.exp(s - l)
                got[h // group, seen] += e
                much[h // group, seen] += np.stack([e, e * scale * (np.abs(keys) @ np.abs(row)), e * (np.abs(s) + abs(l))], -1)
        for j in range(length):
            if 0 <= page[j] < pages:
                old = 0.0 if j >= length - n else decay * out[page[j], :, slot[j]]
                out[page[j], :, slot[j]] = old + got[:, j]
                size[page[j], :, slot[j]] = much[:, j]
    return out, size


def evict(weights, page_table, kv_len, keep, recent):
    """(lengths, kept): kept is sequences x kv_heads x keep."""
    pages, kv_heads, page_size = weights.shape
    kept = np.full((len(kv_len), kv_heads, keep), -1, np.int32)
    lengths = np.minimum(np.asarray(kv_len), keep).astype(np.int32)
    for b in range(len(kv_len)):
        length, n = int(kv_len[b]), int(lengths[b])
        late = length - min(n, recent)
        for h in range(kv_heads):
            def rank(j):
                page = page_table[b, j // page_size]
                if not 0 <= page < pages:
                    return (2, 0.0, j)
                w = float(weights[page, h, j % page_size])
                return (0, 0.0, j) if np.isnan(w) else (1, -w, j)
            chosen = list(range(late, length)) + sorted(range(late), key=rank)[:n - (length - late)]
            kept[b, h, :n] = sorted(chosen)
    return lengths, kept


def move(rows, page_table, into, kept, page_size, pages):
    """New pages (pages x kv_heads x page_size x ...) with the kept tokens' rows at their new places."""
    out = np.array(rows)
    for b, h, i in zip(*np.nonzero(kept >= 0)):
        j = kept[b, h, i]
        at, to = page_table[b, j // page_size], into[b, i // page_size]
        if 0 <= at < pages and 0 <= to < pages:
            out[to, h, i % page_size] = rows[at, h, j % page_size]
    return out
