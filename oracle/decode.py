"""Plain 64-bit forms of the decoding operators -- TEST INFRASTRUCTURE ONLY.

Straight from the definitions in ``include/asd.h``, in numpy float64, one row, head and token at a
time; they share no code with the HIP path.  Parity unpinned: the paper has no such operators,
so the tests pin these against hand-made cases and, on the GPU, against the kernels.
"""
import numpy as np


def requests(block_lens, row_offsets, cache_lens, total_rows, room):
    """(first row, rows, cached tokens) of every request, None for one that is skipped."""
    out, at = [], 0
    for i, k in enumerate(block_lens):
        count = max(int(k), 0) + 1
        first = at if row_offsets is None else int(row_offsets[i])
        at += count
        cached = int(cache_lens[i])
        ok = 0 <= first <= total_rows - count and 0 <= cached <= room - count
        out.append((first, count, cached) if ok else None)
    return out


def slot(page_table, num_pages, page_size, i, token):
    """(page, place) of a token, or None where the page id is outside the cache."""
    page = int(page_table[i, token // page_size])
    return (page, token % page_size) if 0 <= page < num_pages else None


def rope(x, weight, eps, position, inv_freq, interleaved):
    """One head, normed and turned: (result, bound): |n_a| + |n_b| of each element's pair."""
    n = x.astype(np.float64)
    if weight is not None:
        n = n / np.sqrt(np.mean(n * n) + eps) * weight.astype(np.float64)
    y, size = n.copy(), np.abs(n)
    half = len(inv_freq)
    j = np.arange(half)
    a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + half)
    angle = float(position) * inv_freq.astype(np.float64)
    y[a] = n[a] * np.cos(angle) - n[b] * np.sin(angle)
    y[b] = n[a] * np.sin(angle) + n[b] * np.cos(angle)
    size[a] = size[b] = np.abs(n[a]) + np.abs(n[b])
    return y, size


def rope_append(q, k, v, k_cache, v_cache, page_table, cache_lens, block_lens, inv_freq,
                q_norm=None, k_norm=None, eps=1e-6, positions=None, interleaved=False,
                row_offsets=None):
    """float64 (q_out, k_cache, v_cache) and the bounds of q_out and k_cache; NaN in q_out where
    nothing is written, the caches as they were where nothing is written."""
    rows = k.shape[0]
    pages, size = k_cache.shape[:2]
    keys, values = k_cache.astype(np.float64), v_cache.astype(np.float64)
    out = None if q is None else np.full(q.shape, np.nan)
    out_size = None if q is None else np.zeros(q.shape)
    key_size = np.zeros(keys.shape)
    freq = np.zeros(0) if inv_freq is None else inv_freq
    for i, r in enumerate(requests(block_lens, row_offsets, cache_lens, rows,
                                   page_table.shape[1] * size)):
        if r is None:
            continue
        first, count, cached = r
        for p in range(count):
            row = first + p
            pos = cached + p if positions is None else positions[row]
            if q is not None:
                for h in range(q.shape[1]):
                    out[row, h], out_size[row, h] = rope(q[row, h], q_norm, eps, pos, freq, interleaved)
            at = slot(page_table, pages, size, i, cached + p)
            if at is not None:
                for h in range(k.shape[1]):
                    keys[at][h], key_size[at][h] = rope(k[row, h], k_norm, eps, pos, freq, interleaved)
                    values[at][h] = v[row, h]
    return out, keys, values, out_size, key_size


def block_attention(q, k_cache, v_cache, page_table, cache_lens, block_lens, scale, mask=None,
                    row_offsets=None):
    """float64 (out, weighted |V| of every element, sum |q k| of every row and head); NaN in out
    where nothing is written."""
    rows, heads, dim = q.shape
    pages, size, kv_heads = k_cache.shape[:3]
    out = np.full(q.shape, np.nan)
    mean = np.zeros(q.shape)
    reach = np.zeros((rows, heads))
    for i, r in enumerate(requests(block_lens, row_offsets, cache_lens, rows,
                                   page_table.shape[1] * size)):
        if r is None:
            continue
        first, count, cached = r
        token = np.arange(cached + count)
        page = page_table[i, token // size].astype(np.int64)
        good = (page >= 0) & (page < pages)
        page = np.where(good, page, 0)
        for p in range(count):
            row = first + p
            seen = good.copy()
            for j in range(count):
                if mask is None:
                    visible = j <= p
                else:
                    visible = j < 64 * mask.shape[1] and (int(mask[row, j // 64]) >> (j % 64)) & 1
                seen[cached + j] &= bool(visible)
            at = np.flatnonzero(seen)
            for h in range(heads):
                g = h // (heads // kv_heads)
                if at.size == 0:
                    out[row, h] = 0.0
                    continue
                keys = k_cache[page[at], at % size, g].astype(np.float64)
                values = v_cache[page[at], at % size, g].astype(np.float64)
                x = q[row, h].astype(np.float64)
                with np.errstate(invalid="ignore", over="ignore"):
                    s = scale * (keys @ x)
                    w = np.exp(s - s.max())
                    w /= w.sum()
                    out[row, h] = w @ values
                    mean[row, h] = w @ np.abs(values)
                    reach[row, h] = abs(scale) * (np.abs(keys) @ np.abs(x)).max()
    return out, mean, reach


def sample_row(z, u, t=1.0, k=0, p=1.0, m=0.0):
    """(token, probability) of one row."""
    z = z.astype(np.float64)
    if np.isnan(z).any() or z.max() == -np.inf:
        return -1, 0.0
    if not t > 0:
        return int(np.argmax(z)), 1.0
    top = z.max()
    with np.errstate(invalid="ignore"):
        x = np.where(z == top, 0.0, np.where(np.isinf(z) | np.isinf(top), -np.inf, z - top))
        w = np.where(x == -np.inf, 0.0, np.exp(np.where(x == -np.inf, 0.0, x) / t))
    order = np.lexsort((np.arange(z.size), -z))          # greatest first, then the lowest index
    ranked = w[order]
    n = z.size if k <= 0 else min(int(k), z.size)
    if p < 1:
        run = np.cumsum(ranked[:n])
        n = max(1, int(np.searchsorted(run, p * run[-1], side="left")) + 1)
    if m > 0:
        n = min(n, int(np.sum(ranked >= min(m, 1.0))))
    kept = np.zeros_like(w)
    kept[order[:n]] = ranked[:n]
    run = np.cumsum(kept)
    u = 0.0 if np.isnan(u) else min(max(float(u), 0.0), 1 - 2.0 ** -24)
    token = int(np.searchsorted(run, u * run[-1], side="right"))
    return token, kept[token] / run[-1]
