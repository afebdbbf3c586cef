"""The paged cache from its definitions, in float64 (NumPy): where rows lie, what a row sees, and attention over what it sees.  Written from
include/sdllm.h; shares no code with the package."""
import numpy as np

from oracle.packed_oracle import norm_rope


def rows_of(pages, table_row, n, page_rows):
    """Rows [0, n) of a sequence as [Hkv, n, d]; pages [P, Hkv, page_rows, d]."""
    out = np.zeros((pages.shape[1], n, pages.shape[3]))
    for j in range(n):
        out[:, j] = pages[min(max(int(table_row[j // page_rows]), 0), len(pages) - 1), :, j % page_rows]
    return out


def seen_window(length, count, left, right, sinks, capacity=None):
    """[count, keys] of rows at places length, length + 1, ... of the cache's length + count keys."""
    end = length + count if capacity is None else min(length + count, capacity)
    seen = np.zeros((count, end), bool)
    for i in range(count):
        p = length + i
        for j in range(end):
            seen[i, j] = (right < 0 or j <= p + right) and (left < 0 or j >= p - left or j < sinks)
    return seen


def seen_tree(length, count, mask):
    """[count, length + count]; mask: count integers, or None."""
    seen = np.ones((count, length + count), bool)
    if mask is not None:
        for i in range(count):
            for j in range(count):
                seen[i, length + j] = int(mask[i]) >> j & 1
    return seen


def attention(q, k, v, seen, scale):
    """(out, mean) of rows q [n, d] over k, v [m, d]: keys that a row does not see are not there for it; a row without keys is zero.  mean: the same
    over |v|, what errors of the probabilities are measured in."""
    out, mean = np.zeros(q.shape), np.zeros(q.shape)
    with np.errstate(invalid="ignore", over="ignore"):
        for i in range(len(q)):
            kk, vv = k[seen[i]], v[seen[i]]
            if len(kk) == 0:
                continue
            a = scale * (kk @ q[i])
            p = np.exp(a - a.max())
            p = p / p.sum()
            out[i], mean[i] = p @ vv, p @ np.abs(vv)
    return out, mean


def append(k_pages, v_pages, k, v, table, lengths, counts, pick, positions, *, page_rows, weight, inv_freq, rot, pairing, norm, eps, pos_begin=0):
    """Pages after the call: new float64 arrays.  k, v [B, Hkv, n, d]."""
    k_pages, v_pages = np.array(k_pages, np.float64), np.array(v_pages, np.float64)
    capacity = table.shape[1] * page_rows if len(k_pages) else 0
    n = k.shape[2]
    for b in range(len(k)):
        length = min(max(int(lengths[b]), 0), capacity)
        for i in range(n if counts is None else min(max(int(counts[b]), 0), n)):
            r = i if pick is None else min(max(int(pick[b][i]), 0), n - 1)
            place = length + i
            if place >= capacity or not 0 <= table[b][place // page_rows] < len(k_pages):
                continue
            at = place + pos_begin if positions is None else int(positions[b][r])
            page, row = int(table[b][place // page_rows]), place % page_rows
            k_pages[page, :, row] = norm_rope(k[b][:, r:r + 1], weight, inv_freq, np.array([[at]]), rot=rot, pairing=pairing, norm=norm, eps=eps)[:, 0]
            v_pages[page, :, row] = v[b][:, r]
    return k_pages, v_pages
