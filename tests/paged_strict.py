"""Results of the paged cache's attentions that are no numbers, one by one: what tests/paged_util.py's bounds leave open where a bound is itself infinite."""
import numpy as np
import torch

from oracle import paged_oracle as pg
from tests.paged_util import host

KINDS = {"nan": [float("nan")], "inf": [float("inf"), float("-inf")]}


def same_classes(got, want):
    """Finite where the other is, infinities of the same sign, NaN where the other is."""
    mark = lambda x: np.where(np.isfinite(x), 0.0, x)
    return np.array_equal(mark(got), mark(want), equal_nan=True)


def wanted(c):
    """(sequence, head, result, oracle's result) of a tests.paged_util.Paged that has been run."""
    torch.cuda.synchronize()
    got, q, kb, vb, kp, vp = (host(x) for x in (c.out, c.q, c.k_blk, c.v_blk, c.k_pages, c.v_pages))
    table = c.table.cpu().numpy()
    for b, (length, count) in enumerate(zip(c.host_lengths, c.host_counts)):
        rows = lambda x, n: pg.rows_of(x, table[b], n, c.page_rows)
        if c.kind == "tree":
            k, v = (np.concatenate([rows(x, length), y[b, :, :count]], 1) for x, y in ((kp, kb), (vp, vb)))
            seen = pg.seen_tree(length, count, None if c.host_mask is None else [x & (1 << 64) - 1 for x in c.host_mask[b]])
        else:
            k, v, seen = rows(kp, length + count), rows(vp, length + count), pg.seen_window(length, count, *c.window)
        for h in range(c.Hq):
            g = h // (c.Hq // c.Hkv)
            yield b, h, got[b, h, :count], pg.attention(q[b, h, :count], k[g], v[g], seen, c.scale)[0]


def check_strictly(c):
    c.check()
    some = False
    for b, h, got, want in wanted(c):
        assert same_classes(got, want), (b, h, np.argwhere(~np.isclose(got, want, rtol=1, atol=1, equal_nan=True))[:4].tolist())
        some |= not np.isfinite(want).all()
    assert some, "nothing that is no number is seen"


def one_a_tile(kinds):
    """An edit of Paged: in every 32-row tile of every sequence one value of V, in a channel of the tile's own."""
    def edit(k_pages, v_pages, c):
        d = v_pages.shape[3]
        for b, (length, count) in enumerate(zip(c.host_lengths, c.host_counts)):
            cached = length + (count if c.kind == "window" else 0)
            for t in range(-(-cached // 32)):
                j = min(32 * t + (7 * t + 3) % 32, cached - 1)
                v_pages[int(c.table[b, j // c.page_rows]), t % c.Hkv, j % c.page_rows, t % d] = kinds[t % len(kinds)]
            if c.kind == "tree":
                for j in range(0, count, 5):
                    c.v_blk[b, j % c.Hkv, j, d - 1 - j // 5] = kinds[j % len(kinds)]
    return edit
