"""Calls of the paged cache's attentions with everything they read, and the comparison with the float64 oracle."""
import numpy as np
import torch

from oracle import paged_oracle as pg
from paper_2508_02558_amd import binding as B

DEV = "cuda"
TYPES = {"bf16": (torch.bfloat16, B.SDLLM_BF16), "f32": (torch.float32, B.SDLLM_F32)}


def host(t):
    return t.detach().cpu().double().numpy()


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def tolerance(q, k, mean, want, scale, v, dtype):
    """Of attention over m keys with products, sums and exponentials in fp32 (u = 2^-24).  A logit is a sum of d products and a multiple of log2(e); a
    probability is off by as much, relatively, and by the exponential's two steps; sums over keys and the merge add half a step a term.  No result or
    numerator below the smallest normal number can be held.  bf16: half a step, 2^-8 relative, for the numerators and for the result."""
    u, d, m = 2.0 ** -24, q.shape[-1], max(1, len(k))
    logit = (np.abs(q) @ np.abs(k).T).max(-1, keepdims=True) * scale if len(k) else np.zeros((len(q), 1))
    p = (d + 8) * u * logit + 4 * u
    tol = (2 * p + (m + 16) * 2 * u) * mean + u * np.abs(want) + m * (np.abs(v).max() if len(v) else 0) * 2.0 ** -126
    if dtype == "bf16":
        tol = tol + 2.0 ** -8 * mean + 2.0 ** -8 * np.abs(want)
    return tol


class Paged:
    """A pool with sequences in it.  Rows that no sequence has hold NaN, as does all of the output before a call."""

    def __init__(self, kind, Hq, Hkv, d, n, lengths, dtype, counts=None, page_rows=32, layout="heads", seed=0, spare=2, mask=None, edit=None, scale=0.0,
                 left=-1, right=0, sinks=0, table_pages=None):
        td, code = TYPES[dtype]
        g = torch.Generator().manual_seed(seed + 7 * sum(lengths) + n)
        self.kind, self.dtype, self.n, self.Hq, self.Hkv = kind, dtype, n, Hq, Hkv
        self.host_lengths, self.host_counts = list(lengths), [n] * len(lengths) if counts is None else list(counts)
        self.window, self.page_rows = (left, right, sinks), page_rows
        Bt = len(lengths)
        kept = [length + (c if kind == "window" else 0) for length, c in zip(lengths, self.host_counts)]
        needed = [-(-x // page_rows) for x in kept]
        n_pages = sum(needed) + spare
        width = (max(needed) if needed else 0) + 1 if table_pages is None else table_pages
        self.table = torch.full((Bt, width), -7, dtype=torch.int32)
        free = torch.randperm(n_pages, generator=g)[:sum(needed)].tolist()
        pool = lambda: torch.full((n_pages, Hkv, page_rows, d), float("nan"))
        k_pages, v_pages = pool(), pool()
        for b, pages in enumerate(needed):
            for i in range(pages):
                page = free.pop()
                self.table[b, i] = page
                rows = min(page_rows, kept[b] - i * page_rows)
                for x in (k_pages, v_pages):
                    x[page, :, :rows] = torch.randn(Hkv, rows, d, generator=g)
        make = lambda H: torch.randn(Bt, n, H, d, generator=g).permute(0, 2, 1, 3) if layout == "rows" else torch.randn(Bt, H, n, d, generator=g)
        self.q, self.k_blk, self.v_blk = make(Hq), make(Hkv), make(Hkv)
        for b, c in enumerate(self.host_counts):
            for x in (self.q, self.k_blk, self.v_blk):
                x[b, :, max(0, c):] = float("nan")
        if edit:
            edit(k_pages, v_pages, self)
        laid = lambda x: x.to(td).to(DEV) if layout == "heads" else x.to(td).to(DEV).permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)
        self.k_pages, self.v_pages, self.q, self.k_blk, self.v_blk = (laid(x) for x in (k_pages, v_pages, self.q, self.k_blk, self.v_blk))
        self.out = torch.full_like(self.q, float("nan"))
        self.mask = None if mask is None else torch.tensor(mask, dtype=torch.int64, device=DEV).reshape(Bt, n)
        self.host_mask = mask
        self.table = self.table.to(DEV)
        self.lengths = ints(lengths)
        self.counts = None if counts is None else ints(counts)
        self.scale = scale or d ** -0.5
        self.shape = B.make_paged_shape(batch=Bt, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=d, rows=n, dtype=code, n_pages=n_pages, page_rows=page_rows,
                                        table_pages=width, window_left=left, window_right=right, sinks=sinks, softmax_scale=scale,
                                        q_stride=B.strides_of(self.q), blk_stride=B.strides_of(self.k_blk), out_stride=B.strides_of(self.out),
                                        page_stride=B.strides_of(self.k_pages))
        self.op = B.SDLLM_OP_TREE_ATTN_PAGED if kind == "tree" else B.SDLLM_OP_WINDOW_ATTN_PAGED
        self.ws = torch.empty(B.sdllm_paged_workspace_bytes(self.shape, self.op), dtype=torch.uint8, device=DEV).fill_(0xFF)

    def run(self, stream=None, out=None):
        out = self.out if out is None else out
        if self.kind == "tree":
            B.sdllm_tree_attn_paged(self.shape, self.q, self.k_pages, self.v_pages, self.table, self.lengths, self.counts, self.k_blk, self.v_blk,
                                    self.mask, out, self.ws, stream)
        else:
            B.sdllm_window_attn_paged(self.shape, self.q, self.k_pages, self.v_pages, self.table, self.lengths, self.counts, out, self.ws, stream)

    def check(self, out=None):
        torch.cuda.synchronize()
        got, q, kb, vb = (host(x) for x in (self.out if out is None else out, self.q, self.k_blk, self.v_blk))
        kp, vp, table = host(self.k_pages), host(self.v_pages), self.table.cpu().numpy()
        capacity = table.shape[1] * self.page_rows if len(kp) else 0
        lengths, counts = self.lengths.cpu().tolist(), [self.n] * len(table) if self.counts is None else self.counts.cpu().tolist()
        for b in range(len(table)):
            length, count = min(max(lengths[b], 0), capacity), min(max(counts[b], 0), self.n)
            assert np.isnan(got[b, :, count:]).all(), "rows that are not there were written"
            if self.kind == "tree":
                k, v = (np.concatenate([pg.rows_of(x, table[b], length, self.page_rows), y[b, :, :count]], 1) for x, y in ((kp, kb), (vp, vb)))
                masks = None if self.mask is None else [x & (1 << 64) - 1 for x in self.mask[b].cpu().tolist()]
                seen = pg.seen_tree(length, count, masks)
            else:
                seen = pg.seen_window(length, count, *self.window, capacity)
                # what nobody sees is in no page that has to be there
                needed = np.flatnonzero(seen.any(0))
                k, v = (np.zeros((self.Hkv, seen.shape[1], kp.shape[3])) for _ in range(2))
                for j in needed:
                    page = min(max(int(table[b][j // self.page_rows]), 0), len(kp) - 1)
                    k[:, j], v[:, j] = kp[page, :, j % self.page_rows], vp[page, :, j % self.page_rows]
            for h in range(self.Hq):
                kk, vv = k[h // (self.Hq // self.Hkv)], v[h // (self.Hq // self.Hkv)]
                want, mean = pg.attention(q[b, h, :count], kk, vv, seen, self.scale)
                err = np.abs(got[b, h, :count] - want)
                with np.errstate(invalid="ignore"):
                    seen_by_some = seen.any(0) if count else np.zeros(len(kk), bool)
                    tol = tolerance(q[b, h, :count], np.nan_to_num(kk[seen_by_some], posinf=0, neginf=0), mean, want, self.scale,
                                    np.nan_to_num(vv[seen_by_some], posinf=0, neginf=0), self.dtype)
                same = (np.isnan(want) & np.isnan(got[b, h, :count])) | (np.isinf(want) & (want == got[b, h, :count]))
                ok = same | (err <= tol)
                assert ok.all(), (b, h, np.argwhere(~ok)[:4].tolist(), float(np.nanmax(np.where(same, 0, err / tol))))


def tree_masks(Bt, n, seed):
    """Ancestors of the rows of random trees, a row itself among them."""
    rng = np.random.default_rng(seed)
    out = []
    for _ in range(Bt):
        masks = []
        for i in range(n):
            parent = int(rng.integers(-1, i))if i else -1
            m = (masks[parent] if parent >= 0 else 0) | 1 << i
            masks.append(m)
        out.append([m - (1 << 64) if m >> 63 else m for m in masks])
    return out
