"""Sequences of unlike lengths in one paged cache, one layer: prompts, single tokens, and trees of drafted tokens that are checked at once.

    prompts        x W  ->  sdllm_append_paged (queries turned, keys and values to the pages)  ->  sdllm_window_attn_paged
    a token each   the same calls with one row; a HIP graph replays them, as lengths are read on the device
    a drafted tree x W  ->  sdllm_qk_norm_rope (positions by depth)  ->  sdllm_tree_attn_paged
    what is kept   sdllm_append_paged with `pick`: the rows of the accepted path, already turned, to the pages

    python -m examples.paged_serving [--prompts 4096,700,1500 --q-heads 28 --kv-heads 4 --window 1023 --sinks 4 --tokens 32 --tree 32]

prints the pages in use and the time of a token step, eager and replayed, and of checking a tree.
"""
from __future__ import annotations

import argparse

import torch

from paper_2508_02558_amd import binding as B

DEV = "cuda"


class PagedLayer:
    """Projection and norm weights of one attention layer, random, and its pages for `batch` sequences of up to `room` rows."""

    def __init__(self, batch, room, hidden, q_heads, kv_heads, head_dim=128, page_rows=64, window=-1, sinks=0, base=1e6, seed=0, dtype=torch.bfloat16):
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        rn = lambda *s: torch.randn(*s, generator=g, device=DEV)
        self.batch, self.q_heads, self.kv_heads, self.head_dim, self.page_rows = batch, q_heads, kv_heads, head_dim, page_rows
        self.window, self.sinks, self.dtype = window, sinks, dtype
        self.w_qkv = (rn(hidden, (q_heads + 2 * kv_heads) * head_dim) * hidden ** -0.5).to(dtype)
        self.q_norm, self.k_norm = ((1 + 0.1 * rn(head_dim)).to(dtype) for _ in range(2))
        half = torch.arange(0, head_dim, 2, device=DEV, dtype=torch.float64)
        self.inv_freq = (base ** (-half / head_dim)).float()
        self.width = -(-room // page_rows)
        self.n_pages = batch * self.width
        self.k_pages, self.v_pages = (torch.zeros(self.n_pages, kv_heads, page_rows, head_dim, dtype=dtype, device=DEV) for _ in range(2))
        self.table = torch.full((batch, self.width), -1, dtype=torch.int32, device=DEV)
        self.free = torch.randperm(self.n_pages, generator=g, device=DEV).tolist()
        self.rows = [0] * batch                                   # the lengths as the host knows them: it hands out the pages
        self.held = [0] * batch
        self.lengths = torch.zeros(batch, dtype=torch.int32, device=DEV)
        self.workspace = {}

    def reserve(self, counts):
        """Pages for `counts` more rows of the sequences."""
        for b, count in enumerate(counts):
            while self.held[b] * self.page_rows < self.rows[b] + count:
                self.table[b, self.held[b]] = self.free.pop()
                self.held[b] += 1

    def grow(self, counts):
        self.rows = [r + c for r, c in zip(self.rows, counts)]
        self.lengths += torch.tensor(counts, dtype=torch.int32, device=DEV)

    def _shapes(self, n, strides, *, norm=True, q_heads=None):
        code = B.SDLLM_BF16 if self.dtype == torch.bfloat16 else B.SDLLM_F32
        more = dict(batch=self.batch, n_kv_heads=self.kv_heads, head_dim=self.head_dim, rows=n, dtype=code)
        qk = B.make_qk_shape(n_q_heads=self.q_heads if q_heads is None else q_heads, q_in_stride=strides, k_in_stride=strides, pos_stride=n,
                             norm=B.SDLLM_NORM_RMS if norm else B.SDLLM_NORM_NONE, rot_dim=None if norm else 0, **more)
        shape = B.make_paged_shape(n_q_heads=self.q_heads, n_pages=self.n_pages, page_rows=self.page_rows, table_pages=self.width, window_left=self.window,
                                   sinks=self.sinks, blk_stride=strides, **more)
        return qk, shape

    def _ws(self, shape, op):
        key = (op, shape.rows)
        if key not in self.workspace:
            self.workspace[key] = torch.empty(B.sdllm_paged_workspace_bytes(shape, op), dtype=torch.uint8, device=DEV)
        return self.workspace[key]

    def _project(self, x):
        batch, n, _ = x.shape
        hq, hkv, d = self.q_heads, self.kv_heads, self.head_dim
        p = (x @ self.w_qkv).view(batch, n, hq + 2 * hkv, d).permute(0, 2, 1, 3)
        return p, p[:, :hq], p[:, hq:hq + hkv], p[:, hq + hkv:]

    def extend(self, x, counts=None, out=None):
        """Outputs [B, Hq, n, d] of the new rows x [B, n, hidden], which go to the pages; counts: how many of them each sequence has (device)."""
        n = x.shape[1]
        p, q, k, v = self._project(x)
        qk, shape = self._shapes(n, B.strides_of(p))
        turned = torch.empty(self.batch, self.q_heads, n, self.head_dim, dtype=self.dtype, device=DEV)
        out = torch.zeros_like(turned) if out is None else out
        B.sdllm_append_paged(qk, shape, q, k, v, self.q_norm, self.k_norm, self.inv_freq, None, None, self.lengths, counts, self.table, turned, self.k_pages,
                             self.v_pages)
        B.sdllm_window_attn_paged(shape, turned, self.k_pages, self.v_pages, self.table, self.lengths, counts, out, self._ws(shape, B.SDLLM_OP_WINDOW_ATTN_PAGED))
        return out

    def check_tree(self, x, depth, mask):
        """Outputs of drafted rows x [B, n, hidden] at depths [B, n] behind the cache, each seeing the cache and the rows in mask [B, n]; and their turned keys
        and their values, for keep()."""
        n = x.shape[1]
        p, q, k, v = self._project(x)
        st = B.strides_of(p)
        qk, shape = self._shapes(n, st)
        qk.q_out_stride[:] = qk.k_out_stride[:] = st
        B.sdllm_qk_norm_rope(qk, q, k, self.q_norm, self.k_norm, self.inv_freq, (self.lengths[:, None] + depth).int(), q, k)     # in place
        out = torch.empty(self.batch, self.q_heads, n, self.head_dim, dtype=self.dtype, device=DEV)
        shape.q_stride[:] = st
        B.sdllm_tree_attn_paged(shape, q, self.k_pages, self.v_pages, self.table, self.lengths, None, k, v, mask, out, self._ws(shape, B.SDLLM_OP_TREE_ATTN_PAGED))
        return out, k, v

    def keep(self, k, v, pick, counts):
        """Appends rows pick[b, :counts[b]] of a checked tree."""
        qk, shape = self._shapes(k.shape[2], B.strides_of(k), norm=False, q_heads=0)
        B.sdllm_append_paged(qk, shape, None, k, v, None, None, None, None, pick, self.lengths, counts, self.table, None, self.k_pages, self.v_pages)


def random_tree(batch, n, seed=0):
    """Depths and masks [B, n] of trees whose rows' parents come before them."""
    g = torch.Generator().manual_seed(seed)
    depth, mask = torch.zeros(batch, n, dtype=torch.int64), torch.zeros(batch, n, dtype=torch.int64)
    for i in range(n):
        parent = torch.randint(-1, i, (batch,), generator=g) if i else torch.full((batch,), -1)
        at = parent.clamp(min=0)[:, None]
        has = parent >= 0
        depth[:, i] = torch.where(has, depth.gather(1, at)[:, 0] + 1, 0)
        mask[:, i] = torch.where(has, mask.gather(1, at)[:, 0], 0) | (1 << i if i < 63 else -1 << 63)
    return depth.to(DEV), mask.to(DEV)


def _time_us(call, n=100):
    for _ in range(10):
        call()
    a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    a.record()
    for _ in range(n):
        call()
    b.record()
    torch.cuda.synchronize()
    return a.elapsed_time(b) * 1e3 / n


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--prompts", default="4096,700,1500")
    for name, default in (("hidden", 2048), ("q-heads", 28), ("kv-heads", 4), ("page-rows", 64), ("window", -1), ("sinks", 0), ("tokens", 32), ("tree", 32)):
        ap.add_argument("--" + name, type=int, default=default)
    a = ap.parse_args()
    prompts = [int(x) for x in a.prompts.split(",")]
    if min(prompts) < 1:
        ap.error("--prompts: every sequence has one token at least")
    if not 1 <= a.tree <= 64:
        ap.error("--tree: a tree has 1 to 64 rows")
    if a.tokens < 1:
        ap.error("--tokens: one at least")
    batch, room = len(prompts), max(prompts) + a.tokens + a.tree
    layer = PagedLayer(batch, room, a.hidden, a.q_heads, a.kv_heads, page_rows=a.page_rows, window=a.window, sinks=a.sinks)
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    rows = lambda n: torch.randn(batch, n, a.hidden, generator=g, device=DEV).bfloat16()
    layer.reserve(prompts)
    layer.extend(rows(max(prompts)), torch.tensor(prompts, dtype=torch.int32, device=DEV))
    layer.grow(prompts)

    x, one = rows(1), [1] * batch
    out = torch.zeros(batch, a.q_heads, 1, layer.head_dim, dtype=layer.dtype, device=DEV)
    layer.reserve([a.tokens + a.tree] * batch)
    layer.extend(x, out=out)
    eager = _time_us(lambda: layer.extend(x, out=out))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.extend(x, out=out)
    for _ in range(a.tokens):
        x.copy_(rows(1))
        graph.replay()
        layer.grow(one)
    print(f"{sum(layer.held)} pages of {a.page_rows} rows, lengths {layer.rows}")
    print(f"a token of each sequence: {eager:7.2f} us, replayed {_time_us(graph.replay):7.2f} us (with the projection)")

    depth, mask = random_tree(batch, a.tree)
    tree = rows(a.tree)
    _, k, v = layer.check_tree(tree, depth, mask)
    pick = torch.zeros(batch, a.tree, dtype=torch.int32, device=DEV)   # the path to the last row
    counts = []
    for b, m in enumerate(mask[:, -1].tolist()):
        path = [i for i in range(a.tree) if m >> i & 1]
        pick[b, :len(path)] = torch.tensor(path, dtype=torch.int32)
        counts.append(len(path))
    layer.keep(k, v, pick, torch.tensor(counts, dtype=torch.int32, device=DEV))
    print(f"a tree of {a.tree} rows for each: {_time_us(lambda: layer.check_tree(tree, depth, mask)):7.2f} us, {counts} rows kept")


if __name__ == "__main__":
    main()
