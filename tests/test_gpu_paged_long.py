"""Attention over the paged cache where a wavefront, or a workgroup whose waves share tiles, goes over more than the 64 tiles whose places are looked up at once."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as pg
from paper_2508_02558_amd import binding as B
from tests.paged_util import DEV, TYPES, host, ints, tolerance, tree_masks

pytestmark = pytest.mark.gpu


def run(kind, Hq, Hkv, d, n, length, dtype, form, tiles_at_once, page_rows=16, window=(-1, 0, 0), checked=3):
    """One sequence.  All KV heads read the same rows (a head stride of 0); `tiles_at_once`: tiles that one look-up's owner goes over together with the others of
    its workgroup, which are as many as its wavefronts in the streaming form.  Nothing is cut, so that a workgroup has all of an item's tiles."""
    td, code = TYPES[dtype]
    g = torch.Generator().manual_seed(length + n)
    total = length + (n if kind == "window" else 0)
    width = -(-total // page_rows)
    n_pages = width + 3
    table = torch.randperm(n_pages, generator=g)[:width].int()[None]
    k1, v1 = (torch.randn(n_pages, 1, page_rows, d, generator=g).to(td).to(DEV) for _ in range(2))
    q = torch.randn(1, Hq, n, d, generator=g).to(td).to(DEV)
    kb1, vb1 = (torch.randn(1, 1, n, d, generator=g).to(td).to(DEV) for _ in range(2))
    wide = lambda x: x.expand(-1, Hkv, -1, -1)
    out = torch.full_like(q, float("nan"))
    masks = tree_masks(1, n, 4) if kind == "tree" else None
    scale = 0.4                                          # a few keys take most of it, wherever they are
    left, right, sinks = window
    s = B.make_paged_shape(batch=1, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=d, rows=n, dtype=code, n_pages=n_pages, page_rows=page_rows, table_pages=width,
                           window_left=left, window_right=right, sinks=sinks, softmax_scale=scale, page_stride=B.strides_of(wide(k1)), blk_stride=B.strides_of(wide(kb1)))
    op = B.SDLLM_OP_TREE_ATTN_PAGED if kind == "tree" else B.SDLLM_OP_WINDOW_ATTN_PAGED
    p = B.sdllm_paged_plan(s, op)
    assert (p.shared, p.block_cols, p.waves, p.least_tiles) == form + (0,)
    assert length // 32 > 64 * tiles_at_once
    ws = torch.empty(B.sdllm_paged_workspace_bytes(s, op), dtype=torch.uint8, device=DEV)
    if kind == "tree":
        mask = torch.tensor(masks, dtype=torch.int64, device=DEV)
        B.sdllm_tree_attn_paged(s, q, k1, v1, table.to(DEV), ints([length]), None, kb1, vb1, mask, out, ws)
    else:
        B.sdllm_window_attn_paged(s, q, k1, v1, table.to(DEV), ints([length]), None, out, ws)
    torch.cuda.synchronize()
    assert out.isfinite().all()
    k, v = (pg.rows_of(host(x), table[0].tolist(), total, page_rows)[0] for x in (k1, v1))
    if kind == "tree":
        k, v = np.concatenate([k, host(kb1)[0, 0]]), np.concatenate([v, host(vb1)[0, 0]])
        seen = pg.seen_tree(length, n, [x & (1 << 64) - 1 for x in masks[0]])
    else:
        at, key = length + np.arange(n)[:, None], np.arange(total)
        seen = (key <= at + right) if right >= 0 else np.ones((n, total), bool)
        if left >= 0:
            seen = seen & ((key >= at - left) | (key < sinks))
    rows = sorted({0, 1, n // 3, n // 2, n - 2, n - 1} & set(range(n)))
    for h in sorted({0, Hq // 2, Hq - 1}):
        x = host(q[0, h])[rows]
        want, mean = pg.attention(x, k, v, seen[rows], scale)
        err, tol = np.abs(host(out[0, h])[rows] - want), tolerance(x, k, mean, want, scale, v, dtype)
        assert (err <= tol).all(), (h, float((err / tol).max()))


# Tiles a step: 256 columns one of head_dim 128 and two of 64, 128 columns two and four.  The last block's tiles are a multiple of 64, or one more, or one less.
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("length", [64 * 32 * 2 - 2110, 64 * 32 * 2 - 2110 + 1, 64 * 32 * 3 - 2110 - 40, 64 * 32 * 2 - 2110 + 97])
def test_prompts_of_256_columns(d, length):
    run("window", 16, 4, d, 2110, length + 2048, "bf16", (1, 256, 8), 1)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("window", [(-1, -1, 0), (2500, 0, 100)])
def test_windows_of_256_columns(d, window):
    run("window", 16, 4, d, 2110, 2300, "bf16", (1, 256, 8), 1, page_rows=32, window=window)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("end", [64 * 32 * 2, 64 * 32 * 2 + 1, 64 * 32 * 3 - 33])
@pytest.mark.parametrize("kind", ["window", "tree"])
def test_128_columns(d, end, kind):
    run(kind, 2 * 129, 129, d, 40, end - 40, "bf16", (1, 128, 8), 1)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kind,group,n,cols", [("window", 1, 1, 16), ("tree", 1, 1, 16), ("window", 6, 4, 32), ("tree", 3, 8, 32)])
def test_streaming(d, kind, group, n, cols):
    run(kind, group * 1025, 1025, d, n, 64 * 32 * 4 + 100, "bf16", (0, cols, 4), 4)


@pytest.mark.parametrize("d,waves", [(64, 8), (128, 4)])
@pytest.mark.parametrize("kind", ["window", "tree"])
def test_streaming_fp32(d, waves, kind):
    run(kind, 2 * 513, 513, d, 2, 64 * 32 * waves + 100, "f32", (0, 16, waves), waves, page_rows=32)
