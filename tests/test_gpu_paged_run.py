"""The paged cache's operators together, as a decoder uses them: prompts, tokens, drafted trees; graphs, streams, far offsets; every form of the attentions."""
import numpy as np
import pytest
import torch

from examples import paged_serving as ex
from oracle import packed_oracle as po
from oracle import paged_oracle as pg
from paper_2508_02558_amd import binding as B
from tests.paged_util import DEV, Paged, host, ints, tolerance, tree_masks

pytestmark = pytest.mark.gpu


def oracle_rows(layer, p, at):
    """Turned queries and keys, and values, of projected rows p [heads, n, d] at positions `at`."""
    hq, hkv = layer.q_heads, layer.kv_heads
    turn = lambda h, w: po.norm_rope(h, host(w), host(layer.inv_freq), np.broadcast_to(at, h.shape[:2]), rot=layer.head_dim, pairing=po.HALVES, norm=True, eps=1e-6)
    return turn(p[:hq], layer.q_norm), turn(p[hq:hq + hkv], layer.k_norm), p[hq + hkv:]


@pytest.mark.parametrize("dtype,d,page_rows,window,sinks", [(torch.bfloat16, 128, 16, -1, 0), (torch.bfloat16, 64, 64, 40, 3), (torch.float32, 64, 32, -1, 0),
                                                            (torch.float32, 128, 16, 25, 5)])
def test_prompts_tokens_and_trees(dtype, d, page_rows, window, sinks):
    prompts, hidden, hq, hkv, n = [70, 5, 33], 96, 6, 2, 11
    layer = ex.PagedLayer(3, 160, hidden, hq, hkv, head_dim=d, page_rows=page_rows, window=window, sinks=sinks, dtype=dtype)
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    rows = lambda m: torch.randn(3, m, hidden, generator=g, device=DEV).to(dtype)
    seen, outputs = [[] for _ in prompts], [[] for _ in prompts]

    def extend(x, counts):
        layer.reserve(counts)
        out = layer.extend(x, ints(counts))
        projected = host(layer._project(x)[0])
        for b, c in enumerate(counts):
            seen[b].append(projected[b, :, :c])
            outputs[b].append(out[b, :, :c])
        layer.grow(counts)
    extend(rows(max(prompts)), prompts)
    for _ in range(3):
        extend(rows(1), [1, 1, 1])

    # a tree, and the path to its last row
    depth, mask = ex.random_tree(3, n, 7)
    tree = rows(n)
    before = list(layer.rows)
    tree_out, k, v = layer.check_tree(tree, depth, mask)
    paths = [[i for i in range(n) if m >> i & 1] for m in mask[:, -1].tolist()]
    pick = torch.zeros(3, n, dtype=torch.int32, device=DEV)
    for b, path in enumerate(paths):
        pick[b, :len(path)] = ints(path)
    layer.reserve([len(x) for x in paths])
    layer.keep(k, v, pick, ints([len(x) for x in paths]))
    layer.grow([len(x) for x in paths])
    for b, path in enumerate(paths):
        seen[b].append(host(layer._project(tree)[0])[b][:, path])
        outputs[b].append(None)
    extend(rows(2), [2, 1, 2])

    torch.cuda.synchronize()
    kind = "bf16" if dtype == torch.bfloat16 else "f32"
    u = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
    # a query as the kernel turned and rounded it is off from the oracle's by a step and what norm and angle leave, of its pair's size: |q| |k| 2 of a logit each,
    # twice that of a probability and of the result
    slack = lambda q, k, mean: 2 * 2 * 2 * (2 * u + (d // 2 + 16) * 2.0 ** -24) * np.linalg.norm(q, axis=-1, keepdims=True) * np.linalg.norm(k, axis=-1).max() * d ** -0.5 * mean
    for b in range(3):
        x = np.concatenate(seen[b], 1)
        total = x.shape[1]
        q, kk, vv = oracle_rows(layer, x, np.arange(total))
        cached = pg.rows_of(host(layer.k_pages), layer.table[b].tolist(), total, page_rows), pg.rows_of(host(layer.v_pages), layer.table[b].tolist(), total, page_rows)
        # keys: rounded once, and the norm and angle in fp32 ((d / 2 + 16) half steps of a pair's size, as in the test of norm and rotation); values as they are
        pair = np.abs(kk).reshape(hkv, total, 2, d // 2).sum(2)
        assert (np.abs(cached[0] - kk) <= u * np.abs(kk) + (d // 2 + 16) * 2.0 ** -24 * 2 * np.concatenate([pair, pair], -1) + 1e-30).all()
        assert np.array_equal(cached[1], vv)
        # attention over the rows as they are in the pages, with the queries as they were rounded
        qr = torch.tensor(q).to(dtype).double().numpy()
        mask_all = pg.seen_window(0, total, window, 0, sinks)
        at = 0
        for out in outputs[b]:
            if out is None:
                at += len(paths[b])
                continue
            m = out.shape[1]
            for h in range(hq):
                for i in range(m):
                    vis = mask_all[at + i]
                    want, mean = pg.attention(qr[h, at + i:at + i + 1], cached[0][h // (hq // hkv)][vis], cached[1][h // (hq // hkv)][vis], np.ones((1, vis.sum()), bool), d ** -0.5)
                    tol = tolerance(qr[h, at + i:at + i + 1], cached[0][h // (hq // hkv)][vis], mean, want, d ** -0.5, cached[1][h // (hq // hkv)][vis], kind)
                    tol = tol + slack(qr[h, at + i:at + i + 1], cached[0][h // (hq // hkv)][vis], mean)
                    assert (np.abs(host(out[h, i]) - want[0]) <= tol[0] + 1e-30).all(), (b, h, i)
            at += m
        # the tree's rows see the whole cache, whatever the window
        tq, tk, tv = oracle_rows(layer, host(layer._project(tree)[0])[b], before[b] + depth[b].cpu().numpy())
        tq, tk = (torch.tensor(t).to(dtype).double().numpy() for t in (tq, tk))
        vis = pg.seen_tree(before[b], n, [int(m) for m in mask[b].tolist()])
        for h in range(hq):
            kh = np.concatenate([cached[0][h // (hq // hkv)][:before[b]], tk[h // (hq // hkv)]])
            vh = np.concatenate([cached[1][h // (hq // hkv)][:before[b]], tv[h // (hq // hkv)]])
            want, mean = pg.attention(tq[h], kh, vh, vis, d ** -0.5)
            tol = tolerance(tq[h], kh, mean, want, d ** -0.5, vh, kind) + 2 * slack(tq[h], kh, mean) + 1e-30   # and its keys
            assert (np.abs(host(tree_out[b, h]) - want) <= tol).all(), (b, h)


def test_a_captured_step_follows_the_lengths():
    torch.manual_seed(0)
    make = lambda: ex.PagedLayer(3, 400, 128, 8, 2, page_rows=16, window=60, sinks=2)
    a, b = make(), make()
    x = torch.randn(3, 300, 128, device=DEV).bfloat16()
    for layer in (a, b):
        layer.reserve([300, 20, 7])
        layer.extend(x, ints([300, 20, 7]))
        layer.grow([300, 20, 7])
        layer.reserve([30] * 3)
    token = torch.zeros(3, 1, 128, dtype=torch.bfloat16, device=DEV)
    out = torch.zeros(3, 8, 1, 128, dtype=torch.bfloat16, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        a.extend(token, out=out)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.extend(token, out=out)
    for i in range(6):
        token.copy_(torch.randn(3, 1, 128, device=DEV))
        graph.replay()
        want = b.extend(token)                       # the same calls, eager, in between
        torch.cuda.synchronize()
        assert torch.equal(out, want), i
        for layer in (a, b):
            layer.grow([1, 1, 1])
    assert torch.equal(a.k_pages, b.k_pages) and torch.equal(a.v_pages, b.v_pages)


def test_two_graphs_share_a_workspace():
    c = Paged("window", 8, 2, 128, 1, (5000, 900), "bf16", page_rows=64)
    t = Paged("tree", 8, 2, 128, 4, (3000, 20), "bf16", page_rows=64, mask=tree_masks(2, 4, 1))
    assert B.sdllm_paged_plan(c.shape, c.op).least_tiles and B.sdllm_paged_plan(t.shape, t.op).least_tiles
    c.ws = t.ws = torch.empty(max(c.ws.numel(), t.ws.numel()), dtype=torch.uint8, device=DEV)
    graphs = []
    for x in (c, t):
        x.run()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            x.run()
        graphs.append(g)
    for _ in range(3):
        for x, g in zip((c, t), graphs):
            x.out.fill_(float("nan"))
            g.replay()
            x.check()
        c.ws.fill_(0xFF)


@pytest.mark.parametrize("kind,Hq,Hkv,n,lengths", [("window", 8, 2, 1, (5000, 900)), ("tree", 14, 2, 20, (700, 4000)), ("window", 8, 1, 200, (100, 900))])
def test_another_stream_and_the_same_bits(kind, Hq, Hkv, n, lengths):
    c = Paged(kind, Hq, Hkv, 128, n, lengths, "bf16", page_rows=64, mask=tree_masks(2, n, 1) if kind == "tree" else None)
    c.run()
    first = c.out.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        out = torch.full_like(c.out, float("nan"))
        side.wait_stream(torch.cuda.current_stream())
        c.run(stream=side, out=out)
        side.synchronize()
        assert torch.equal(out, first)
    c.check()


def test_pages_beyond_32_bit_offsets():
    # 3 * 2^31 bytes of pages, the rows in use at their ends
    n_pages, page, d = 3 * (1 << 31) // (2 * 64 * 128), 64, 128
    c = Paged("window", 4, 1, d, 3, (150, 70), "bf16", page_rows=page)
    k, v = (torch.empty(n_pages, 1, page, d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    far = [n_pages - 1, 0, n_pages // 2 + 1, n_pages - 2, 5, n_pages // 3 * 2]
    at = 0
    for b in range(2):
        for i in range(-(-(c.host_lengths[b] + 3) // page)):
            k[far[at]], v[far[at]] = c.k_pages[c.table[b, i].long()], c.v_pages[c.table[b, i].long()]
            c.table[b, i] = far[at]
            at += 1
    s = B.make_paged_shape(batch=2, n_q_heads=4, n_kv_heads=1, head_dim=d, rows=3, dtype=B.SDLLM_BF16, n_pages=n_pages, page_rows=page, table_pages=c.table.shape[1],
                           q_stride=B.strides_of(c.q), out_stride=B.strides_of(c.out))
    ws = torch.empty(B.sdllm_paged_workspace_bytes(s, c.op), dtype=torch.uint8, device=DEV)
    B.sdllm_window_attn_paged(s, c.q, k, v, c.table, c.lengths, None, c.out, ws)
    small = Paged("window", 4, 1, d, 3, (150, 70), "bf16", page_rows=page)   # the same rows
    small.run()
    torch.cuda.synchronize()
    assert torch.equal(c.out, small.out)
    # and appended there
    qk = B.make_qk_shape(batch=2, n_q_heads=0, n_kv_heads=1, head_dim=d, rows=3, dtype=B.SDLLM_BF16, rot_dim=0, norm=B.SDLLM_NORM_NONE)
    rows = torch.randn(2, 1, 3, d, device=DEV).bfloat16()
    B.sdllm_append_paged(qk, s, None, rows, rows, None, None, None, None, None, c.lengths, None, c.table, None, k, v)
    torch.cuda.synchronize()
    for b, length in enumerate(c.host_lengths):
        for i in range(3):
            page_at = int(c.table[b, (length + i) // page])
            assert torch.equal(k[page_at, 0, (length + i) % page], rows[b, 0, i]) and torch.equal(v[page_at, 0, (length + i) % page], rows[b, 0, i])


@pytest.mark.parametrize("kind,Hq,Hkv,n,lengths", [("window", 8, 2, 1, (5000, 900, 33)), ("tree", 28, 4, 40, (700, 2000, 0)), ("window", 16, 1, 64, (1500, 300, 7))])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_pages_named_more_than_once(kind, Hq, Hkv, n, lengths, dtype):
    c = Paged(kind, Hq, Hkv, 64, n, lengths, dtype, page_rows=32, mask=tree_masks(3, n, 1) if kind == "tree" else None)
    c.table[:] = c.table[0, :3].repeat(c.table.shape[1])[:c.table.shape[1]]   # all sequences share three pages, again and again
    c.run()
    c.check()


# the forms of the attentions: streaming or shared tiles, columns, wavefronts, cut or not
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kind,Hq,Hkv,n,lengths,form", [
    ("window", 16, 1, 1, (2000,), (0, 16, 8, True)), ("window", 16, 1, 1, (300,), (0, 16, 8, False)), ("window", 3, 1, 1, (900,) * 65, (0, 16, 4, True)),
    ("window", 16, 16, 1, (100,) * 65, (0, 16, 4, False)), ("tree", 17, 1, 1, (2000,), (0, 32, 8, True)), ("tree", 30, 1, 4, (100,), (0, 32, 8, False)),
    ("tree", 8, 1, 4, (900,) * 65, (0, 32, 4, True)), ("tree", 8, 1, 8, (60,) * 65, (0, 32, 4, False)), ("tree", 2, 1, 40, (1000,) * 17, (1, 128, 8, True)),
    ("tree", 2, 1, 40, (100,) * 17, (1, 128, 8, False)), ("tree", 5, 1, 33, (1200, 30), (1, 256, 8, True)), ("window", 5, 1, 160, (60, 0), (1, 256, 8, False))])
def test_forms(d, kind, Hq, Hkv, n, lengths, form):
    c = Paged(kind, Hq, Hkv, d, n, lengths, "bf16", page_rows=32, mask=tree_masks(len(lengths), n, 2) if kind == "tree" else None)
    p = B.sdllm_paged_plan(c.shape, c.op)
    assert (p.shared, p.block_cols, p.waves, p.least_tiles > 0) == form
    c.run()
    c.check()


# more tiles than one look-up of places holds (64 a wavefront or a share), whole and at odd ends
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kind,Hq,Hkv,n,length,dtype", [("window", 200, 1, 2, 7001, "bf16"), ("tree", 200, 200, 1, 20003, "bf16"), ("tree", 70, 70, 1, 17000, "f32")])
def test_long_shares(d, kind, Hq, Hkv, n, length, dtype):
    Hq, Hkv = (Hq, Hkv) if d == 128 else (Hq // 2, max(1, Hkv // 2))
    batch = 1 if kind == "tree" else 1
    c = Paged(kind, Hq, Hkv, d, n, (length,) * batch, dtype, page_rows=64, mask=tree_masks(batch, n, 2) if kind == "tree" else None)
    c.run()
    # a few heads against the oracle: the others' rows are made the same way
    torch.cuda.synchronize()
    got, q, kb, vb = (host(x) for x in (c.out, c.q, c.k_blk, c.v_blk))
    kp, vp, table = host(c.k_pages), host(c.v_pages), c.table.cpu().numpy()
    for h in (0, Hq // 2, Hq - 1):
        g = h // (Hq // Hkv)
        pages = table[0][:-(-(length + (n if kind == "window" else 0)) // 64)]
        end = length + (n if kind == "window" else 0)
        k, v = (x[pages, g].reshape(-1, d)[:end] for x in (kp, vp))
        if kind == "tree":
            k, v, seen = np.concatenate([k, kb[0, g]]), np.concatenate([v, vb[0, g]]), pg.seen_tree(length, n, [x & (1 << 64) - 1 for x in c.host_mask[0]])
        else:
            seen = pg.seen_window(length, n, -1, 0, 0)
        want, mean = pg.attention(q[0, h], k, v, seen, c.scale)
        assert (np.abs(got[0, h] - want) <= tolerance(q[0, h], k, mean, want, c.scale, v, dtype)).all(), h


def test_the_command(monkeypatch, capsys):
    monkeypatch.setattr("sys.argv", ["paged_serving", "--prompts", "100,7", "--hidden", "128", "--q-heads", "4", "--kv-heads", "2", "--tokens", "3", "--tree", "9",
                                     "--window", "50", "--sinks", "2"])
    ex.main()
    said = capsys.readouterr().out
    assert "pages of 64 rows, lengths [103, 10]" in said and "replayed" in said and "rows kept" in said
