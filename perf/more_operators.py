"""What the speed of the paged cache's operators is judged by.

A batch of sequences of unlike lengths shares one pool of pages.  New rows are normalised, turned by their position and put there
(`append`); a block of rows, or a tree of drafted tokens, attends over its sequence's rows and its own (`tree`); tokens that are in the
cache already, one of a sequence or thousands, attend to a window before them and to a few first tokens (`window`).  Kinds of a case:

  append  sdllm_append_paged: queries, keys and values as views of one projection [B, rows, (Hq + 2 Hkv) d]; queries to a tensor of their own,
          keys and values into the pages.  `picked`: the rows of a tree that were accepted, rotated before
  tree    sdllm_tree_attn_paged: rows [B, Hq, n, d] over the cache and the rows' own keys and values, which are in no page yet
  window  sdllm_window_attn_paged: the last rows of a cache over it

Row j of a sequence is row j % page_rows of page table[b][j / page_rows].  `lengths` are the rows of the sequences before the new ones.
Head counts and sizes are those of the repository's workloads (32 / 32 and 28 / 4 heads of 128, prompts of 1024 to 32768 tokens, blocks of 32) and its
tests (other groups, head dimension 64, fp32, odd lengths); batches of tens of sequences, windows and trees are generic.
"""
import math

import torch

own = False
DEVICE = "cuda"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---------------------------------------------------------------- cases
# lengths of the sequences: `shortest` to `longest`, evenly spread; new rows of a sequence: `rows`, or (ragged) a quarter of them to all
def _case(kind, batch, q_heads, kv_heads, rows, shortest, longest, **more):
    c = dict(kind=kind, batch=batch, q_heads=q_heads, kv_heads=kv_heads, head_dim=128, dtype="bf16", rows=rows, ragged=False, shortest=shortest,
             longest=longest, page_rows=64, layout="heads")
    if kind == "append":
        c.update(rot=128, pairing="halves", norm=True, base=1e6, picked=False)
    elif kind == "tree":
        c.update(masked=True)
    elif kind == "window":
        c.update(left=-1, right=0, sinks=0)
    c.update(more)
    return c


def listed():
    return [
        # one token of one sequence: latency
        _case("append", 1, 28, 4, 1, 4096, 4096, name="append_token_b1"),
        # the accepted rows of drafted trees, already turned; single precision, odd sizes, part of a page of 16 rows
        _case("append", 5, 0, 2, 23, 77, 1001, ragged=True, head_dim=64, dtype="f32", page_rows=16, rot=0, norm=False, picked=True,
              name="append_accepted_f32"),
        # prompts of a batch on their way into an empty cache and behind a shared beginning
        _case("append", 8, 32, 8, 4096, 0, 512, ragged=True, base=5e5, name="append_prompts_b8"),
        # a decoding block of one sequence behind a 1k prompt: every row sees all of its block
        _case("tree", 1, 32, 32, 32, 1024, 1024, masked=False, name="tree_block_mha_b1"),
        # drafted trees of a batch of grouped-query heads, lengths far apart
        _case("tree", 8, 28, 4, 64, 500, 8000, ragged=True, name="tree_gqa_b8"),
        # few drafted tokens behind a very long document
        _case("tree", 2, 32, 8, 8, 65000, 131000, page_rows=256, layout="rows", name="tree_long"),
        # single precision, odd
        _case("tree", 3, 6, 3, 13, 0, 333, head_dim=64, dtype="f32", page_rows=16, name="tree_f32_odd"),
        # one new token in each of many sequences that see everything before them ...
        _case("window", 32, 28, 4, 1, 1000, 16000, name="window_tokens_all"),
        # ... or a window and four first tokens; the smallest attention
        _case("window", 4, 28, 4, 1, 3000, 9000, left=1023, sinks=4, name="window_tokens_1k"),
        # prompts with a window
        _case("window", 4, 28, 4, 4096, 0, 2000, left=1023, sinks=4, ragged=True, name="window_prompts_gqa"),
        # one prompt to its whole past, head dimension 64, in pages with rows before heads
        _case("window", 1, 16, 2, 8192, 1000, 1000, head_dim=64, layout="rows", page_rows=128, name="window_prompt_causal_d64"),
        # both directions, single precision, odd
        _case("window", 2, 4, 1, 333, 100, 555, head_dim=64, dtype="f32", left=99, right=50, sinks=3, page_rows=32, ragged=True, name="window_f32_both"),
    ]


def draw(rng):
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    while True:
        kind = rng.choice(("append", "tree", "window", "window"))
        dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
        d = rng.choice((64, 128, 128))
        q_heads, kv_heads = rng.choice(((32, 32), (28, 4), (8, 8), (16, 2), (4, 1), (2, 2), (14, 2), (32, 8), (6, 3)))
        batch = rng.choice((1, 1, 2, 3, 5, 8, 17, 32))
        longest = log(1, 40000)
        more = dict(head_dim=d, dtype=dtype, page_rows=rng.choice((16, 32, 64, 128, 256)), layout=rng.choice(("heads", "rows")),
                    ragged=rng.random() < 0.5)
        shortest = rng.choice((longest, longest // 2, longest // 10, 0))
        if kind == "append":
            picked = rng.random() < 0.25
            c = _case(kind, batch, 0 if picked else q_heads, kv_heads, log(1, 64) if picked else log(1, 4096), min(shortest, 2000), min(longest, 2000),
                      rot=rng.choice((d, d, d // 2, 16, d - 16)), pairing=rng.choice(("halves", "adjacent")), norm=rng.random() < 0.7,
                      base=rng.choice((1e4, 5e5, 1e6)), picked=picked, **more)
        elif kind == "tree":
            c = _case(kind, batch, q_heads, kv_heads, rng.choice((1, 4, 8, 16, 32, 64, rng.randint(1, 64))), shortest, longest,
                      masked=rng.random() < 0.8, **more)
        else:
            rows = rng.choice((1, 1, log(1, 8192), log(1, 8192)))
            window = dict(left=rng.choice((-1, log(16, 8192), log(16, 8192))), right=rng.choice((0, 0, 0, -1, log(1, 100))), sinks=rng.choice((0, 1, 4, rng.randint(1, 130))))
            c = _case(kind, batch, q_heads, kv_heads, rows, shortest, longest, **window, **more)
        w, scale = work(c), 1 if dtype == "bf16" else 16
        # the pool fits, and no case is more than the largest listed ones
        pool = 4 * batch * kv_heads * (c["longest"] + c["rows"]) * d
        pairs = q_heads * c["rows"] * (c["longest"] + c["rows"]) if kind != "append" else 0
        if pool <= 1.2e9 and pairs <= 3e9 and w["bytes"] <= 8e8 and w["flops"] * scale <= 1.7e11:
            return c


def _spread(lo, hi, n):
    return [hi if n == 1 else lo + (hi - lo) * i // (n - 1) for i in range(n)]


def _lengths(c):
    return _spread(c["shortest"], c["longest"], c["batch"])


def _counts(c):
    """New rows, the shortest sequences' most."""
    return _spread(c["rows"], max(1, c["rows"] // 4), c["batch"]) if c["ragged"] else [c["rows"]] * c["batch"]


# ---------------------------------------------------------------- what a server has in hand
def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEVICE)


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    c, d, dt = case, case["head_dim"], TYPES[case["dtype"]]
    batch, hq, hkv, n, page = c["batch"], c["q_heads"], c["kv_heads"], c["rows"], c["page_rows"]
    # which sequence has which length depends on the seed
    order = torch.randperm(batch, generator=g, device=DEVICE).tolist()
    lengths, counts = [_lengths(c)[i] for i in order], [_counts(c)[i] for i in order]
    needed = [-(-(length + count) // page) for length, count in zip(lengths, counts)]
    n_pages = sum(needed) + 3
    # pages in no order; entries past a sequence's end name none
    free = torch.randperm(n_pages, generator=g, device=DEVICE).int()
    table = torch.full((batch, max(needed) + 1), -1, dtype=torch.int32, device=DEVICE)
    at = 0
    for b, p in enumerate(needed):
        table[b, :p] = free[at:at + p]
        at += p

    def pool():
        x = torch.empty(n_pages, hkv, page, d, dtype=dt, device=DEVICE) if c["layout"] == "heads" else \
            torch.empty(n_pages, page, hkv, d, dtype=dt, device=DEVICE).permute(0, 2, 1, 3)
        for i in range(0, n_pages, 1024):
            x[i:i + 1024] = _randn(g, *x[i:i + 1024].shape)
        return x

    tensor = lambda values: torch.tensor(values, dtype=torch.int32, device=DEVICE)
    state = dict(case=c, host=(lengths, counts), lengths=tensor(lengths), counts=tensor(counts) if c["ragged"] or c.get("picked") else None, table=table,
                 k_pages=pool(), v_pages=pool())
    # keys of a model have channels of unlike size
    size = torch.exp(0.4 * _randn(g, 1, 1, 1, d))
    state["k_pages"].mul_(size.to(dt))
    if c["kind"] == "append":
        x = (_randn(g, batch, n, hq + 2 * hkv, d) * torch.exp(0.3 * _randn(g, 1, 1, hq + 2 * hkv, d))).to(dt).permute(0, 2, 1, 3)
        state["q"], state["k"], state["v"] = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
        state["q_weight"], state["k_weight"] = ((1 + 0.1 * _randn(g, d)).to(dt) if c["norm"] else None for _ in range(2))
        half = torch.arange(0, c["rot"], 2, device=DEVICE, dtype=torch.float64)
        state["inv_freq"] = (c["base"] ** (-half / max(1, c["rot"]))).float()
        state["q_out"] = torch.zeros(batch, hq, n, d, dtype=dt, device=DEVICE)
        if c["picked"]:
            # ascending rows of the tree, a path; positions of a tree's rows are their depths behind the cache
            pick = torch.rand(batch, n, generator=g, device=DEVICE).argsort(-1)
            for b, count in enumerate(counts):
                pick[b, :count] = pick[b, :count].sort().values
            state["pick"] = pick.int()
            depth = torch.randint(0, 8, (batch, n), generator=g, device=DEVICE)
            state["positions"] = (state["lengths"][:, None] + depth).int()
    else:
        state["q"] = _randn(g, batch, n, hq, d).to(dt).permute(0, 2, 1, 3)
        state["out"] = torch.zeros(batch, n, hq, d, dtype=dt, device=DEVICE).permute(0, 2, 1, 3)
        if c["kind"] == "tree":
            x = _randn(g, batch, n, 2 * hkv, d)
            x[:, :, :hkv] *= size
            x = x.to(dt).permute(0, 2, 1, 3)
            state["k_blk"], state["v_blk"] = x[:, :hkv], x[:, hkv:]
            # a row sees what its parent sees, and itself
            rows = torch.arange(n, device=DEVICE)
            parent = (torch.rand(batch, n, generator=g, device=DEVICE) * (rows + 1)).long() - 1
            mask = torch.zeros(batch, n, dtype=torch.int64, device=DEVICE)
            for i in range(n):
                above = torch.where(parent[:, i] < 0, 0, mask.gather(1, parent[:, i:i + 1].clamp(min=0))[:, 0])
                mask[:, i] = above | 1 << i if i < 63 else above | -1 << 63
            state["mask"] = mask if c["masked"] else None
    return state


# ---------------------------------------------------------------- one pass
def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"append": _own_append, "tree": _own_tree, "window": _own_window}[kind](state)
    return {"append": _plain_append, "tree": _plain_tree, "window": _plain_window}[kind](state)


def _places(s, first, end, b):
    """Pages and rows within them of rows [first, end) of sequence b."""
    at = torch.arange(first, end, device=DEVICE)
    page = s["case"]["page_rows"]
    return s["table"][b].long()[at // page], at % page


def _appended(s):
    return ((s["q_out"],) if s["case"]["q_heads"] else ()) + (s["k_pages"], s["v_pages"])


def _plain_append(s):
    c = s["case"]
    for b, (length, count) in enumerate(zip(*s["host"])):
        rows = s["pick"][b, :count].long() if c["picked"] else torch.arange(count, device=DEVICE)
        position = (s["positions"][b][rows] if c["picked"] else length + rows).double()
        angle = position[:, None] * s["inv_freq"].double()
        cos, sin = angle.cos().float(), angle.sin().float()

        def one(x, weight):
            dt, x = x.dtype, x[:, rows].float()
            if c["norm"]:
                x = x * (x.square().mean(-1, keepdim=True) + 1e-6).rsqrt() * weight.float()
            turned, rest = x[..., :c["rot"]], x[..., c["rot"]:]
            if c["pairing"] == "halves":
                a, z = turned.chunk(2, -1)
                turned = torch.cat([a * cos - z * sin, a * sin + z * cos], -1)
            else:
                a, z = turned[..., 0::2], turned[..., 1::2]
                turned = torch.stack([a * cos - z * sin, a * sin + z * cos], -1).flatten(-2)
            return torch.cat([turned, rest], -1).to(dt)

        if c["q_heads"]:
            s["q_out"][b, :, :count] = one(s["q"][b], s["q_weight"])
        pages, at = _places(s, length, length + count, b)
        s["k_pages"][pages, :, at] = one(s["k"][b], s["k_weight"]).transpose(0, 1)
        s["v_pages"][pages, :, at] = s["v"][b][:, rows].transpose(0, 1)
    return _appended(s)


def _cached(s, b, end):
    """Rows [0, end) of sequence b, [Hkv, end, d] each, in 32 bits."""
    pages, at = _places(s, 0, end, b)
    return (s[x][pages, :, at].transpose(0, 1).float() for x in ("k_pages", "v_pages"))


def _attention(q, k, v, seen):
    """Queries [Hq, n, d] over keys and values [Hkv, m, d]; seen [n, m].  A row that sees nothing is zero."""
    heads, n, d = q.shape
    logits = torch.matmul(q.float().reshape(k.shape[0], -1, d), k.transpose(-1, -2).contiguous()) / math.sqrt(d)
    logits = logits.reshape(k.shape[0], -1, n, k.shape[1]).masked_fill_(~seen, -math.inf)
    top = logits.amax(-1, keepdim=True) if k.shape[1] else logits.new_zeros(*logits.shape[:3], 1)
    p = (logits - torch.where(top == -math.inf, 0.0, top)).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p.reshape(k.shape[0], -1, k.shape[1]), v).reshape(*logits.shape[:3], d) / torch.where(total == 0, 1.0, total)
    return out.reshape(heads, n, d).to(q.dtype)


def _plain_tree(s):
    c, out = s["case"], torch.zeros_like(s["out"])
    for b, (length, count) in enumerate(zip(*s["host"])):
        k, v = _cached(s, b, length)
        k, v = torch.cat([k, s["k_blk"][b, :, :count].float()], 1), torch.cat([v, s["v_blk"][b, :, :count].float()], 1)
        seen = torch.ones(count, length + count, dtype=torch.bool, device=DEVICE)
        if c["masked"]:
            seen[:, length:] = (s["mask"][b, :count, None] >> torch.arange(count, device=DEVICE) & 1).bool()
        out[b, :, :count] = _attention(s["q"][b, :, :count], k, v, seen)
    return out


def _plain_window(s):
    c, out = s["case"], torch.zeros_like(s["out"])
    for b, (length, count) in enumerate(zip(*s["host"])):
        k, v = _cached(s, b, length + count)
        place, key = (length + torch.arange(count, device=DEVICE))[:, None], torch.arange(length + count, device=DEVICE)
        seen = key >= place - c["left"] if c["left"] >= 0 else torch.ones(count, length + count, dtype=torch.bool, device=DEVICE)
        seen = seen | (key < c["sinks"])
        if c["right"] >= 0:
            seen = seen & (key <= place + c["right"])
        out[b, :, :count] = _attention(s["q"][b, :, :count], k, v, seen)
    return out


def _shape(B, s):
    c = s["case"]
    strides = dict(page_stride=B.strides_of(s["k_pages"]))
    if c["kind"] != "append":
        strides.update(q_stride=B.strides_of(s["q"]), out_stride=B.strides_of(s["out"]))
    if c["kind"] == "tree":
        strides.update(blk_stride=B.strides_of(s["k_blk"]))
    if c["kind"] == "window":
        strides.update(window_left=c["left"], window_right=c["right"], sinks=c["sinks"])
    return B.make_paged_shape(batch=c["batch"], n_q_heads=c["q_heads"] or c["kv_heads"], n_kv_heads=c["kv_heads"], head_dim=c["head_dim"], rows=c["rows"],
                              dtype=B.SDLLM_BF16 if c["dtype"] == "bf16" else B.SDLLM_F32, n_pages=s["k_pages"].shape[0], page_rows=c["page_rows"],
                              table_pages=s["table"].shape[1], **strides)


def _own_append(s):
    from paper_2508_02558_amd import binding as B
    c = s["case"]
    if "shape" not in s:
        s["shape"] = _shape(B, s)
        s["qk"] = B.make_qk_shape(batch=c["batch"], n_q_heads=c["q_heads"], n_kv_heads=c["kv_heads"], head_dim=c["head_dim"], rows=c["rows"],
                                  dtype=s["shape"].dtype, rot_dim=c["rot"], norm=B.SDLLM_NORM_RMS if c["norm"] else B.SDLLM_NORM_NONE,
                                  pairing=B.SDLLM_PAIR_HALVES if c["pairing"] == "halves" else B.SDLLM_PAIR_ADJACENT, eps=1e-6, pos_stride=c["rows"],
                                  q_in_stride=B.strides_of(s["q"]), k_in_stride=B.strides_of(s["k"]))
    some = lambda x: x if c["q_heads"] else None
    B.sdllm_append_paged(s["qk"], s["shape"], some(s["q"]), s["k"], s["v"], s["q_weight"], s["k_weight"], s["inv_freq"] if c["rot"] else None,
                         s.get("positions"), s.get("pick"), s["lengths"], s["counts"], s["table"], some(s["q_out"]), s["k_pages"], s["v_pages"])
    return _appended(s)


def _workspace(B, s, op):
    if "shape" not in s:
        s["shape"] = _shape(B, s)
        s["ws"] = torch.empty(B.sdllm_paged_workspace_bytes(s["shape"], op), dtype=torch.uint8, device=DEVICE)
    return s["ws"]


def _own_tree(s):
    from paper_2508_02558_amd import binding as B
    ws = _workspace(B, s, B.SDLLM_OP_TREE_ATTN_PAGED)
    B.sdllm_tree_attn_paged(s["shape"], s["q"], s["k_pages"], s["v_pages"], s["table"], s["lengths"], s["counts"], s["k_blk"], s["v_blk"], s["mask"], s["out"], ws)
    return s["out"]


def _own_window(s):
    from paper_2508_02558_amd import binding as B
    ws = _workspace(B, s, B.SDLLM_OP_WINDOW_ATTN_PAGED)
    B.sdllm_window_attn_paged(s["shape"], s["q"], s["k_pages"], s["v_pages"], s["table"], s["lengths"], s["counts"], s["out"], ws)
    return s["out"]


# ---------------------------------------------------------------- what a pass cannot do without
def _seen_sums(c, length, count):
    """Keys that the rows at places length .. length + count - 1 see: all together, and how many different ones."""
    end, total, first, last = length + count, 0, length + count, -1
    for p in range(length, end):
        hi = end - 1 if c["right"] < 0 else min(end - 1, p + c["right"])
        lo = 0 if c["left"] < 0 else max(0, p - c["left"])
        total += hi - lo + 1 + min(c["sinks"], lo)
        first, last = min(first, lo), max(last, hi)
    return total, last - first + 1 + min(c["sinks"], first) if count else 0


def work(case):
    c, d = case, case["head_dim"]
    es = 2 if c["dtype"] == "bf16" else 4
    size = flops = 0
    for length, count in zip(_lengths(c), _counts(c)):
        if c["kind"] == "append":
            values = count * d * (c["q_heads"] + 2 * c["kv_heads"])
            size += 2 * values * es
            flops += 10 * count * d * (c["q_heads"] + c["kv_heads"])
            continue
        if c["kind"] == "tree":
            # a row of a random tree sees about log(count) rows of it
            pairs = count * length + (round(count * (1 + math.log(count))) if c["masked"] else count * count)
            keys = length + count
            size += 8 * count
        else:
            pairs, keys = _seen_sums(c, length, count)
        size += 2 * c["q_heads"] * count * d * es + 2 * c["kv_heads"] * keys * d * es
        flops += 4 * d * c["q_heads"] * pairs
    return dict(bytes=size + 8 * c["batch"], flops=flops)


# ---------------------------------------------------------------- the same from the definitions, in 64 bits
def exact(case, seed):
    s, c, d = prepare(case, seed), case, case["head_dim"]
    page = c["page_rows"]
    f64 = lambda x: x.to(torch.float64)
    where = s["table"].tolist()
    if c["kind"] == "append":
        got = [f64(s["q_out"]), f64(s["k_pages"]), f64(s["v_pages"])]
        half = c["rot"] // 2
        first = torch.arange(half, device=DEVICE) * (1 if c["pairing"] == "halves" else 2)
        second = first + (half if c["pairing"] == "halves" else 1)
        for b, (length, count) in enumerate(zip(*s["host"])):
            source = s["pick"][b].tolist()[:count] if c["picked"] else list(range(count))
            position = torch.tensor([s["positions"][b].tolist()[r] for r in source] if c["picked"] else [length + i for i in range(count)],
                                    dtype=torch.float64, device=DEVICE)
            # a pair as a complex number, turned by exp(i angle)
            turn = torch.polar(torch.ones(count, half, dtype=torch.float64, device=DEVICE), position[:, None] * f64(s["inv_freq"]))
            turned = []
            for x, w in ((s["q"], s["q_weight"]), (s["k"], s["k_weight"])):
                x = f64(x[b])[:, source]
                if c["norm"]:
                    x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / d + 1e-6) * f64(w)
                z = torch.complex(x[..., first], x[..., second]) * turn
                x[..., first], x[..., second] = z.real, z.imag
                turned.append(x)
            if c["q_heads"]:
                got[0][b, :, :count] = turned[0]
            values = f64(s["v"][b])[:, source]
            # page by page
            i = 0
            while i < count:
                r = (length + i) % page
                take = min(page - r, count - i)
                p = where[b][(length + i) // page]
                got[1][p, :, r:r + take] = turned[1][:, i:i + take]
                got[2][p, :, r:r + take] = values[:, i:i + take]
                i += take
        return tuple(got if c["q_heads"] else got[1:])
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device=DEVICE)
    group = c["q_heads"] // c["kv_heads"]
    for b, (length, count) in enumerate(zip(*s["host"])):
        end = length if c["kind"] == "tree" else length + count
        named = where[b][:-(-end // page)]
        for h in range(c["kv_heads"]):
            k, v = (f64(s[x][named, h].reshape(-1, d)[:end]) for x in ("k_pages", "v_pages"))
            if c["kind"] == "tree":
                k, v = torch.cat([k, f64(s["k_blk"][b, h, :count])]), torch.cat([v, f64(s["v_blk"][b, h, :count])])
                hidden = torch.zeros(count, length + count, dtype=torch.bool, device=DEVICE)
                if c["masked"]:
                    hidden[:, length:] = torch.tensor([[(m >> j & 1) == 0 for j in range(count)] for m in s["mask"][b, :count].tolist()], device=DEVICE)
            else:
                key = torch.arange(end, device=DEVICE)[None].expand(count, end)
                ahead = torch.arange(count, device=DEVICE)[:, None] + length - key          # how far a key is behind the row
                hidden = torch.zeros_like(key, dtype=torch.bool)
                if c["left"] >= 0:
                    hidden |= (ahead > c["left"]) & (key >= c["sinks"])
                if c["right"] >= 0:
                    hidden |= -ahead > c["right"]
            for x in range(h * group, (h + 1) * group):
                logits = torch.matmul(f64(s["q"][b, x, :count]), k.t().contiguous()) * d ** -0.5
                w = torch.softmax(logits.masked_fill_(hidden, -math.inf), -1)
                out[b, x, :count] = torch.matmul(torch.where(hidden.all(-1, keepdim=True), 0.0, w), v)
    return out
