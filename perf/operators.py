"""What the speed of the block decoder's operators beside its bf16 / fp32 cache is judged by.

A decoding block of one layer starts from the projections of its positions: queries and keys are normalised per head and turned by
their position (`rope`), the retained keys and values of the sequence are gathered once per block into a cache of 4 bits a value
(`pack`), and every further step attends over that cache and the block's own rows (`attend`).  Kinds of a case:

  rope    sdllm_qk_norm_rope: queries and keys as views of one projection [B, rows, (Hq + 2 Hkv) d], results [B, H, rows, d]
  pack    sdllm_compact_kv_packed, and sdllm_unpack_kv, which gives the values that the cache stands for
  attend  sdllm_sparse_attn_packed: block queries over the packed rows and the block's own keys and values

Packed values are e2m1 numbers (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives) times 2^e with one e for 32 of them: 32 channels of a
key, or one channel of 32 retained value rows in a row.  e is the smallest integer of [-125, 125] for which all magnitudes are below 7 2^e; values
go to the nearest number, ties to the even code, past the ends to the last one.  A group that holds an infinity or a NaN is NaN as a whole.

Head counts and sizes are those of the repository's workloads (32 / 32 and 28 / 4 heads of 128, prompts of 1024 to 32768 tokens) and
its tests (other groups, head dimension 64, fp32, block lengths other than 32, odd lengths).
"""
import math

import torch

own = False
DEVICE = "cuda"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
TILE = 32


# ---------------------------------------------------------------- cases
def _rope(batch, q_heads, kv_heads, rows, first, **more):
    c = dict(kind="rope", batch=batch, q_heads=q_heads, kv_heads=kv_heads, head_dim=128, dtype="bf16", rows=rows, first=first, rot=128,
             pairing="halves", norm=True, base=1e6)
    c.update(more)
    return c


def _pack(batch, kv_heads, seq_len, kept, **more):
    c = dict(kind="pack", batch=batch, kv_heads=kv_heads, head_dim=128, dtype="bf16", seq_len=seq_len, kept=kept)
    c.update(more)
    return c


def _attend(batch, q_heads, kv_heads, cached, **more):
    c = dict(kind="attend", batch=batch, q_heads=q_heads, kv_heads=kv_heads, head_dim=128, dtype="bf16", block=32, cached=cached)
    c.update(more)
    return c


def listed():
    return [
        # a block's rows of one sequence: latency
        _rope(1, 28, 4, 32, 4096, name="rope_block_gqa_b1"),
        # all rows of a batch of 4k prompts, as a full-sequence step needs them
        _rope(8, 32, 32, 4352, 0, base=5e5, name="rope_full_mha_b8"),
        # part of the head turned, adjacent pairs, no norm, far positions, odd rows, single precision
        _rope(2, 14, 2, 333, 90001, head_dim=64, dtype="f32", rot=32, pairing="adjacent", norm=False, base=1e4, name="rope_f32_partial"),
        # a cache rebuild of one sequence ...
        _pack(1, 4, 4352, 2160, name="pack_gqa_b1"),
        # ... of a batch, ...
        _pack(8, 32, 4352, 2160, name="pack_mha_b8"),
        # ... and of odd lengths in single precision
        _pack(3, 2, 2133, 1051, head_dim=64, dtype="f32", name="pack_f32_odd"),
        # the thirty-of-32 steps, from one sequence with a 1k prompt ...
        _attend(1, 32, 32, 624, name="attend_mha_b1"),
        # ... over a long document ...
        _attend(1, 28, 4, 8312, name="attend_gqa_long"),
        # ... and batches of grouped-query heads ...
        _attend(8, 28, 4, 2288, name="attend_gqa_b8"),
        # ... to the benchmark shape
        _attend(8, 32, 32, 2160, name="attend_mha_b8"),
        # single tokens (blocks of one position) of a small model over an odd number of rows
        _attend(4, 16, 2, 1337, head_dim=64, block=1, name="attend_single_token"),
        # single precision: the reference runs people compare against, small and odd
        _attend(1, 2, 2, 77, head_dim=64, dtype="f32", block=13, name="attend_f32_tiny"),
    ]


def draw(rng):
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    kind = rng.choice(("rope", "pack", "attend", "attend"))
    dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
    d = rng.choice((64, 128, 128))
    q_heads, kv_heads = rng.choice(((32, 32), (28, 4), (8, 8), (16, 2), (4, 1), (2, 2), (14, 2), (32, 8), (6, 3)))
    while True:
        batch = rng.choice((1, 1, 2, 3, 4, 8))
        if kind == "rope":
            c = _rope(batch, q_heads, kv_heads, log(1, 4352), log(1, 120000), head_dim=d, dtype=dtype, rot=rng.choice((d, d, d // 2, 16, d - 16)),
                      pairing=rng.choice(("halves", "adjacent")), norm=rng.random() < 0.7, base=rng.choice((1e4, 5e5, 1e6)))
            size = batch * (q_heads + kv_heads) * c["rows"] * d * (1 if dtype == "bf16" else 2)
            if size <= 8 * 64 * 4352 * 128 // 2:
                return c
        elif kind == "pack":
            n = log(33, 33000)
            c = _pack(batch, kv_heads, n, max(1, min(n, int(n * rng.choice((0.25, 0.5, 0.5, 0.8, 1.0))))), head_dim=d, dtype=dtype)
            if batch * kv_heads * c["kept"] * d * (1 if dtype == "bf16" else 2) <= 8 * 32 * 2160 * 128:
                return c
        else:
            c = _attend(batch, q_heads, kv_heads, log(1, 33000) - (1 if rng.random() < 0.1 else 0), head_dim=d, dtype=dtype,
                        block=rng.choice((1, 4, 7, 16, 32, 32, 33, 64, rng.randint(1, 64))))
            if batch * kv_heads * c["cached"] * d <= 8 * 32 * 2160 * 128 and batch * q_heads * c["block"] * c["cached"] <= 8 * 32 * 32 * 2160:
                return c


# ---------------------------------------------------------------- what a decoder has in hand
def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEVICE)


def _kv(g, batch, heads, rows, d):
    """Keys with channels of unlike size, as rotations leave them, and a few salient rows; values."""
    k = _randn(g, batch, heads, rows, d) * torch.exp(0.4 * _randn(g, batch, heads, 1, d))
    k *= 1 + 2 * (torch.rand(batch, heads, rows, 1, generator=g, device=DEVICE) < 0.02)
    return k, _randn(g, batch, heads, rows, d)


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    c, d, dt = case, case["head_dim"], TYPES[case["dtype"]]
    batch, hkv = c["batch"], c["kv_heads"]
    state = dict(case=c)
    if c["kind"] == "rope":
        hq, n = c["q_heads"], c["rows"]
        x = _randn(g, batch, n, hq + 2 * hkv, d) * torch.exp(0.3 * _randn(g, 1, 1, hq + 2 * hkv, d))
        x = x.to(dt).permute(0, 2, 1, 3)
        state["q"], state["k"] = x[:, :hq], x[:, hq:hq + hkv]
        state["q_weight"], state["k_weight"] = ((1 + 0.1 * _randn(g, d)).to(dt) if c["norm"] else None for _ in range(2))
        half = torch.arange(0, c["rot"], 2, device=DEVICE, dtype=torch.float64)
        state["inv_freq"] = (c["base"] ** (-half / c["rot"])).float()
        # every sequence of the batch is somewhere else
        state["positions"] = (c["first"] + 37 * torch.arange(batch, device=DEVICE)[:, None] + torch.arange(n, device=DEVICE)).int()
        state["q_out"] = torch.empty(batch, hq, n, d, dtype=dt, device=DEVICE)
        state["k_out"] = torch.empty(batch, hkv, n, d, dtype=dt, device=DEVICE)
    elif c["kind"] == "pack":
        k, v = _kv(g, batch, hkv, c["seq_len"], d)
        state["k"], state["v"] = k.to(dt), v.to(dt)
        order = torch.rand(batch, hkv, c["seq_len"], generator=g, device=DEVICE).argsort(-1)[..., :c["kept"]]
        state["idx"] = order.sort(-1).values.int()
        state["k_out"] = torch.empty(batch, hkv, c["kept"], d, dtype=dt, device=DEVICE)
        state["v_out"] = torch.empty_like(state["k_out"])
    else:
        hq, b, n = c["q_heads"], c["block"], c["cached"]
        tiles = -(-n // TILE)
        cache = torch.empty(batch, hkv, tiles, 34 * d, dtype=torch.uint8, device=DEVICE)
        for i in range(batch if n else 0):
            k, v = _kv(g, 1, hkv, n, d)
            cache[i] = _packed(k.to(dt).float(), v.to(dt).float())[0]
        state["cache"] = cache
        state["q"] = _randn(g, batch, b, hq, d).to(dt).permute(0, 2, 1, 3)
        # the block's keys and values are views of its projection
        x = _randn(g, batch, b, 2 * hkv, d).to(dt).permute(0, 2, 1, 3)
        state["k_blk"], state["v_blk"] = x[:, :hkv], x[:, hkv:]
        state["out"] = torch.empty(batch, b, hq, d, dtype=dt, device=DEVICE).permute(0, 2, 1, 3)
    return state


# ---------------------------------------------------------------- the packed cache, plainly
def _power_of_two(e):
    return ((e + 127) << 23).to(torch.int32).view(torch.float32)


def _groups(x):
    """e of the groups of 32 along the last axis, whether they are finite, and the codes (sign in bit 3)."""
    amax = x.abs().amax(-1, keepdim=True)
    finite = torch.isfinite(amax) & ~torch.isnan(x).any(-1, keepdim=True)
    mantissa, e = torch.frexp(torch.where(finite, amax, 0.0))            # in [0.5, 1)
    e = torch.where(amax == 0, -125, e.int() - 3 + (mantissa >= 0.875).int()).clamp(-125, 125)
    a = torch.where(finite, x.abs() * _power_of_two(-e), 0.0)
    code = ((a > 0.25).byte() + (a >= 0.75).byte() + (a > 1.25).byte() + (a >= 1.75).byte() + (a > 2.5).byte() + (a >= 3.5).byte() + (a > 5).byte())
    return e, finite, code + 8 * (x < 0).byte()


def _rounded(x):
    """The values that groups of 32 along the last axis of x have once they are packed."""
    e, finite, code = _groups(x)
    grid = torch.tensor(GRID + tuple(-v for v in GRID), device=x.device)
    return torch.where(finite, grid[code.long()] * _power_of_two(e), math.nan)


def _rounded_rows(k, v):
    """Rows of keys and values as they are read from the cache: a key's channels by 32, a channel's rows by 32."""
    shape, rows = k.shape, k.shape[2]
    keys = _rounded(k.reshape(*shape[:3], -1, TILE)).reshape(shape)
    v = torch.nn.functional.pad(v, (0, 0, 0, -rows % TILE))
    v = v.reshape(*shape[:2], -1, TILE, shape[3]).transpose(-1, -2).contiguous()
    return keys, _rounded(v).transpose(-1, -2).reshape(*shape[:2], -1, shape[3])[:, :, :rows]


def _bytes_of(codes):
    return codes[..., 0::2] | codes[..., 1::2] << 4


def _scale_bytes(e, finite):
    return torch.where(finite, e + 127, 255).to(torch.uint8)[..., 0]


def _packed(k, v):
    """The cache of rows [B, H, n, d], a tile of 34 d bytes for 32 rows (the last one filled up with zeros):
      key codes     [d / 32 groups of channels][32 keys][16 bytes]
      value codes   [i: d / 64][h: 2][m: 32][16 bytes]: channels (d / 32) m + 2 i + j, j = 0, 1, eight bytes each, whose nibble 4 a + p is
                    row 8 a + 4 h + p of the tile
      key scales    [32 keys][d / 32 groups], value scales [d channels]: bytes e + 127, 255 for a group that is NaN"""
    batch, heads, n, d = k.shape
    k, v = (torch.nn.functional.pad(x, (0, 0, 0, -n % TILE)).reshape(batch, heads, -1, TILE, d) for x in (k, v))
    tiles = k.shape[2]
    e, finite, code = _groups(k.reshape(batch, heads, tiles, TILE, d // 32, 32))
    k_scales = _scale_bytes(e, finite).reshape(batch, heads, tiles, -1)
    k_codes = _bytes_of(code).transpose(3, 4).reshape(batch, heads, tiles, -1)
    e, finite, code = _groups(v.transpose(-1, -2))                       # [.., d, 32 rows]
    v_scales = _scale_bytes(e, finite).reshape(batch, heads, tiles, -1)
    # channels (m, i, j), rows (a, h, p)
    code = code.reshape(batch, heads, tiles, 32, d // 64, 2, 4, 2, 4).permute(0, 1, 2, 4, 7, 3, 5, 6, 8)
    v_codes = _bytes_of(code.reshape(batch, heads, tiles, -1, 16)).reshape(batch, heads, tiles, -1)
    return torch.cat([k_codes, v_codes, k_scales, v_scales], -1)


def _unpacked(cache, n, d):
    """Keys and values [B, H, n, d] that a cache holds, in 32 bits."""
    batch, heads, tiles, _ = cache.shape
    kb, vb, ks, vs = cache.split([TILE * d // 2, TILE * d // 2, d, d], -1)
    grid = torch.tensor(GRID + tuple(-v for v in GRID), device=cache.device)
    scale = lambda s: torch.where(s == 255, math.nan, _power_of_two(s.int() - 127))
    values = lambda b: grid[torch.stack([b & 15, b >> 4], -1).long()].flatten(-2)
    k = values(kb.reshape(batch, heads, tiles, d // 32, TILE, 16)).transpose(3, 4)
    k = k * scale(ks.reshape(batch, heads, tiles, TILE, d // 32, 1))
    v = values(vb.reshape(batch, heads, tiles, d // 64, 2, 32, 2, 8)).reshape(batch, heads, tiles, d // 64, 2, 32, 2, 4, 4)
    v = v.permute(0, 1, 2, 7, 4, 8, 5, 3, 6).reshape(batch, heads, tiles, TILE, d) * scale(vs)[..., None, :]
    return k.reshape(batch, heads, tiles * TILE, d)[:, :, :n], v.reshape(batch, heads, tiles * TILE, d)[:, :, :n]


# ---------------------------------------------------------------- one pass
def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"rope": _own_rope, "pack": _own_pack, "attend": _own_attend}[kind](state)
    return {"rope": _plain_rope, "pack": _plain_pack, "attend": _plain_attend}[kind](state)


def _plain_rope(s):
    c = s["case"]
    angle = s["positions"].double()[:, None, :, None] * s["inv_freq"].double()
    cos, sin = angle.cos().float(), angle.sin().float()

    def one(x, weight):
        dt, x = x.dtype, x.float()
        if c["norm"]:
            x = x * (x.square().mean(-1, keepdim=True) + 1e-6).rsqrt() * weight.float()
        turned, rest = x[..., :c["rot"]], x[..., c["rot"]:]
        if c["pairing"] == "halves":
            a, b = turned.chunk(2, -1)
            turned = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
        else:
            a, b = turned[..., 0::2], turned[..., 1::2]
            turned = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
        return torch.cat([turned, rest], -1).to(dt)

    return one(s["q"], s["q_weight"]), one(s["k"], s["k_weight"])


def _plain_pack(s):
    at = s["idx"].long()[..., None].expand(-1, -1, -1, s["case"]["head_dim"])
    k, v = _rounded_rows(s["k"].gather(2, at).float(), s["v"].gather(2, at).float())
    return k.to(s["k"].dtype), v.to(s["v"].dtype)


def _plain_attend(s):
    c = s["case"]
    batch, hkv, b, d = c["batch"], c["kv_heads"], c["block"], c["head_dim"]
    k, v = _unpacked(s["cache"], c["cached"], d)
    k, v = torch.cat([k, s["k_blk"].float()], 2), torch.cat([v, s["v_blk"].float()], 2)
    q = s["q"].float().reshape(batch, hkv, -1, d)                        # the query heads of a group are neighbours
    logits = torch.matmul(q, k.transpose(-1, -2).contiguous()) / math.sqrt(d)
    p = (logits - logits.amax(-1, keepdim=True)).exp()
    out = torch.matmul(p, v) / p.sum(-1, keepdim=True)
    return out.reshape(batch, c["q_heads"], b, d).to(s["q"].dtype)


def _dtype(B, c):
    return B.SDLLM_BF16 if c["dtype"] == "bf16" else B.SDLLM_F32


def _own_rope(s):
    from paper_2508_02558_amd import binding as B
    if "shape" not in s:
        c = s["case"]
        s["shape"] = B.make_qk_shape(batch=c["batch"], n_q_heads=c["q_heads"], n_kv_heads=c["kv_heads"], head_dim=c["head_dim"], rows=c["rows"],
                                     dtype=_dtype(B, c), rot_dim=c["rot"], norm=B.SDLLM_NORM_RMS if c["norm"] else B.SDLLM_NORM_NONE,
                                     pairing=B.SDLLM_PAIR_HALVES if c["pairing"] == "halves" else B.SDLLM_PAIR_ADJACENT, eps=1e-6,
                                     pos_stride=c["rows"], q_in_stride=B.strides_of(s["q"]), k_in_stride=B.strides_of(s["k"]))
    B.sdllm_qk_norm_rope(s["shape"], s["q"], s["k"], s["q_weight"], s["k_weight"], s["inv_freq"], s["positions"], s["q_out"], s["k_out"])
    return s["q_out"], s["k_out"]


def _own_pack(s):
    from paper_2508_02558_amd import binding as B
    c = s["case"]
    if "shape" not in s:
        # every position of the sequence is a candidate: the block is behind it
        s["shape"] = B.make_shape(batch=c["batch"], n_q_heads=c["kv_heads"], n_kv_heads=c["kv_heads"], head_dim=c["head_dim"], seq_len=c["seq_len"] + 1,
                                  block_off=c["seq_len"], block_len=1, dtype=_dtype(B, c), retention=c["kept"] / c["seq_len"],
                                  kv_stride=B.strides_of(s["k"]), cache_stride=B.strides_of(s["k_out"]))
        s["cache"] = torch.empty(B.sdllm_packed_cache_bytes(s["shape"], c["kept"]), dtype=torch.uint8, device=DEVICE)
    B.sdllm_compact_kv_packed(s["shape"], s["k"], s["v"], s["idx"], s["cache"], c["kept"])
    B.sdllm_unpack_kv(s["shape"], s["cache"], c["kept"], c["kept"], s["k_out"], s["v_out"])
    return s["k_out"], s["v_out"]


def _own_attend(s):
    from paper_2508_02558_amd import binding as B
    c = s["case"]
    if "shape" not in s:
        s["shape"] = B.make_shape(batch=c["batch"], n_q_heads=c["q_heads"], n_kv_heads=c["kv_heads"], head_dim=c["head_dim"],
                                  seq_len=c["cached"] + c["block"], block_off=c["cached"], block_len=c["block"], dtype=_dtype(B, c),
                                  q_stride=B.strides_of(s["q"]), blk_stride=B.strides_of(s["k_blk"]), out_stride=B.strides_of(s["out"]))
        s["ws"] = torch.empty(B.sdllm_workspace_bytes(s["shape"], B.SDLLM_OP_SPARSE_ATTN_PACKED, c["cached"]), dtype=torch.uint8, device=DEVICE)
    B.sdllm_sparse_attn_packed(s["shape"], s["q"], s["cache"], c["cached"], c["cached"], s["k_blk"], s["v_blk"], s["out"], s["ws"])
    return s["out"]


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    c, d = case, case["head_dim"]
    es = 2 if c["dtype"] == "bf16" else 4
    rows_kv = c["batch"] * c["kv_heads"]
    if c["kind"] == "rope":
        n = c["batch"] * (c["q_heads"] + c["kv_heads"]) * c["rows"] * d
        return dict(bytes=2 * n * es + 4 * c["batch"] * c["rows"] + 2 * c["rot"], flops=10 * n)
    if c["kind"] == "pack":
        n = 2 * rows_kv * c["kept"] * d
        # rows in, cache out, values out
        return dict(bytes=n * es + 4 * rows_kv * c["kept"] + n * 17 // 32 + n * es, flops=6 * n)
    cached, b = c["cached"], c["block"]
    q = c["batch"] * c["q_heads"] * b * d
    return dict(bytes=2 * q * es + 2 * rows_kv * b * d * es + 2 * rows_kv * cached * d * 17 // 32, flops=4 * q * (cached + b))


# ---------------------------------------------------------------- the same from the definitions, in 64 bits
def exact(case, seed):
    s, c, d = prepare(case, seed), case, case["head_dim"]

    def nearest(x, axis):
        """Values of one group along `axis`, from the definition: smallest e with all magnitudes below 7 2^e, nearest number, ties to the even code."""
        top = x.abs().amax(axis, keepdim=True)
        e = torch.floor(torch.log2(torch.clamp(top, min=2.0 ** -130) / 7))
        e = torch.where(top >= 7 * 2.0 ** e, e + 1, e)
        e = torch.where(top >= 7 * 2.0 ** e, e + 1, e).clamp(-125, 125)
        best, off = torch.zeros_like(x), x.abs() / 2.0 ** e
        far = off.clone()
        for code in (2, 4, 6, 1, 3, 5, 7):                                   # odd codes have to be nearer than the even ones
            away = (off - GRID[code]).abs()
            best, far = torch.where(away < far, GRID[code], best), torch.minimum(away, far)
        return torch.sign(x) * best * 2.0 ** e

    if c["kind"] == "rope":
        # a pair as a complex number, turned by exp(i angle)
        turn = torch.polar(torch.ones(c["batch"], 1, c["rows"], c["rot"] // 2, dtype=torch.float64, device=DEVICE),
                           s["positions"].to(torch.float64)[:, None, :, None] * s["inv_freq"].to(torch.float64))
        got = []
        for x, w in ((s["q"], s["q_weight"]), (s["k"], s["k_weight"])):
            x = x.to(torch.float64)
            if c["norm"]:
                x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / d + 1e-6) * w.to(torch.float64)
            half = c["rot"] // 2
            first = torch.arange(half, device=DEVICE) * (1 if c["pairing"] == "halves" else 2)
            second = first + (half if c["pairing"] == "halves" else 1)
            z = torch.complex(x[..., first], x[..., second]) * turn
            x[..., first], x[..., second] = z.real, z.imag
            got.append(x)
        return tuple(got)
    if c["kind"] == "pack":
        pick = lambda x: torch.take_along_dim(x.to(torch.float64), s["idx"].to(torch.int64)[..., None], 2)
        k, v = pick(s["k"]), pick(s["v"])
        for j in range(0, d, 32):
            k[..., j:j + 32] = nearest(k[..., j:j + 32], 3)
        for r in range(0, c["kept"], 32):
            v[:, :, r:r + 32] = nearest(v[:, :, r:r + 32], 2)
        return k, v
    # attention: every byte of the cache by a table of its two values
    n, tiles, g = c["cached"], s["cache"].shape[2], c["q_heads"] // c["kv_heads"]
    number = lambda code: (-1.0 if code & 8 else 1.0) * (0.5 * (code & 1) if code & 7 < 2 else (1 + 0.5 * (code & 1)) * 2.0 ** ((code >> 1 & 3) - 1))
    table = torch.tensor([[number(x & 15), number(x >> 4)] for x in range(256)], dtype=torch.float64, device=DEVICE)
    step = torch.tensor([2.0 ** (x - 127) for x in range(255)] + [math.nan], dtype=torch.float64, device=DEVICE)
    at = torch.arange(d, device=DEVICE)
    row = torch.arange(TILE, device=DEVICE)
    # byte and nibble of every (row, channel) within a tile
    kn = (at[None] // 32 * TILE + row[:, None]) * 32 + at[None] % 32
    per = d // 32
    m, i, j = at // per, at % per // 2, at % 2
    a, h, p = row // 8, row // 4 % 2, row % 4
    vn = (((i[None] * 2 + h[:, None]) * 32 + m[None]) * 2 + j[None]) * 16 + 4 * a[:, None] + p[:, None]
    flat = s["cache"].to(torch.int64)
    kv = []
    for base, nibble, scale_at in ((0, kn, TILE * d + row[:, None] * per + at[None] // 32), (16 * d, vn, TILE * d + d + at[None].expand(TILE, d))):
        x = table[flat[..., base:base + 16 * d]].flatten(-2)[..., nibble.flatten()] * step[flat[..., scale_at.flatten()]]
        kv.append(x.reshape(c["batch"], c["kv_heads"], tiles * TILE, d)[:, :, :n])
    k = torch.cat([kv[0], s["k_blk"].to(torch.float64)], 2)
    v = torch.cat([kv[1], s["v_blk"].to(torch.float64)], 2)
    q = s["q"].to(torch.float64)
    out = torch.empty(q.shape, dtype=torch.float64, device=DEVICE)
    for x in range(c["q_heads"]):
        w = torch.softmax(torch.matmul(q[:, x], k[:, x // g].transpose(-1, -2).contiguous()) * d ** -0.5, -1)
        out[:, x] = torch.matmul(w, v[:, x // g])
    return out
