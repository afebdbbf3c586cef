"""Packing and unpacking of the cache of 4 bits a value against the float64 oracle: exact, byte by byte."""
import numpy as np
import pytest
import torch

from oracle import packed_oracle as po
from paper_2508_02558_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = {"bf16": (torch.bfloat16, B.SDLLM_BF16), "f32": (torch.float32, B.SDLLM_F32)}


def host(t):
    return t.detach().cpu().double().numpy()


def make(Bt, H, L, kept, d, dtype, k, v, idx, cache_rows=None, cache=None, stream=None):
    """Packs rows idx of k and v; returns (cache bytes [B, H, tiles, 34 d], unpacked k, v)."""
    td, code = TYPES[dtype]
    cache_rows = kept if cache_rows is None else cache_rows
    s = B.make_shape(batch=Bt, n_q_heads=H, n_kv_heads=H, head_dim=d, seq_len=L + 1, block_off=L, block_len=1, dtype=code, retention=kept / L,
                     kv_stride=B.strides_of(k), cache_rows=max(1, kept))
    assert B.sdllm_retained_count(s)[0] == kept
    if cache is None:
        cache = torch.full((B.sdllm_packed_cache_bytes(s, cache_rows),), 0xA5, dtype=torch.uint8, device=DEV)
    B.sdllm_compact_kv_packed(s, k, v, idx, cache, cache_rows, stream)
    ko, vo = (torch.full((Bt, H, kept, d), 7.0, dtype=td, device=DEV) for _ in range(2))
    B.sdllm_unpack_kv(s, cache, cache_rows, kept, ko, vo, stream)
    torch.cuda.synchronize()
    tiles = -(-cache_rows // 32)
    return cache[:Bt * H * tiles * 34 * d].reshape(Bt, H, tiles, 34 * d).cpu().numpy(), ko, vo


def rows_of(Bt, H, L, kept, g):
    return torch.rand(Bt, H, L, generator=g).argsort(-1)[..., :kept].sort(-1).values.int().to(DEV)


def check(k, v, idx, got, dtype, all_bytes=True):
    cache, ko, vo = got
    Bt, H, kept = idx.shape
    pick = idx.cpu().long()[..., None].expand(-1, -1, -1, k.shape[-1])
    kr, vr = (host(x.cpu().gather(2, pick)) for x in (k, v))
    kw, vw = po.cache_values(kr, vr)
    assert np.array_equal(host(ko), kw, equal_nan=True)
    assert np.array_equal(host(vo), vw, equal_nan=True)
    if all_bytes:
        for b in range(Bt):
            for h in range(H):
                want = po.cache_bytes(kr[b, h], vr[b, h])
                assert np.array_equal(cache[b, h, :len(want)], want), (b, h)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Bt,H,L,kept", [(1, 1, 1, 1), (1, 2, 40, 31), (2, 1, 64, 32), (1, 3, 50, 33), (2, 2, 200, 77), (1, 1, 700, 700)])
def test_rows_and_bytes(dtype, d, Bt, H, L, kept):
    g = torch.Generator().manual_seed(L + kept)
    td = TYPES[dtype][0]
    k, v = (torch.randn(Bt, H, L, d, generator=g).mul(torch.exp(2 * torch.randn(Bt, H, L, 1, generator=g))).to(td).to(DEV) for _ in range(2))
    idx = rows_of(Bt, H, L, kept, g)
    check(k, v, idx, make(Bt, H, L, kept, d, dtype, k, v, idx), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_ties_ends_of_the_range_and_what_is_not_finite(dtype, d):
    td = TYPES[dtype][0]
    n = 40
    g = torch.Generator().manual_seed(3)
    k = torch.randn(1, 1, n, d, generator=g)
    v = torch.randn(1, 1, n, d, generator=g)
    ties = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 6.5, -0.25, -0.75, -1.25, -1.75, -2.5, -3.5, -5.0, -0.0])
    for e, row in ((0, 0), (-7, 1), (40, 2), (-100, 3)):
        k[0, 0, row, :17] = ties * 2.0 ** e
        k[0, 0, row, 17:32] = 0
        v[0, 0, :17, row] = ties * 2.0 ** e
        v[0, 0, 17:32, row] = 0
    k[0, 0, 4] = 0
    v[0, 0, :, 4] = 0
    top = torch.finfo(td).max
    for row, value in ((5, 7.0), (6, -7.0), (7, 6.96875), (8, 14.0), (9, 2.0 ** -126), (10, 2.0 ** -131), (11, top), (12, -top), (13, 1.75 * 2.0 ** 127),
                       (14, 7 * 2.0 ** -125), (15, 3.5 * 2.0 ** -125)):
        k[0, 0, row, 3] = value
        k[0, 0, row, 32 + 31] = value
        v[0, 0, 31, row] = value
        v[0, 0, 33, row] = value
    for row, value in ((16, float("inf")), (17, float("-inf")), (18, float("nan"))):
        k[0, 0, row, 9] = value
        v[0, 0, 35, row] = value
    k, v = k.to(td).to(DEV), v.to(td).to(DEV)
    idx = torch.arange(n, dtype=torch.int32, device=DEV)[None, None].contiguous()
    got = make(1, 1, n, n, d, dtype, k, v, idx)
    check(k, v, idx, got, dtype, all_bytes=False)
    assert np.isnan(host(got[1])[0, 0, 16:19, :32]).all() and np.isfinite(host(got[1])[0, 0, 16:19, 32:]).all()


def test_strides_capacity_and_order_of_rows():
    # rows of [B, L, H, 2 d] tensors, a cache with room for more rows than are kept, and rows picked in no order, some twice
    Bt, H, L, d, kept, room = 2, 3, 90, 128, 45, 200
    g = torch.Generator().manual_seed(5)
    both = torch.randn(Bt, L, H, 2 * d, generator=g).bfloat16().to(DEV)
    k, v = both[..., :d].permute(0, 2, 1, 3), both[..., d:].permute(0, 2, 1, 3)
    idx = torch.randint(0, L, (Bt, H, kept), generator=g, dtype=torch.int32).to(DEV)
    got = make(Bt, H, L, kept, d, "bf16", k, v, idx, cache_rows=room)
    check(k, v, idx, got, "bf16")
    assert (got[0][:, :, 2:] == 0xA5).all()                      # tiles past the kept rows are not written
    # fewer rows of the same cache, into rows with strides of their own
    s = B.make_shape(batch=Bt, n_q_heads=H, n_kv_heads=H, head_dim=d, seq_len=L + 1, block_off=L, block_len=1, dtype=B.SDLLM_BF16)
    wide = torch.zeros(Bt, 40, H, 2 * d, dtype=torch.bfloat16, device=DEV)
    ko, vo = wide[..., :d].permute(0, 2, 1, 3), wide[..., d:].permute(0, 2, 1, 3)
    s.cache_stride[:] = B.strides_of(ko)
    B.sdllm_unpack_kv(s, torch.from_numpy(got[0].reshape(-1)).to(DEV), room, 37, ko, vo)
    torch.cuda.synchronize()
    assert torch.equal(ko[:, :, :37], got[1][:, :, :37]) and torch.equal(vo[:, :, :37], got[2][:, :, :37]) and not wide[:, 37:].any()


def test_heads_beyond_2_gib_of_cache():
    # the second head starts 2.3 GB on
    L, kept, d, room = 64, 50, 128, 17_000_000
    g = torch.Generator().manual_seed(6)
    k, v = (torch.randn(1, 2, L, d, generator=g).bfloat16().to(DEV) for _ in range(2))
    idx = rows_of(1, 2, L, kept, g)
    s = B.make_shape(batch=1, n_q_heads=2, n_kv_heads=2, head_dim=d, seq_len=L + 1, block_off=L, block_len=1, dtype=B.SDLLM_BF16, retention=kept / L,
                     kv_stride=B.strides_of(k), cache_rows=kept)
    cache = torch.empty(B.sdllm_packed_cache_bytes(s, room), dtype=torch.uint8, device=DEV)
    assert cache.numel() > 2 * (1 << 31)
    B.sdllm_compact_kv_packed(s, k, v, idx, cache, room)
    ko, vo = (torch.zeros(1, 2, kept, d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    B.sdllm_unpack_kv(s, cache, room, kept, ko, vo)
    near = make(1, 2, L, kept, d, "bf16", k, v, idx)
    assert torch.equal(ko, near[1]) and torch.equal(vo, near[2])


def test_another_stream_waits_for_nothing_else():
    L, kept, d = 300, 150, 128
    g = torch.Generator().manual_seed(7)
    k, v = (torch.randn(1, 2, L, d, generator=g).bfloat16().to(DEV) for _ in range(2))
    idx = rows_of(1, 2, L, kept, g)
    want = make(1, 2, L, kept, d, "bf16", k, v, idx)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = make(1, 2, L, kept, d, "bf16", k, v, idx, stream=side)
    assert np.array_equal(got[0], want[0]) and torch.equal(got[1], want[1])
