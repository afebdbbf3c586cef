"""Attention over a cache of 4 bits a value against the float64 oracle on the values that the cache stands for."""
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


def rows_last(Bt, H, n, d, g, td, packed):
    """[B, H, n, d], dense or as rows of a [B, n, 2 H, d] tensor."""
    if not packed:
        return torch.randn(Bt, H, n, d, generator=g).to(td).to(DEV)
    return torch.randn(Bt, n, 2 * H, d, generator=g).to(td).to(DEV).permute(0, 2, 1, 3)[:, 1:1 + H]


class Call:
    def __init__(self, Bt, Hq, Hkv, d, b, n, dtype, room=None, seed=0, strided=False, edit=None, scale=0.0):
        td, code = TYPES[dtype]
        g = torch.Generator().manual_seed(seed + 1000 * n + b)
        self.n, self.dtype, self.Hq, self.Hkv, self.room = n, dtype, Hq, Hkv, n if room is None else room
        k, v = (torch.randn(Bt, Hkv, max(1, n), d, generator=g) for _ in range(2))
        self.q = rows_last(Bt, Hq, b, d, g, td, strided)
        self.kb, self.vb = rows_last(Bt, Hkv, b, d, g, td, strided), rows_last(Bt, Hkv, b, d, g, td, strided)
        if edit:
            edit(k, v, self)
        k, v = k.to(td).to(DEV), v.to(td).to(DEV)
        self.out = torch.full((Bt, b, Hq, d), float("nan"), dtype=td, device=DEV).permute(0, 2, 1, 3) if strided \
            else torch.full((Bt, Hq, b, d), float("nan"), dtype=td, device=DEV)
        self.scale = scale or d ** -0.5
        self.shape = B.make_shape(batch=Bt, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=d, seq_len=max(1, n) + b, block_off=max(1, n), block_len=b, dtype=code,
                                  retention=1.0, softmax_scale=scale, q_stride=B.strides_of(self.q), blk_stride=B.strides_of(self.kb),
                                  kv_stride=B.strides_of(k), out_stride=B.strides_of(self.out))
        self.cache = None
        if n:
            idx = torch.arange(n, dtype=torch.int32, device=DEV).expand(Bt, Hkv, n).contiguous()
            self.cache = torch.full((B.sdllm_packed_cache_bytes(self.shape, self.room),), 0xFF, dtype=torch.uint8, device=DEV)
            B.sdllm_compact_kv_packed(self.shape, k, v, idx, self.cache, self.room)
        self.kc, self.vc = po.cache_values(host(k)[:, :, :n], host(v)[:, :, :n])
        self.ws = torch.empty(B.sdllm_workspace_bytes(self.shape, B.SDLLM_OP_SPARSE_ATTN_PACKED, n), dtype=torch.uint8, device=DEV)

    def run(self, stream=None):
        B.sdllm_sparse_attn_packed(self.shape, self.q, self.cache, self.room, self.n, self.kb, self.vb, self.out, self.ws, stream)

    def check(self):
        torch.cuda.synchronize()
        compare(self.out, self.q, self.kc, self.vc, self.kb, self.vb, self.scale, self.dtype)


def compare(out, q, kc, vc, kb, vb, scale, dtype):
    """out [B, Hq, b, d] against attention of q over rows kc, vc (float64, [B, Hkv, n, d]) and kb, vb."""
    got, q, kb, vb = (host(x) for x in (out, q, kb, vb))
    d, G = q.shape[-1], q.shape[1] // kb.shape[1]
    for b in range(q.shape[0]):
        for h in range(q.shape[1]):
            k = np.concatenate([kc[b, h // G], kb[b, h // G]])
            v = np.concatenate([vc[b, h // G], vb[b, h // G]])
            want, mean = po.attention(q[b, h], k, v, scale)
            # fp32: a logit is a sum of d products and a multiple of log2(e); a probability is off by as much, relatively, and by the
            # exponential's two steps; the sums over the keys add half a step a term
            u = 2.0 ** -24
            logit = (np.abs(q[b, h]) @ np.abs(k).T).max(-1, keepdims=True) * scale
            p = (d + 8) * u * logit + 4 * u
            # and no result or numerator below the smallest normal number can be held
            tol = (2 * p + (len(k) + 8) * 2 * u) * mean + u * np.abs(want) + len(k) * np.abs(v).max() * 2.0 ** -126
            if dtype == "bf16":
                tol = tol + 2.0 ** -8 * mean + 2.0 ** -8 * np.abs(want)      # numerators and the result are rounded to bf16
            assert np.array_equal(np.isnan(got[b, h]), np.isnan(want)), (b, h)
            err = np.abs(got[b, h] - want)
            ok = np.isnan(want) | (err <= tol)
            assert ok.all(), (b, h, float(np.nanmax(err / tol)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Hq,Hkv,b", [(2, 2, 32), (7, 1, 32), (4, 2, 1), (8, 1, 1), (16, 2, 7), (3, 3, 33), (2, 1, 64), (6, 2, 31)])
@pytest.mark.parametrize("n", [0, 1, 31, 32, 33, 100, 517])
def test_against_the_oracle(dtype, d, Hq, Hkv, b, n):
    c = Call(1 if n > 100 else 2, Hq, Hkv, d, b, n, dtype)
    c.run()
    c.check()


# more key splits than one, and enough columns that there is one
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("Bt,Hq,Hkv,b,n", [(1, 1, 1, 32, 4099), (1, 4, 1, 32, 2500), (1, 16, 16, 5, 1300), (2, 14, 2, 1, 6001), (1, 300, 300, 2, 150),
                                           (9, 32, 32, 1, 40)])
def test_splits_and_full_grids(dtype, d, Bt, Hq, Hkv, b, n):
    c = Call(Bt, Hq, Hkv, d, b, n, dtype)
    c.run()
    c.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_strides_and_capacity(dtype, d):
    c = Call(2, 6, 3, d, 37, 300, dtype, room=1000, strided=True)
    c.run()
    c.check()


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("where", [0, 40, 699, "block"])
def test_one_key_takes_nearly_all(dtype, d, where):
    # a maximum that comes late moves the reference of sums that are under way
    def edit(k, v, c):
        q = c.q.float().cpu()
        if where == "block":
            c.kb[:, :, -1] = (q[:, :, 0] * 3).to(c.kb.dtype).to(DEV)
        else:
            k[:, :, where] = q[:, :, 0] * 3
    c = Call(1, 2, 2, d, 32, 700, dtype, edit=edit, scale=0.5)
    c.run()
    c.check()


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128)])
def test_what_is_not_finite_stays_with_its_heads(dtype, d):
    def edit(k, v, c):
        k[0, 0, 50, 3] = float("inf")        # every query of head 0
        v[0, 1, 70, 5] = float("nan")        # channel 5 of head 1
        c.vb[0, 2, 1, 7] = float("inf")      # channel 7 of head 2
    c = Call(1, 4, 4, d, 8, 130, dtype, edit=edit)
    c.run()
    torch.cuda.synchronize()
    out = host(c.out)
    assert np.isnan(out[0, 0]).all()
    assert np.isnan(out[0, 1, :, 5]).all() and np.isfinite(np.delete(out[0, 1], 5, -1)).all()
    assert np.isposinf(out[0, 2, :, 7]).all() and np.isfinite(np.delete(out[0, 2], 7, -1)).all()
    assert np.isfinite(out[0, 3]).all()


def test_what_lies_past_the_rows_is_not_read_as_rows():
    # the cache around the rows is NaN, and so are the block tensors around the block
    c = Call(1, 4, 2, 128, 5, 70, "bf16", room=256)
    wide = torch.full((1, 2, 40, 128), float("nan"), dtype=torch.bfloat16, device=DEV)
    wk, wv = wide.clone(), wide.clone()
    wk[:, :, :5], wv[:, :, :5] = c.kb, c.vb
    c.kb, c.vb = wk[:, :, :5], wv[:, :, :5]
    c.shape.blk_stride[:] = B.strides_of(c.kb)
    c.run()
    c.check()


def test_another_stream_and_twice_the_same():
    c = Call(1, 8, 1, 128, 32, 3000, "bf16")
    c.run()
    c.check()
    first = c.out.clone()
    c.out.fill_(0)
    c.ws.fill_(0xFF)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    c.run(side)
    torch.cuda.synchronize()
    assert torch.equal(c.out, first)


def test_a_cache_that_is_read_past_the_caches():
    # 148 MB; three heads of it against the oracle, on the values that unpacking gives
    Bt, H, n, d = 8, 32, 4250, 128
    g = torch.Generator(device=DEV).manual_seed(1)
    k, v = (torch.randn(Bt, H, n, d, generator=g, device=DEV).bfloat16() for _ in range(2))
    q, kb, vb = (torch.randn(Bt, H, 32, d, generator=g, device=DEV).bfloat16() for _ in range(3))
    s = B.make_shape(batch=Bt, n_q_heads=H, n_kv_heads=H, head_dim=d, seq_len=n + 32, block_off=n, block_len=32, dtype=B.SDLLM_BF16, retention=1.0,
                     kv_stride=B.strides_of(k), cache_rows=n)
    cache = torch.empty(B.sdllm_packed_cache_bytes(s, n), dtype=torch.uint8, device=DEV)
    assert cache.numel() > 128 << 20
    idx = torch.arange(n, dtype=torch.int32, device=DEV).expand(Bt, H, n).contiguous()
    B.sdllm_compact_kv_packed(s, k, v, idx, cache, n)
    out = torch.full_like(q, float("nan"))
    ws = torch.empty(B.sdllm_workspace_bytes(s, B.SDLLM_OP_SPARSE_ATTN_PACKED, n), dtype=torch.uint8, device=DEV)
    B.sdllm_sparse_attn_packed(s, q, cache, n, n, kb, vb, out, ws)
    B.sdllm_unpack_kv(s, cache, n, n, k, v)
    torch.cuda.synchronize()
    assert torch.isfinite(out).all()
    for b, h in ((0, 0), (3, 17), (7, 31)):
        one = lambda t: t[b:b + 1, h:h + 1]
        compare(one(out), one(q), host(one(k)), host(one(v)), one(kb), one(vb), d ** -0.5, "bf16")


def test_in_a_graph():
    c = Call(1, 8, 1, 128, 32, 3000, "bf16")
    c.run()
    torch.cuda.synchronize()
    want = c.out.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.run()
    for _ in range(3):
        c.out.fill_(0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(c.out, want)


@pytest.mark.parametrize("Hq,Hkv,d,b,dtype,prompt", [(4, 4, 128, 32, "bf16", 600), (7, 1, 128, 32, "bf16", 2000), (4, 2, 64, 16, "f32", 200),
                                                     (2, 2, 128, 64, "bf16", 500)])
def test_block_step_runs_the_states(Hq, Hkv, d, b, dtype, prompt):
    td, code = TYPES[dtype]
    L, o = prompt + 3 * b, prompt + b
    g = torch.Generator().manual_seed(prompt)
    q, kf, vf = (torch.randn(1, h, n, d, generator=g).to(td).to(DEV) for h, n in ((Hq, b), (Hkv, L), (Hkv, L)))
    kn, vn = (torch.randn(1, Hkv, b, d, generator=g).to(td).to(DEV) for _ in range(2))
    shape = B.make_shape(batch=1, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=d, seq_len=L, block_off=o, block_len=b, dtype=code)
    kept = B.sdllm_retained_count(shape)[0]
    ws = torch.empty(max(B.sdllm_workspace_bytes(shape, op) for op in (B.SDLLM_OP_BLOCK_STEP, B.SDLLM_OP_BLOCK_STEP_PACKED)), dtype=torch.uint8, device=DEV)
    new = lambda *s: torch.zeros(*s, dtype=td, device=DEV)
    idx, idx_p = (torch.zeros(1, Hkv, kept, dtype=torch.int32, device=DEV) for _ in range(2))
    kc, vc, out, out_p = new(1, Hkv, L - b, d), new(1, Hkv, L - b, d), new(1, Hq, b, d), new(1, Hq, b, d)
    cache = torch.zeros(B.sdllm_packed_cache_bytes(shape, kept), dtype=torch.uint8, device=DEV)
    for step in (0, 1):
        assert B.sdllm_block_step(shape, step, 1, q, kf, vf, idx, kc, vc, out, ws) == step
        assert B.sdllm_block_step_packed(shape, step, 1, q, kf, vf, idx_p, cache, kept, out_p, ws) == step
        torch.cuda.synchronize()
        assert torch.equal(out, out_p), step                     # the same dense rows
    assert torch.equal(idx, idx_p)
    ko, vo = new(1, Hkv, L - b, d), new(1, Hkv, L - b, d)
    B.sdllm_unpack_kv(shape, cache, kept, kept, ko, vo)
    torch.cuda.synchronize()
    want = po.cache_values(host(kc)[:, :, :kept], host(vc)[:, :, :kept])
    assert np.array_equal(host(ko)[:, :, :kept], want[0]) and np.array_equal(host(vo)[:, :, :kept], want[1])
    assert B.sdllm_block_step_packed(shape, 2, 1, q, kn, vn, idx_p, cache, kept, out_p, ws) == 2
    again = torch.zeros_like(out_p)
    B.sdllm_sparse_attn_packed(shape, q, cache, kept, kept, kn, vn, again, ws)
    torch.cuda.synchronize()
    assert torch.equal(again, out_p)
    compare(out_p, q, want[0], want[1], kn, vn, d ** -0.5, dtype)


# ---- heads enough that keys are not split over workgroups, and more than three tiles for each wavefront: the queries go through two 8-bit numbers
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Bt,Hq,Hkv,b,n", [(1, 64, 64, 32, 1290), (2, 64, 32, 7, 1500), (1, 260, 65, 1, 1111), (1, 128, 64, 33, 1024)])
def test_many_tiles_for_each_wavefront(d, Bt, Hq, Hkv, b, n):
    c = Call(Bt, Hq, Hkv, d, b, n, "bf16")
    c.run()
    c.check()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("where", [0, 700, 1289])
def test_one_key_of_many_tiles_takes_nearly_all(d, where):
    def edit(k, v, c):
        k[:, :, where] = c.q.float().cpu()[:, :, 0] * 3
    c = Call(1, 64, 64, d, 32, 1290, "bf16", edit=edit, scale=0.5)
    c.run()
    c.check()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Hkv,n", [(2, 200), (64, 1290)])
def test_queries_with_channels_of_unlike_size_and_an_infinite_one(d, Hkv, n):
    def edit(k, v, c):
        c.q[:, :, :, 5] *= 64
        c.q[:, :, :, 40:44] *= 2.0 ** -12
        c.q[:, :, 3] *= 2.0 ** -100
        c.q[0, 1, 6, 2] = float("inf")
    c = Call(1, Hkv, Hkv, d, 9, n, "bf16", edit=edit, scale=0.02)
    c.run()
    c.q[0, 1, 6, 2] = 1.0                    # the oracle's; that row has to be NaN
    torch.cuda.synchronize()
    assert torch.isnan(c.out[0, 1, 6]).all()
    again = c.out.clone()
    c.run()
    torch.cuda.synchronize()
    again[0, 1, 6] = c.out[0, 1, 6]
    assert torch.equal(again, c.out)         # and no other row has anything of it
    c.check()


@pytest.mark.parametrize("d", [64, 128])
def test_what_is_not_finite_in_many_tiles(d):
    def edit(k, v, c):
        k[0, 0, 1250, 3] = float("inf")      # every query of head 0
        v[0, 1, 1270, 5] = float("nan")      # channel 5 of head 1
        c.vb[0, 2, 1, 7] = float("inf")      # channel 7 of head 2
    c = Call(1, 64, 64, d, 8, 1290, "bf16", edit=edit)
    c.run()
    torch.cuda.synchronize()
    out = host(c.out)
    assert np.isnan(out[0, 0]).all()
    assert np.isnan(out[0, 1, :, 5]).all() and np.isfinite(np.delete(out[0, 1], 5, -1)).all()
    assert np.isposinf(out[0, 2, :, 7]).all() and np.isfinite(np.delete(out[0, 2], 7, -1)).all()
    assert np.isfinite(out[0, 3:]).all()
