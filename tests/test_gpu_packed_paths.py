"""Every form in which attention over the packed cache is launched, asked for by its plan, against the float64 oracle."""
import pytest
import torch

from paper_2508_02558_amd import binding as B
from tests.test_gpu_attn_packed import DEV, TYPES, Call, compare, host

pytestmark = pytest.mark.gpu


def plan_of(shape, n):
    p = B.sdllm_packed_plan(shape, n)
    return p.key_splits, p.waves, p.rounds, p.past_caches


# (batch, query heads, KV heads, head_dim, block), rows, type: (key splits, wavefronts, rounds, past the caches)
@pytest.mark.parametrize("sizes,n,dtype,plan", [
    ((1, 28, 4, 128, 32), 8312, "bf16", (7, 8, 5, 0)), ((1, 28, 4, 64, 32), 8312, "bf16", (7, 8, 5, 0)), ((1, 16, 16, 128, 32), 6001, "bf16", (8, 7, 4, 0)),
    ((1, 32, 32, 128, 32), 4000, "f32", (8, 4, 5, 0)), ((1, 64, 64, 64, 20), 1290, "f32", (4, 4, 3, 0)),
    ((1, 300, 300, 128, 4), 700, "bf16", (1, 4, 6, 0)), ((1, 300, 300, 64, 4), 700, "bf16", (1, 8, 3, 0)), ((3, 200, 100, 128, 33), 900, "bf16", (1, 4, 8, 0)),
    ((1, 300, 300, 128, 2), 700, "f32", (1, 4, 6, 0)), ((1, 64, 64, 128, 32), 1290, "bf16", (1, 7, 6, 0)), ((1, 64, 64, 64, 32), 1290, "bf16", (1, 7, 6, 0))])
def test_splits_rounds_and_wavefronts(sizes, n, dtype, plan):
    Bt, Hq, Hkv, d, b = sizes
    c = Call(Bt, Hq, Hkv, d, b, n, dtype)
    assert plan_of(c.shape, n) == plan
    c.run()
    c.check()


# 128 MiB and more: some heads against the oracle, on the values that unpacking gives
@pytest.mark.parametrize("sizes,n,plan", [
    ((8, 32, 32, 64, 32), 7730, (1, 8, 31, 1)), ((16, 32, 32, 128, 32), 2000, (1, 4, 16, 1)), ((64, 64, 64, 128, 1), 250, (1, 3, 3, 1)),
    ((7, 28, 4, 128, 4), 38401, (8, 8, 19, 1))])
def test_past_the_caches(sizes, n, plan):
    Bt, Hq, Hkv, d, b = sizes
    g = torch.Generator(device=DEV).manual_seed(n)
    new = lambda heads, rows: torch.randn(Bt, heads, rows, d, generator=g, device=DEV).bfloat16()
    k, v, q, kb, vb = new(Hkv, n), new(Hkv, n), new(Hq, b), new(Hkv, b), new(Hkv, b)
    s = B.make_shape(batch=Bt, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=d, seq_len=n + b, block_off=n, block_len=b, dtype=TYPES["bf16"][1], retention=1.0,
                     kv_stride=B.strides_of(k), cache_rows=n)
    assert plan_of(s, n) == plan
    cache = torch.empty(B.sdllm_packed_cache_bytes(s, n), dtype=torch.uint8, device=DEV)
    idx = torch.arange(n, dtype=torch.int32, device=DEV).expand(Bt, Hkv, n).contiguous()
    B.sdllm_compact_kv_packed(s, k, v, idx, cache, n)
    out = torch.full_like(q, float("nan"))
    ws = torch.empty(B.sdllm_workspace_bytes(s, B.SDLLM_OP_SPARSE_ATTN_PACKED, n), dtype=torch.uint8, device=DEV)
    B.sdllm_sparse_attn_packed(s, q, cache, n, n, kb, vb, out, ws)
    B.sdllm_unpack_kv(s, cache, n, n, k, v)
    torch.cuda.synchronize()
    assert torch.isfinite(out).all()
    G = Hq // Hkv
    for x, h in ((0, 0), (Bt // 2, Hkv // 2), (Bt - 1, Hkv - 1)):
        kv, rows = (lambda t: t[x:x + 1, h:h + 1]), (lambda t: t[x:x + 1, G * h:G * h + G])
        compare(rows(out), rows(q), host(kv(k)), host(kv(v)), kv(kb), kv(vb), d ** -0.5, "bf16")
