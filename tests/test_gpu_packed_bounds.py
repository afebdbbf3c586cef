"""What an index buffer or a size may not do to the operators of the packed cache."""
import numpy as np
import pytest
import torch

from oracle import packed_oracle as po
from paper_2508_02558_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = {"bf16": (torch.bfloat16, B.SDLLM_BF16), "f32": (torch.float32, B.SDLLM_F32)}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_packing_stays_within_the_rows_whatever_the_indices_are(dtype, d):
    # the tensors lie between rows of NaN, so that a neighbouring row would show
    td, code = TYPES[dtype]
    Bt, H, L, kept = 2, 3, 50, 37
    g = torch.Generator().manual_seed(d)
    k, v = (torch.full((Bt, H, L + 2, d), float("nan"), dtype=td, device=DEV) for _ in range(2))
    for t in (k, v):
        t[:, :, 1:-1] = torch.randn(Bt, H, L, d, generator=g).to(td).to(DEV)
    k, v = k[:, :, 1:-1], v[:, :, 1:-1]
    idx = torch.randint(0, L, (Bt, H, kept), generator=g, dtype=torch.int32)
    idx[0, 0, 0], idx[0, 1, 5], idx[0, 2, 31], idx[1, 0, 32], idx[1, 2, 36] = -1, L, -2 ** 31, 2 ** 31 - 1, L + 1
    s = B.make_shape(batch=Bt, n_q_heads=H, n_kv_heads=H, head_dim=d, seq_len=L, block_off=L - 1, block_len=1, dtype=code, retention=kept / (L - 1),
                     kv_stride=B.strides_of(k), cache_rows=kept)
    assert B.sdllm_retained_count(s)[0] == kept
    cache = torch.zeros(B.sdllm_packed_cache_bytes(s, kept), dtype=torch.uint8, device=DEV)
    B.sdllm_compact_kv_packed(s, k, v, idx.to(DEV), cache, kept)
    ko, vo = (torch.zeros(Bt, H, kept, d, dtype=td, device=DEV) for _ in range(2))
    B.sdllm_unpack_kv(s, cache, kept, kept, ko, vo)
    torch.cuda.synchronize()
    at = idx.long().clamp(0, L - 1)[..., None].expand(-1, -1, -1, d)
    want = po.cache_values(*(t.cpu().gather(2, at).double().numpy() for t in (k, v)))
    assert np.array_equal(ko.cpu().double().numpy(), want[0]) and np.array_equal(vo.cpu().double().numpy(), want[1])
