"""Norm of rows whose squares single precision cannot hold, and of weights whose product with the norm it cannot."""
import numpy as np
import pytest
import torch

from paper_2508_02558_amd import binding as B
from tests.test_gpu_qk_norm_rope import TYPES, check, freqs

pytestmark = pytest.mark.gpu
DEV = "cuda"


def run(x, weight, eps, dtype):
    """Queries [1, H, n, d] and the same as keys, turned in all channels."""
    H, n, d = x.shape[1:]
    s = B.make_qk_shape(batch=1, n_q_heads=H, n_kv_heads=H, head_dim=d, rows=n, dtype=TYPES[dtype][1], eps=eps, pos_begin=3)
    outs = [torch.full_like(x, 5.0) for _ in range(2)]
    B.sdllm_qk_norm_rope(s, x, x, weight, weight, freqs(d), None, *outs)
    torch.cuda.synchronize()
    assert torch.equal(*outs)
    check(outs[0], x, weight, freqs(d), np.arange(3, 3 + n)[None], d, B.SDLLM_PAIR_HALVES, True, np.float32(eps).astype(float), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("eps", [0.0, 1e-6, 1e-30])
def test_large_and_small_rows_beside_ordinary_ones(dtype, d, eps):
    g = torch.Generator().manual_seed(d)
    x = torch.randn(1, 5, 12, d, generator=g).clamp(-3.5, 3.5)
    for row, power in enumerate((0, 62, 63, 64, 90, 126, -44, -45, -46, -63, -80, -110)):
        x[:, :, row] *= 2.0 ** power
    x[:, 1, 0, 7] = 3e38                                     # one channel of a row
    run(x.to(TYPES[dtype][0]).to(DEV), None, eps, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_weights_beyond_what_the_norm_alone_may_be_multiplied_with(dtype):
    g = torch.Generator().manual_seed(2)
    x = torch.randn(1, 4, 6, 128, generator=g) * 2.0 ** -40
    w = (1 + 0.3 * torch.rand(128, generator=g)) * 2.0 ** 110
    td = TYPES[dtype][0]
    run(x.to(td).to(DEV), w.to(td).to(DEV), 0.0, dtype)


def test_what_is_not_finite_stays_in_its_row():
    x = torch.randn(1, 3, 4, 128, generator=torch.Generator().manual_seed(4)).to(DEV)
    x[0, 1, 2, 9] = float("inf")
    x[0, 2, 0, 70] = float("nan")
    s = B.make_qk_shape(batch=1, n_q_heads=3, n_kv_heads=0, head_dim=128, rows=4, dtype=B.SDLLM_F32, rot_dim=0)
    out = torch.full_like(x, 5.0)
    B.sdllm_qk_norm_rope(s, x, None, None, None, None, None, out, None)
    torch.cuda.synchronize()
    # infinity over infinity is no number, anything else over it is zero
    assert out[0, 1, 2, 9].isnan() and (out[0, 1, 2, torch.arange(128, device=DEV) != 9] == 0).all()
    assert out[0, 2, 0].isnan().all()
    rest = torch.ones(3, 4, dtype=torch.bool, device=DEV)
    rest[1, 2] = rest[2, 0] = False
    assert torch.isfinite(out[0][rest]).all()
