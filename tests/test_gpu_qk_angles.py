"""Cosine and sine that norm and rotation turn by, to the last bits of single precision: also where they are small."""
import numpy as np
import pytest
import torch

from paper_2508_02558_amd import binding as B
from tests.test_gpu_qk_norm_rope import freqs

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("first", [0, 4096, -3000])
def test_cosine_and_sine(d, first):
    # pairs (1, 0): what comes out are the two, no other rounding
    n = 2500
    x = torch.zeros(1, 1, n, d, device=DEV)
    x[..., :d // 2] = 1
    s = B.make_qk_shape(batch=1, n_q_heads=1, n_kv_heads=0, head_dim=d, rows=n, dtype=B.SDLLM_F32, norm=B.SDLLM_NORM_NONE, pos_begin=first)
    out = torch.full_like(x, 5.0)
    freq = freqs(d)
    B.sdllm_qk_norm_rope(s, x, None, None, None, freq, None, out, None)
    got = out[0, 0].cpu().double().numpy()
    t = np.arange(first, first + n, dtype=np.float64)[:, None] * freq.cpu().double().numpy()
    want = np.concatenate([np.cos(t), np.sin(t)], -1)
    # the functions are good to a step of their values, the angle's part that single precision leaves off is put back with a rounding more;
    # the angle itself is rounded twice in 64 bits, and what is put back is a product of single precision
    tol = 2.0 ** -22 * np.abs(want) + 2.0 ** -45 + 2.0 ** -51 * np.abs(np.concatenate([t, t], -1))
    err = np.abs(got - want)
    assert (err <= tol).all(), float((err / tol).max())
