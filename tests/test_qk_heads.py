"""Norm and rotation count heads in 32 bits, a step past the last one included."""
import ctypes

import pytest

from paper_2508_02558_amd import binding as B

fake, z = ctypes.c_void_p(0x1000), ctypes.c_void_p(None)


@pytest.mark.parametrize("dtype", [B.SDLLM_BF16, B.SDLLM_F32])
@pytest.mark.parametrize("hq,hkv", [(2147483647, 0), (0, 2147483640), (1 << 30, 1), (2147483632, 15)])
def test_more_heads_than_are_stepped_over(hq, hkv, dtype):
    s = B.make_qk_shape(batch=1, n_q_heads=hq, n_kv_heads=hkv, head_dim=64, rows=1, dtype=dtype)
    assert B.load().sdllm_qk_norm_rope(ctypes.byref(s), fake, fake, z, z, fake, z, fake, fake, z) == B.SDLLM_ERR_UNSUPPORTED
