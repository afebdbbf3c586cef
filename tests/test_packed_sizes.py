"""Sizes whose products do not fit what they are counted in: refused, and before anything is enqueued."""
import ctypes

import pytest

from paper_2508_02558_amd import binding as B

fake, z = ctypes.c_void_p(0x1000), ctypes.c_void_p(None)


def shape(batch, heads, seq_len=500, **more):
    s = B.make_shape(batch=1, n_q_heads=1, n_kv_heads=1, head_dim=128, seq_len=seq_len, block_off=0, block_len=32, dtype=B.SDLLM_BF16, retention=1.0, **more)
    s.batch, s.n_q_heads, s.n_kv_heads = batch, heads, heads     # strides of one head: no tensor is this large
    return s


# products of 2^32, 2^40, 2^60, of nearly 2^62, and ones that leave little in 32 or 64 bits
MANY = [(1 << 16, 1 << 16), (1 << 20, 1 << 20), (1 << 30, 1 << 30), (2147483647, 2147483647), ((1 << 16) + 1, 1 << 16), (1 << 30, (1 << 30) + 4)]


@pytest.mark.parametrize("batch,heads", MANY)
@pytest.mark.parametrize("seq_len", [500, 544, 1 << 28])
def test_more_heads_in_all_than_can_be_counted(batch, heads, seq_len):
    lib, s, n = B.load(), shape(batch, heads, seq_len), ctypes.c_size_t()
    kept = seq_len - 32
    by = ctypes.byref(s)
    assert lib.sdllm_packed_cache_bytes(by, kept, ctypes.byref(n)) == B.SDLLM_ERR_UNSUPPORTED
    assert lib.sdllm_compact_kv_packed(by, fake, fake, fake, fake, kept, z) == B.SDLLM_ERR_UNSUPPORTED
    assert lib.sdllm_unpack_kv(by, fake, kept, kept, fake, fake, z) == B.SDLLM_ERR_UNSUPPORTED
    for op in (B.SDLLM_OP_SPARSE_ATTN_PACKED, B.SDLLM_OP_BLOCK_STEP_PACKED):
        assert lib.sdllm_workspace_bytes(by, op, kept, ctypes.byref(n)) == B.SDLLM_ERR_UNSUPPORTED
    for rows in (0, kept):
        assert lib.sdllm_sparse_attn_packed(by, fake, fake, kept, rows, fake, fake, fake, fake, 1 << 60, z) == B.SDLLM_ERR_UNSUPPORTED
        assert lib.sdllm_packed_plan(by, rows, ctypes.byref(B.sdllm_packed_plan_t())) == B.SDLLM_ERR_UNSUPPORTED
    for step in (0, 1, 2):
        assert lib.sdllm_block_step_packed(by, step, 1, fake, fake, fake, fake, fake, kept, fake, fake, 1 << 60, z, None) == B.SDLLM_ERR_UNSUPPORTED


@pytest.mark.parametrize("batch,heads,rows", [(1 << 16, 1 << 14, 2147483647), (1 << 15, 1 << 14, 2147483647), (46340, 46340, 1 << 30)])
def test_a_cache_of_more_bytes_than_can_be_counted(batch, heads, rows):
    n = ctypes.c_size_t()
    assert lib_bytes(batch, heads, rows, n) == B.SDLLM_ERR_UNSUPPORTED


def lib_bytes(batch, heads, rows, n):
    return B.load().sdllm_packed_cache_bytes(ctypes.byref(shape(batch, heads)), rows, ctypes.byref(n))


def test_the_largest_that_can():
    n = ctypes.c_size_t()
    assert lib_bytes(1 << 12, 1 << 12, 2147483647, n) == B.SDLLM_OK and n.value == (1 << 24) * (1 << 26) * 4352
    assert lib_bytes(2147483647, 1, 32, n) == B.SDLLM_OK and n.value == 2147483647 * 4352
