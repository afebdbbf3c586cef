"""Host side of the packed cache and of the norm and rotation: sizes, struct layout, and refusals before anything is enqueued."""
import ctypes
import os
import subprocess

import pytest

from paper_2508_02558_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
fake, odd, z = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1008), ctypes.c_void_p(None)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2508_02558_amd.build import build_library
        build_library(verbose=False)
    return B.load()


def _shape(**kw):
    base = dict(batch=2, n_q_heads=8, n_kv_heads=2, head_dim=128, seq_len=500, block_off=300, block_len=32, dtype=B.SDLLM_BF16)
    base.update(kw)
    return B.make_shape(**base)


def _qk(**kw):
    base = dict(batch=2, n_q_heads=8, n_kv_heads=2, head_dim=128, rows=40, dtype=B.SDLLM_BF16)
    base.update(kw)
    return B.make_qk_shape(**base)


def test_qk_shape_has_the_headers_layout(lib, tmp_path):
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "sdllm.h"\n'
                   'int main(void){printf("%zu %zu %zu %zu %zu\\n", sizeof(sdllm_qk_shape_t), offsetof(sdllm_qk_shape_t, eps),'
                   ' offsetof(sdllm_qk_shape_t, pos_stride), offsetof(sdllm_qk_shape_t, q_in_stride), offsetof(sdllm_qk_shape_t, k_out_stride));'
                   'return 0;}\n')
    exe = tmp_path / "layout"
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)])
    S = B.sdllm_qk_shape_t
    assert [int(x) for x in subprocess.check_output([str(exe)]).split()] == [
        ctypes.sizeof(S), S.eps.offset, S.pos_stride.offset, S.q_in_stride.offset, S.k_out_stride.offset]


def test_names_of_the_header_are_bound(lib):
    text = open(os.path.join(ROOT, "include", "sdllm.h")).read()
    for name in ("sdllm_packed_cache_bytes", "sdllm_compact_kv_packed", "sdllm_unpack_kv", "sdllm_sparse_attn_packed", "sdllm_block_step_packed",
                 "sdllm_qk_norm_rope"):
        assert name + "(" in text and name in B.EXPORTED and hasattr(lib, name) and callable(getattr(B, name))
    for name in ("SDLLM_OP_SPARSE_ATTN_PACKED", "SDLLM_OP_BLOCK_STEP_PACKED", "SDLLM_NORM_NONE", "SDLLM_NORM_RMS", "SDLLM_PAIR_HALVES",
                 "SDLLM_PAIR_ADJACENT"):
        assert f"#define {name} {getattr(B, name)}\n" in text


@pytest.mark.parametrize("rows,d,want", [(0, 128, 256), (1, 128, 4 * 4352), (32, 128, 4 * 4352), (33, 128, 8 * 4352), (33, 64, 8 * 2176),
                                         (2147483647, 128, 4 * 67108864 * 4352)])
def test_cache_size(lib, rows, d, want):
    assert B.sdllm_packed_cache_bytes(_shape(head_dim=d), rows) == want


def test_cache_size_refusals(lib):
    n = ctypes.c_size_t()
    assert lib.sdllm_packed_cache_bytes(ctypes.byref(_shape()), -1, ctypes.byref(n)) == B.SDLLM_ERR_INVALID_ARG
    assert lib.sdllm_packed_cache_bytes(ctypes.byref(_shape()), 5, None) == B.SDLLM_ERR_INVALID_ARG
    assert lib.sdllm_packed_cache_bytes(None, 5, ctypes.byref(n)) == B.SDLLM_ERR_INVALID_ARG
    assert lib.sdllm_packed_cache_bytes(ctypes.byref(_shape(head_dim=96)), 5, ctypes.byref(n)) == B.SDLLM_ERR_UNSUPPORTED


def test_compaction_refusals(lib):
    s = _shape()
    kept = B.sdllm_retained_count(s)[0]
    call = lambda k=fake, v=fake, idx=fake, cache=fake, rows=kept, shape=s: lib.sdllm_compact_kv_packed(ctypes.byref(shape), k, v, idx, cache, rows, z)
    for kw in (dict(k=z), dict(v=z), dict(idx=z), dict(cache=z), dict(k=odd), dict(v=odd), dict(cache=odd), dict(rows=kept - 1), dict(rows=-1),
               dict(shape=_shape(kv_stride=(4096, 64, 64))), dict(shape=_shape(batch=0))):
        assert call(**kw) == B.SDLLM_ERR_INVALID_ARG, kw
    none = _shape(retention=0.0)
    assert call(k=z, v=z, idx=z, cache=z, rows=0, shape=none) == B.SDLLM_OK          # nothing is kept


def test_unpack_refusals(lib):
    s = _shape()
    call = lambda cache=fake, rows=100, n=100, k=fake, v=fake, shape=s: lib.sdllm_unpack_kv(ctypes.byref(shape), cache, rows, n, k, v, z)
    for kw in (dict(cache=z), dict(cache=odd), dict(rows=99), dict(n=-1), dict(k=z), dict(v=z), dict(k=odd), dict(v=odd),
               dict(shape=_shape(cache_stride=(4096, 64, 64)))):
        assert call(**kw) == B.SDLLM_ERR_INVALID_ARG, kw
    assert call(cache=z, k=z, v=z, n=0) == B.SDLLM_OK


def test_attention_refusals(lib):
    s = _shape()
    need = B.sdllm_workspace_bytes(s, B.SDLLM_OP_SPARSE_ATTN_PACKED, 400)

    def call(q=fake, cache=fake, rows=400, n=400, k=fake, v=fake, out=fake, ws=fake, size=need, shape=s):
        return lib.sdllm_sparse_attn_packed(ctypes.byref(shape), q, cache, rows, n, k, v, out, ws, size, z)
    for kw in (dict(q=z), dict(q=odd), dict(cache=z), dict(cache=odd), dict(rows=399), dict(n=-1), dict(k=z), dict(v=z), dict(k=odd), dict(v=odd),
               dict(out=z), dict(out=odd), dict(shape=_shape(blk_stride=(4096, 64, 64))), dict(shape=_shape(out_stride=(4096, 64, 64))),
               dict(shape=_shape(q_stride=(4096, 64, 64)))):
        assert call(**kw) == B.SDLLM_ERR_INVALID_ARG, kw
    long = 20000                                                         # its keys are split
    need = B.sdllm_workspace_bytes(s, B.SDLLM_OP_SPARSE_ATTN_PACKED, long)
    assert need > 256
    for ws, size in ((z, need), (fake, need - 1), (odd, need)):
        assert call(rows=long, n=long, ws=ws, size=size) == B.SDLLM_ERR_WORKSPACE
    with pytest.raises(B.SdllmError):
        B.sdllm_workspace_bytes(s, B.SDLLM_OP_SPARSE_ATTN_PACKED, -1)
    huge = _shape(batch=1 << 24, n_q_heads=64, n_kv_heads=64)
    assert call(shape=huge, size=1 << 60) == B.SDLLM_ERR_UNSUPPORTED     # more threads than a launch has


def test_block_step_refusals(lib):
    s = _shape()
    kept, need = B.sdllm_retained_count(s)[0], B.sdllm_workspace_bytes(s, B.SDLLM_OP_BLOCK_STEP_PACKED)
    assert need >= max(B.sdllm_workspace_bytes(s, B.SDLLM_OP_SPARSE_ATTN_PACKED, kept), B.sdllm_workspace_bytes(s, B.SDLLM_OP_SCORE_SELECT))

    def call(step=2, delay=1, q=fake, k=fake, v=fake, idx=fake, cache=fake, rows=kept, out=fake, ws=fake, size=need):
        return lib.sdllm_block_step_packed(ctypes.byref(s), step, delay, q, k, v, idx, cache, rows, out, ws, size, z, None)
    for step in (0, 1, 2):
        for kw in (dict(q=z), dict(k=z), dict(v=z), dict(out=z), dict(out=odd), dict(delay=-1)):
            assert call(step, **kw) == B.SDLLM_ERR_INVALID_ARG, (step, kw)
        for kw in (dict(ws=z), dict(ws=odd), dict(size=need - 1)):
            assert call(step, **kw) == B.SDLLM_ERR_WORKSPACE, (step, kw)
    for step in (1, 2):
        for kw in (dict(cache=z), dict(cache=odd), dict(rows=kept - 1)):
            assert call(step, **kw) == B.SDLLM_ERR_INVALID_ARG, (step, kw)
    assert call(1, idx=z) == B.SDLLM_ERR_INVALID_ARG
    assert call(-1) == B.SDLLM_ERR_INVALID_ARG


def test_norm_and_rotation_refusals(lib):
    def call(q=fake, k=fake, qw=fake, kw=fake, freq=fake, pos=fake, qo=fake, ko=fake, **shape):
        return lib.sdllm_qk_norm_rope(ctypes.byref(_qk(**shape)), q, k, qw, kw, freq, pos, qo, ko, z)
    for kw in (dict(q=z), dict(k=z), dict(qo=z), dict(ko=z), dict(q=odd), dict(k=odd), dict(qo=odd), dict(ko=odd), dict(qw=odd), dict(kw=odd),
               dict(freq=z), dict(batch=0), dict(rows=-1), dict(n_q_heads=-1), dict(n_q_heads=0, n_kv_heads=0), dict(dtype=2), dict(rot_dim=-16),
               dict(rot_dim=144), dict(rot_dim=31), dict(pairing=2), dict(norm=2), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")),
               dict(pos_stride=-1), dict(q_in_stride=(1, 128, 128)), dict(k_out_stride=(4096, 128, 64)), dict(q_in_stride=(4096, -128, 128)),
               dict(pos=z, pos_begin=2147483647 - 38)):
        assert call(**kw) == B.SDLLM_ERR_INVALID_ARG, kw
    for kw in (dict(head_dim=96), dict(rot_dim=24), dict(batch=1 << 20, rows=1 << 20)):
        assert call(**kw) == B.SDLLM_ERR_UNSUPPORTED, kw
    assert lib.sdllm_qk_norm_rope(None, fake, fake, z, z, fake, fake, fake, fake, z) == B.SDLLM_ERR_INVALID_ARG
    s = _qk()
    s.reserved = 1
    assert lib.sdllm_qk_norm_rope(ctypes.byref(s), fake, fake, z, z, fake, fake, fake, fake, z) == B.SDLLM_ERR_INVALID_ARG
    assert call(rows=0) == B.SDLLM_OK                                    # nothing to do


def test_norm_and_rotation_of_more_rows_than_a_launch_has_threads_for(lib):
    # a wavefront of 64 threads for each, four to a workgroup
    for rows in (2 ** 26 - 3, 2 ** 26, 2 ** 31 - 1):
        shape = _qk(batch=1, rows=rows, pos_begin=0)
        assert lib.sdllm_qk_norm_rope(ctypes.byref(shape), fake, fake, z, z, fake, fake, fake, fake, z) == B.SDLLM_ERR_UNSUPPORTED, rows


pycall = pytest.mark.skipif(B._pycall is None, reason="built without the interpreter's headers")


class _Tensor:
    def __init__(self, at, numel=0):
        self.at, self.n = at, numel

    def data_ptr(self):
        return self.at

    def numel(self):
        return self.n

    def element_size(self):
        return 2


@pycall
def test_arguments_arrive_where_the_prototypes_have_them():
    vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
    seen = []

    def recorder(*types):
        @ctypes.CFUNCTYPE(i32, *types)
        def f(*args):
            seen.append(args)
            return 0
        return f, ctypes.cast(f, vp).value
    t = [_Tensor(0x7f0000000000 + 16 * i, 3) for i in range(9)]
    at = [x.at for x in t]
    f, a = recorder(vp, i32, i32, vp, vp, vp, vp, vp, i32, vp, vp, sz, vp, vp)
    assert B._pycall.block_step_packed(a, 5, 7, 3, t[0], t[1], t[2], t[3], t[4], 77, t[5], t[6], 9) == -1      # the recorder sets no state
    assert seen[-1][:13] == (5, 7, 3, *at[:5], 77, at[5], at[6], 6, 9)
    f, a = recorder(vp, vp, vp, i32, i32, vp, vp, vp, vp, sz, vp)
    assert B._pycall.sparse_attn_packed(a, 5, t[0], t[1], 70, 60, t[2], t[3], t[4], None, 9) == 0
    assert seen[-1] == (5, at[0], at[1], 70, 60, at[2], at[3], at[4], None, 0, 9)
    f, a = recorder(vp, vp, vp, vp, vp, i32, vp)
    assert B._pycall.compact_packed(a, 5, t[0], t[1], t[2], t[3], 70, 9) == 0
    assert seen[-1] == (5, *at[:4], 70, 9)
    f, a = recorder(vp, vp, i32, i32, vp, vp, vp)
    assert B._pycall.unpack_kv(a, 5, t[0], 70, 60, t[1], t[2], 9) == 0
    assert seen[-1] == (5, at[0], 70, 60, at[1], at[2], 9)
    f, a = recorder(*[vp] * 10)
    assert B._pycall.qk_norm_rope(a, 5, t[0], t[1], None, t[3], t[4], t[5], t[6], t[7], 9) == 0
    assert seen[-1] == (5, at[0], at[1], None, at[3], at[4], at[5], at[6], at[7], 9)
    with pytest.raises(TypeError):
        B._pycall.qk_norm_rope(a, 5)
