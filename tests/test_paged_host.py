"""Host side of the paged cache: struct layout, names, workspace sizes, and refusals before anything is enqueued."""
import ctypes
import os
import re
import subprocess

import pytest

from paper_2508_02558_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
fake, odd, z = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1008), ctypes.c_void_p(None)
ws, big = ctypes.c_void_p(0x10000), 1 << 40
INVALID, UNSUPPORTED, WORKSPACE = B.SDLLM_ERR_INVALID_ARG, B.SDLLM_ERR_UNSUPPORTED, B.SDLLM_ERR_WORKSPACE
TREE, WINDOW = B.SDLLM_OP_TREE_ATTN_PAGED, B.SDLLM_OP_WINDOW_ATTN_PAGED


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2508_02558_amd.build import build_library
        build_library(verbose=False)
    return B.load()


def _shape(**kw):
    base = dict(batch=2, n_q_heads=8, n_kv_heads=2, head_dim=128, rows=40, dtype=B.SDLLM_BF16, n_pages=50, page_rows=64, table_pages=20)
    base.update(kw)
    return B.make_paged_shape(**base)


def _qk(**kw):
    base = dict(batch=2, n_q_heads=8, n_kv_heads=2, head_dim=128, rows=40, dtype=B.SDLLM_BF16)
    base.update(kw)
    return B.make_qk_shape(**base)


def tree(lib, s, q=fake, kp=fake, vp=fake, table=fake, lengths=fake, counts=z, kb=fake, vb=fake, mask=fake, out=fake, w=ws, n=big):
    return lib.sdllm_tree_attn_paged(None if s is None else ctypes.byref(s), q, kp, vp, table, lengths, counts, kb, vb, mask, out, w, n, z)


def window(lib, s, q=fake, kp=fake, vp=fake, table=fake, lengths=fake, counts=z, out=fake, w=ws, n=big):
    return lib.sdllm_window_attn_paged(None if s is None else ctypes.byref(s), q, kp, vp, table, lengths, counts, out, w, n, z)


def append(lib, h, s, q=fake, k=fake, v=fake, qw=fake, kw=fake, freq=fake, pos=z, pick=z, lengths=fake, counts=z, table=fake, qo=fake, kp=fake, vp=fake):
    ref = lambda x: None if x is None else ctypes.byref(x)
    return lib.sdllm_append_paged(ref(h), ref(s), q, k, v, qw, kw, freq, pos, pick, lengths, counts, table, qo, kp, vp, z)


def test_layout_is_the_headers(lib, tmp_path):
    S = B.sdllm_paged_shape_t
    names = [n for n, _ in S._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "sdllm.h"\nint main(void){printf("%zu", sizeof(sdllm_paged_shape_t));' +
                   "".join(f'printf(" %zu", offsetof(sdllm_paged_shape_t, {n}));' for n in names) + "return 0;}\n")
    exe = tmp_path / "layout"
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)])
    assert [int(x) for x in subprocess.check_output([str(exe)]).split()] == [ctypes.sizeof(S)] + [getattr(S, n).offset for n in names]


def test_names_of_the_header_are_bound(lib):
    text = open(os.path.join(ROOT, "include", "sdllm.h")).read()
    for name in ("sdllm_paged_workspace_bytes", "sdllm_append_paged", "sdllm_tree_attn_paged", "sdllm_window_attn_paged"):
        assert name + "(" in text and name in B.EXPORTED and hasattr(lib, name) and callable(getattr(B, name))
    for name in ("SDLLM_OP_TREE_ATTN_PAGED", "SDLLM_OP_WINDOW_ATTN_PAGED"):
        assert f"#define {name} {getattr(B, name)}\n" in text


BAD = [dict(batch=0), dict(n_q_heads=7), dict(n_q_heads=0), dict(n_kv_heads=0), dict(rows=-1), dict(dtype=2), dict(n_pages=-1), dict(page_rows=0),
       dict(page_rows=-64), dict(table_pages=-1), dict(sinks=-1), dict(softmax_scale=-1.0), dict(softmax_scale=float("nan")), dict(softmax_scale=float("inf")),
       dict(table_stride=-1), dict(mask_stride=-1), dict(q_stride=(8, 8, -128)), dict(out_stride=(8, 4, 128)), dict(page_stride=(8, 8, 132)),
       dict(blk_stride=(1, 8, 128))]
NOT_HERE = [dict(head_dim=96), dict(page_rows=8), dict(page_rows=48), dict(page_rows=512), dict(rows=(1 << 29) + 1), dict(table_pages=1 << 24, page_rows=64)]


@pytest.mark.parametrize("kw", BAD)
def test_bad_shapes(lib, kw):
    s = _shape(**kw)
    n = ctypes.c_size_t()
    assert lib.sdllm_paged_workspace_bytes(ctypes.byref(s), WINDOW, ctypes.byref(n)) == INVALID
    assert tree(lib, s) == window(lib, s) == append(lib, _qk(), s) == INVALID


@pytest.mark.parametrize("kw", NOT_HERE)
def test_shapes_without_a_kernel(lib, kw):
    s = _shape(**kw)
    n = ctypes.c_size_t()
    assert lib.sdllm_paged_workspace_bytes(ctypes.byref(s), WINDOW, ctypes.byref(n)) == UNSUPPORTED
    assert window(lib, s) == append(lib, _qk(), s) == UNSUPPORTED


def test_reserved_and_null_shapes(lib):
    s = _shape()
    s.reserved = 1
    assert tree(lib, s) == window(lib, s) == append(lib, _qk(), s) == INVALID
    assert tree(lib, None) == window(lib, None) == append(lib, None, _shape()) == append(lib, _qk(), None) == INVALID
    n = ctypes.c_size_t()
    assert lib.sdllm_paged_workspace_bytes(None, TREE, ctypes.byref(n)) == INVALID
    assert lib.sdllm_paged_workspace_bytes(ctypes.byref(_shape()), TREE, None) == INVALID
    for op in (-1, 0, B.SDLLM_OP_SPARSE_ATTN_PACKED, 8):
        assert lib.sdllm_paged_workspace_bytes(ctypes.byref(_shape()), op, ctypes.byref(n)) == INVALID


def test_a_tree_has_64_rows_at_most(lib):
    n = ctypes.c_size_t()
    assert lib.sdllm_paged_workspace_bytes(ctypes.byref(_shape(rows=65)), TREE, ctypes.byref(n)) == UNSUPPORTED
    assert tree(lib, _shape(rows=65)) == UNSUPPORTED
    assert B.sdllm_paged_workspace_bytes(_shape(rows=64), TREE) > 0 and B.sdllm_paged_workspace_bytes(_shape(rows=65), WINDOW) > 0


@pytest.mark.parametrize("call", [tree, window])
def test_pointers_of_the_attentions(lib, call):
    names = ["q", "kp", "vp", "table", "lengths", "out"] + (["kb", "vb"] if call is tree else [])
    for name in names:
        assert call(lib, _shape(), **{name: z}) == INVALID, name
    for name in names:
        if name not in ("table", "lengths"):
            assert call(lib, _shape(), **{name: odd}) == INVALID, name
    if call is tree:
        assert tree(lib, _shape(), mask=ctypes.c_void_p(0x1004)) == INVALID
    need = B.sdllm_paged_workspace_bytes(_shape(), TREE if call is tree else WINDOW)
    assert call(lib, _shape(), w=z) == call(lib, _shape(), w=ctypes.c_void_p(0x10010)) == call(lib, _shape(), n=need - 1) == WORKSPACE
    # rows that overlap
    for name in ("q_stride", "out_stride", "page_stride") + (("blk_stride",) if call is tree else ()):
        assert call(lib, _shape(**{name: (8, 8, 64)})) == INVALID, name
    # rows too far apart to be addressed from their first in 32 bits
    assert call(lib, _shape(page_stride=(8, 8, 1 << 26))) == UNSUPPORTED


@pytest.mark.parametrize("call", [tree, window])
def test_no_rows_is_no_work(lib, call):
    assert call(lib, _shape(rows=0)) == B.SDLLM_OK
    assert append(lib, _qk(rows=0), _shape(rows=0)) == B.SDLLM_OK


@pytest.mark.parametrize("call,kw", [(tree, dict(rows=64)), (window, dict(rows=1 << 29))])
def test_grids_that_do_not_fit_are_refused(lib, call, kw):
    assert call(lib, _shape(n_q_heads=1 << 30, n_kv_heads=1, **kw)) == UNSUPPORTED          # columns
    assert call(lib, _shape(batch=1 << 20, n_q_heads=1 << 20, n_kv_heads=1 << 20, **kw)) == UNSUPPORTED
    assert call(lib, _shape(batch=1 << 30, n_q_heads=2, n_kv_heads=2, **kw)) == UNSUPPORTED


def test_pointers_of_appending(lib):
    for name in ("q", "k", "v", "freq", "lengths", "table", "qo", "kp", "vp"):
        assert append(lib, _qk(), _shape(), **{name: z}) == INVALID, name
    for name in ("q", "k", "v", "qw", "kw", "qo", "kp", "vp"):
        assert append(lib, _qk(), _shape(), **{name: odd}) == INVALID, name
    assert append(lib, _qk(), _shape(), pick=fake) == INVALID                                # with queries
    for kw in (dict(batch=3), dict(n_kv_heads=4), dict(head_dim=64), dict(rows=41), dict(dtype=B.SDLLM_F32)):
        assert append(lib, _qk(**kw), _shape()) == INVALID, kw
    for kw in (dict(eps=-1.0), dict(norm=2), dict(pairing=2), dict(rot_dim=130), dict(pos_stride=-1), dict(k_in_stride=(8, 8, 64)),
               dict(q_out_stride=(8, 8, 100)), dict(pos_begin=2147483647)):
        assert append(lib, _qk(**kw), _shape()) == INVALID, kw
    assert append(lib, _qk(rot_dim=24), _shape()) == UNSUPPORTED
    assert append(lib, _qk(batch=1 << 20, rows=1 << 10), _shape(batch=1 << 20, rows=1 << 10)) == UNSUPPORTED


def test_an_empty_pool_needs_no_pointers(lib):
    for kw in (dict(n_pages=0), dict(table_pages=0)):
        assert tree(lib, _shape(rows=0, **kw), kp=z, vp=z, table=z) == B.SDLLM_OK
        assert window(lib, _shape(rows=0, **kw), kp=z, vp=z, table=z) == B.SDLLM_OK
        assert append(lib, _qk(rows=0), _shape(rows=0, **kw), kp=z, vp=z, table=z) == B.SDLLM_OK
        assert window(lib, _shape(rows=0, **kw), kp=z, vp=z, table=z, lengths=z) == INVALID


def test_workspace_holds_a_partial_for_every_share(lib):
    for kw in (dict(), dict(rows=1), dict(dtype=B.SDLLM_F32), dict(head_dim=64), dict(batch=200), dict(window_left=100)):
        for op in (TREE, WINDOW):
            n = B.sdllm_paged_workspace_bytes(_shape(**kw), op)
            assert 256 <= n < 1 << 30 and n % 256 == 0


def test_refusals_are_the_same_with_and_without_the_binding_module(lib, monkeypatch):
    class T:
        def __init__(self, at, n=1 << 20): self.at, self.n = at, n
        def data_ptr(self): return self.at
        def numel(self): return self.n
        def element_size(self): return 1
    t, o, w = T(0x1000), T(0x1008), T(0x10000)

    def refusals():
        got = []
        for call in (lambda: B.sdllm_tree_attn_paged(_shape(), o, t, t, t, t, None, t, t, None, t, w, stream=1),
                     lambda: B.sdllm_tree_attn_paged(_shape(), t, t, t, t, t, None, t, t, None, t, None, stream=1),
                     lambda: B.sdllm_window_attn_paged(_shape(), t, t, t, None, t, t, t, w, stream=1),
                     lambda: B.sdllm_window_attn_paged(_shape(), t, t, t, t, t, t, t, T(0x10000, 5), stream=1),
                     lambda: B.sdllm_append_paged(_qk(), _shape(), t, t, o, t, t, t, None, None, t, None, t, t, t, t, stream=1),
                     lambda: B.sdllm_append_paged(_qk(batch=1), _shape(), t, t, t, t, t, t, None, None, t, None, t, t, t, t, stream=1)):
            with pytest.raises(B.SdllmError) as e:
                call()
            got.append(str(e.value))
        return got
    with_it = refusals()
    assert len(set(re.sub(r"_\w+", "", x) for x in with_it)) == 2
    monkeypatch.setattr(B, "_pycall", None)
    assert refusals() == with_it
