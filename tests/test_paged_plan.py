"""How attention over the paged cache is launched, on either side of the lines of its rules.  The lines and what was measured on both sides
stand at the rules in csrc/paged_api.hip; here they are pinned, and the GPU tests that are meant for one form ask whether they reach it."""
import ctypes
import os
import subprocess

import pytest

from paper_2508_02558_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
TREE, WINDOW = B.SDLLM_OP_TREE_ATTN_PAGED, B.SDLLM_OP_WINDOW_ATTN_PAGED


def shape(batch, q_heads, kv_heads, rows, capacity=65536, d=128, dtype="bf16", **more):
    return B.make_paged_shape(batch=batch, n_q_heads=q_heads, n_kv_heads=kv_heads, head_dim=d, rows=rows, dtype=B.SDLLM_BF16 if dtype == "bf16" else B.SDLLM_F32,
                              n_pages=1, page_rows=64, table_pages=capacity // 64, **more)


def plan(*args, op=WINDOW, **more):
    p = B.sdllm_paged_plan(shape(*args, **more), op)
    return p.shared, p.block_cols, p.waves, p.workgroups, p.least_tiles


def test_layout_and_refusals(tmp_path):
    S = B.sdllm_paged_plan_t
    names = [n for n, _ in S._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "sdllm_bench.h"\nint main(void){printf("%zu", sizeof(sdllm_paged_plan_t));' +
                   "".join(f'printf(" %zu", offsetof(sdllm_paged_plan_t, {n}));' for n in names) + "return 0;}\n")
    exe = tmp_path / "layout"
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)])
    assert [int(x) for x in subprocess.check_output([str(exe)]).split()] == [ctypes.sizeof(S)] + [getattr(S, n).offset for n in names]
    lib, p = B.load(), S()
    assert lib.sdllm_paged_plan(None, WINDOW, ctypes.byref(p)) == B.SDLLM_ERR_INVALID_ARG
    assert lib.sdllm_paged_plan(ctypes.byref(shape(1, 1, 1, 1)), WINDOW, None) == B.SDLLM_ERR_INVALID_ARG
    assert lib.sdllm_paged_plan(ctypes.byref(shape(1, 1, 1, 1)), 0, ctypes.byref(p)) == B.SDLLM_ERR_INVALID_ARG
    assert lib.sdllm_paged_plan(ctypes.byref(shape(1, 1, 1, 65)), TREE, ctypes.byref(p)) == B.SDLLM_ERR_UNSUPPORTED


@pytest.mark.parametrize("args,want", [((1, 16, 1, 1), (0, 16)), ((1, 17, 1, 1), (0, 32)), ((1, 32, 1, 2), (0, 32)), ((1, 13, 1, 5), (0, 32)),
                                       ((1, 128, 1, 1), (0, 32)), ((1, 129, 1, 1), (1, 256)), ((17, 65, 1, 1), (1, 128)), ((17, 64, 1, 1), (0, 32)),
                                       ((17, 129, 1, 1), (1, 256)), ((4, 28, 4, 4096), (1, 256))])
def test_columns_choose_the_kernel(args, want):
    assert plan(*args)[:2] == want


def test_fp32_streams():
    assert plan(4, 28, 4, 64, dtype="f32")[:3] == (0, 16, 4) and plan(4, 28, 4, 64, dtype="f32", d=64)[:3] == (0, 16, 8)


def test_shares():
    assert plan(1, 28, 4, 1) == (0, 16, 8, 256, 8) and plan(32, 1, 1, 1) == (0, 16, 8, 256, 8)   # few items: a tile for every wavefront is a share
    assert plan(33, 1, 1, 1) == (0, 16, 8, 256, 48)
    assert plan(64, 1, 1, 1) == (0, 16, 8, 256, 48) and plan(65, 1, 1, 1) == (0, 16, 4, 512, 24)
    assert plan(512, 1, 1, 1) == (0, 16, 4, 1024, 24) and plan(1024, 1, 1, 1) == (0, 16, 4, 2048, 24)
    assert plan(1025, 1, 1, 1) == (0, 16, 4, 1025, 0)                  # more: nothing is cut
    assert plan(1, 28, 4, 1, capacity=992)[3:] == (4, 0) and plan(1, 28, 4, 1, capacity=1024)[3:] == (256, 8)   # nor where there are few tiles
    assert plan(33, 1, 1, 1, capacity=1536)[3:] == (33, 0) and plan(33, 1, 1, 1, capacity=1600)[3:] == (256, 48)
    assert plan(1, 28, 4, 1, window_left=900, sinks=4)[3:] == (4, 0) and plan(1, 28, 4, 1, window_left=4000)[3:] == (256, 8)
    assert plan(8, 4, 4, 2, dtype="f32")[3:] == (256, 4) and plan(9, 4, 4, 2, dtype="f32")[3:] == (256, 8)
    assert plan(32, 256, 4, 4) == (1, 256, 8, 256, 8) and plan(33, 256, 4, 4) == (1, 256, 8, 132, 0)
    assert plan(8, 28, 4, 64, op=TREE) == (1, 256, 8, 256, 8)
    assert plan(4, 28, 4, 4096) == (1, 256, 8, 4 * 4 * 112, 0)


def test_the_workspace_is_for_the_workgroups():
    for args, more in (((1, 28, 4, 1), {}), ((8, 28, 4, 64), {}), ((65, 8, 2, 1), {}), ((3, 14, 2, 9), dict(dtype="f32", d=64))):
        _, cols, _, groups, least = plan(*args, **more)
        d = more.get("d", 128)
        need = B.sdllm_paged_workspace_bytes(shape(*args, **more), WINDOW)
        assert least == 0 or need >= groups * cols * (d + 2) * 4
