"""How attention over the packed cache is launched, on either side of the lines of its rules.  The lines and what was measured on both sides
stand at the rules in csrc/api.hip; here they are pinned, and the GPU tests that are meant for one form ask whether they reach it."""
import ctypes
import os
import subprocess

import pytest

from paper_2508_02558_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def shape(batch, q_heads, kv_heads, d=128, block=32, dtype="bf16"):
    return B.make_shape(batch=batch, n_q_heads=q_heads, n_kv_heads=kv_heads, head_dim=d, seq_len=block + 1, block_off=1, block_len=block,
                        dtype=B.SDLLM_BF16 if dtype == "bf16" else B.SDLLM_F32)


def plan(n, *args, **more):
    p = B.sdllm_packed_plan(shape(*args, **more), n)
    return p.key_splits, p.waves, p.rounds, p.past_caches


def test_layout_and_refusals(tmp_path):
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "sdllm_bench.h"\n'
                   'int main(void){printf("%zu %zu %zu\\n", sizeof(sdllm_packed_plan_t), offsetof(sdllm_packed_plan_t, rounds),'
                   ' offsetof(sdllm_packed_plan_t, past_caches));return 0;}\n')
    exe = tmp_path / "layout"
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)])
    S = B.sdllm_packed_plan_t
    assert [int(x) for x in subprocess.check_output([str(exe)]).split()] == [ctypes.sizeof(S), S.rounds.offset, S.past_caches.offset]
    lib, p = B.load(), S()
    assert lib.sdllm_packed_plan(None, 5, ctypes.byref(p)) == B.SDLLM_ERR_INVALID_ARG
    assert lib.sdllm_packed_plan(ctypes.byref(shape(1, 1, 1)), 5, None) == B.SDLLM_ERR_INVALID_ARG
    assert lib.sdllm_packed_plan(ctypes.byref(shape(1, 1, 1)), -1, ctypes.byref(p)) == B.SDLLM_ERR_INVALID_ARG


@pytest.mark.parametrize("args,n,splits", [((1, 32, 32), 624, 1), ((1, 32, 32), 1000, 1), ((1, 28, 4), 8312, 7), ((1, 28, 4), 2160, 5), ((1, 28, 4), 4000, 6),
                                           ((1, 8, 8), 4000, 8), ((8, 28, 4), 2288, 1), ((8, 32, 32), 2160, 1), ((1, 8, 8), 0, 1)])
def test_key_splits(args, n, splits):
    assert plan(n, *args)[0] == splits


def test_no_split_just_past_a_multiple_of_eight():
    for units in (1, 2, 4, 8, 16):
        for tiles in range(1, 700, 7):
            assert plan(32 * tiles, 1, units, units)[0] % 8 not in (1, 2) or plan(32 * tiles, 1, units, units)[0] < 8, (units, tiles)


def test_wavefronts():
    assert plan(640, 1, 32, 32) == (1, 7, 3, 0)                  # 20 tiles and the block's: no more than what takes three rounds
    assert plan(2160, 8, 32, 32) == (1, 8, 9, 0)                 # 256 units
    assert plan(2160, 1, 257, 257) == (1, 4, 18, 0)              # more: two workgroups to a CU
    assert plan(2160, 1, 257, 257, d=64) == (1, 8, 9, 0)         # which eight wavefronts of 64 channels leave room for
    assert plan(0, 1, 4, 4)[:3] == (1, 1, 1) and plan(0, 1, 4, 4, block=33)[:3] == (1, 2, 1)
    assert plan(2160, 1, 256, 256, dtype="f32")[1] == 4


def test_past_the_caches():
    rows = (128 << 20) // (256 * 34 * 128) * 32                  # a tile of each of 256 heads more is 128 MiB
    assert plan(rows, 8, 32, 32)[3] == 0 and plan(rows + 1, 8, 32, 32)[3] == 1
    assert plan(rows + 1, 8, 32, 32, d=64)[3] == 0 and plan(2 * rows + 64, 8, 32, 32, d=64)[3] == 1
    assert plan(rows + 1, 8, 64, 32)[3] == 0                     # two blocks of columns read the same tiles
    assert plan(rows + 1, 8, 32, 32, dtype="f32")[3] == 0
