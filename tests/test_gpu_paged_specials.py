"""Infinities and NaN among the values of the paged cache: the rows that see them have them, the others do not, in every form of the attentions."""
import pytest

from paper_2508_02558_amd import binding as B
from tests.paged_strict import KINDS, check_strictly, one_a_tile
from tests.paged_util import Paged, tree_masks

pytestmark = pytest.mark.gpu

ALL, CAUSAL = (-1, -1, 0), (-1, 0, 0)


def call(kind, Hq, Hkv, d, n, lengths, window, dtype="bf16", form=None, kinds="nan", **more):
    left, right, sinks = window or CAUSAL
    c = Paged(kind, Hq, Hkv, d, n, lengths, dtype, mask=tree_masks(len(lengths), n, 2) if kind == "tree" else None, left=left, right=right, sinks=sinks,
              edit=one_a_tile(KINDS[kinds]), **more)
    if form:
        p = B.sdllm_paged_plan(c.shape, c.op)
        assert (p.shared, p.block_cols, p.waves, p.least_tiles > 0) == form
    c.run()
    check_strictly(c)


# A step of the shared form takes two tiles of head_dim 64, of which one may be whole and the other masked: next to the diagonal, next to a tree's own
# rows, or where a share ends with an odd tile
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kinds", ["nan", "inf"])
@pytest.mark.parametrize("kind,Hq,n,lengths,window,form", [
    ("window", 1, 160, (0,), CAUSAL, (1, 256, 8, False)), ("window", 5, 160, (64, 0), ALL, (1, 256, 8, False)), ("window", 5, 60, (64, 5), (-1, 3, 2), (1, 256, 8, False)),
    ("window", 5, 64, (1200, 33), ALL, (1, 256, 8, True)), ("window", 5, 64, (1200, 33), (700, 0, 40), (1, 256, 8, True)),
    ("tree", 5, 33, (96, 30), None, (1, 256, 8, False)), ("tree", 5, 33, (1200, 30), None, (1, 256, 8, True))])
def test_whole_tiles_beside_masked_ones(d, kinds, kind, Hq, n, lengths, window, form):
    call(kind, Hq, 1, d, n, lengths, window, form=form, kinds=kinds)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kind,n,lengths,window,form", [
    ("window", 40, (88,) * 17, CAUSAL, (1, 128, 8, False)), ("window", 40, tuple(range(100, 117)), ALL, (1, 128, 8, False)),
    ("window", 40, (1000,) * 17, CAUSAL, (1, 128, 8, True)), ("tree", 40, tuple(range(60, 77)), None, (1, 128, 8, False)), ("tree", 40, (1000,) * 17, None, (1, 128, 8, True))])
def test_whole_tiles_beside_masked_ones_with_two_key_groups(d, kind, n, lengths, window, form):
    call(kind, 2, 1, d, n, lengths, window, form=form)


# Two key groups of a workgroup: where the tiles do not come out even, one group's tiles past the last are copies that count for nothing, whatever it has seen itself
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kinds", ["nan", "inf"])
@pytest.mark.parametrize("kind,Hq,n,lengths,window,form", [
    ("tree", 2, 40, tuple(range(1, 18)), None, (1, 128, 8, False)), ("tree", 4, 20, tuple(range(1, 18)), None, (1, 128, 8, False)),
    ("tree", 2, 40, (0,) * 17, None, (1, 128, 8, False)), ("window", 2, 40, (60,) * 17, (0, 0, 0), (1, 128, 8, False)),
    ("window", 4, 20, (20,) * 17, (0, 0, 0), (1, 128, 8, False)), ("window", 2, 40, tuple(range(100, 117)), ALL, (1, 128, 8, False)),
    ("window", 2, 40, (88,) * 17, CAUSAL, (1, 128, 8, False)), ("tree", 2, 40, tuple(range(900, 1002, 6)), None, (1, 128, 8, True)),
    ("window", 2, 40, tuple(range(900, 1002, 6)), CAUSAL, (1, 128, 8, True)), ("window", 2, 40, tuple(range(900, 1002, 6)), (300, 0, 7), (1, 128, 8, True))])
def test_copies_of_the_last_tile_count_for_nothing(d, kinds, kind, Hq, n, lengths, window, form):
    call(kind, Hq, 1, d, n, lengths, window, form=form, kinds=kinds)


# Every form by its name, streaming ones and fp32 among them
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kinds", ["nan", "inf"])
@pytest.mark.parametrize("kind,Hq,Hkv,n,lengths,window,dtype,form", [
    ("window", 16, 1, 1, (2000,), (1500, 0, 40), "bf16", (0, 16, 8, True)), ("window", 16, 1, 1, (300,), CAUSAL, "bf16", (0, 16, 8, False)),
    ("window", 3, 1, 1, (900,) * 65, CAUSAL, "bf16", (0, 16, 4, True)), ("window", 4, 4, 2, (100,) * 17, CAUSAL, "bf16", (0, 16, 4, False)),
    ("tree", 17, 1, 1, (2000,), None, "bf16", (0, 32, 8, True)), ("window", 2, 1, 50, (77,), (9, 3, 2), "bf16", (0, 32, 8, False)),
    ("tree", 2, 1, 64, (200, 33), None, "bf16", (0, 32, 8, False)), ("window", 2, 1, 30, (900,) * 65, CAUSAL, "bf16", (0, 32, 4, True)),
    ("tree", 8, 1, 8, (60,) * 65, None, "bf16", (0, 32, 4, False)), ("tree", 4, 2, 40, (70, 0), None, "bf16", (0, 32, 8, False))])
def test_streaming_forms(d, kinds, kind, Hq, Hkv, n, lengths, window, dtype, form):
    call(kind, Hq, Hkv, d, n, lengths, window, dtype, form, kinds)


@pytest.mark.parametrize("d,waves", [(64, 8), (128, 4)])
@pytest.mark.parametrize("kinds", ["nan", "inf"])
@pytest.mark.parametrize("kind,Hq,Hkv,n,lengths,window,cut", [
    ("window", 4, 2, 90, (100,), (9, 0, 2), False), ("window", 6, 2, 3, (2000, 31), CAUSAL, True), ("tree", 4, 2, 40, (70, 0), None, False),
    ("tree", 2, 1, 64, (3000, 33), None, True)])
def test_fp32(d, waves, kinds, kind, Hq, Hkv, n, lengths, window, cut):
    call(kind, Hq, Hkv, d, n, lengths, window, "f32", (0, 16, waves, cut), kinds)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("kind,window", [("window", (9, 0, 2)), ("tree", None)])
def test_keys_and_values_of_few_rows(dtype, d, kind, window):
    # keys that are no numbers make NaN of the rows that see them, values what they are; 180 and 80 columns
    def edit(k_pages, v_pages, c):
        if kind == "tree":
            c.v_blk[0, 0, 7, 3], c.v_blk[0, 1, 7, 5], c.v_blk[0, 1, 33, 5] = float("nan"), float("inf"), float("-inf")
            c.v_blk[1, 0, 20], c.k_blk[1, 1, 11] = float("-inf"), float("nan")
            return
        for j, x in ((130, float("nan")), (160, float("inf")), (161, float("-inf"))):
            v_pages[int(c.table[0, j // 32]), 0, j % 32, j % 7] = x
        k_pages[int(c.table[0, 150 // 32]), 1, 150 % 32, 2] = float("nan")
    n, lengths = (90, (100,)) if kind == "window" else (40, (70, 0))
    left, right, sinks = window or CAUSAL
    c = Paged(kind, 4, 2, d, n, lengths, dtype, mask=tree_masks(2, n, 1) if kind == "tree" else None, left=left, right=right, sinks=sinks, edit=edit)
    c.run()
    check_strictly(c)
