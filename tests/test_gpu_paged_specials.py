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
