"""Attention of drafted trees over the paged cache against the float64 oracle."""
import pytest
import torch

from tests.paged_util import DEV, Paged, ints, tree_masks

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Hq,Hkv,n", [(2, 2, 32), (7, 1, 32), (4, 2, 1), (8, 1, 7), (3, 3, 33), (2, 1, 64), (20, 1, 64)])
@pytest.mark.parametrize("lengths,page_rows", [((0,), 32), ((1, 31), 16), ((33, 100, 0), 16), ((517, 64), 64), ((300,), 256)])
def test_against_the_oracle(dtype, d, Hq, Hkv, n, lengths, page_rows):
    c = Paged("tree", Hq, Hkv, d, n, lengths, dtype, page_rows=page_rows, mask=tree_masks(len(lengths), n, 3))
    c.run()
    c.check()


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("Hq,Hkv,n,lengths", [(1, 1, 32, (4099,)), (4, 1, 16, (2500, 3, 900)), (14, 2, 1, (6001, 17)), (28, 4, 40, (1111, 2222, 0, 700)),
                                              (64, 64, 5, (150,) * 9), (2, 1, 3, tuple(range(0, 700, 7)))])
def test_splits_and_full_grids(dtype, d, Hq, Hkv, n, lengths):
    c = Paged("tree", Hq, Hkv, d, n, lengths, dtype, page_rows=64, layout="rows", mask=tree_masks(len(lengths), n, 5))
    c.run()
    c.check()


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
def test_no_mask_is_a_block(dtype, d):
    c = Paged("tree", 6, 3, d, 37, (300, 0), dtype, counts=(37, 20))
    c.run()
    c.check()


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("counts", [(0, 9, 64), (64, 0, 1), (-3, 70, 33)])
def test_counts_and_rows_that_see_nothing(dtype, d, counts):
    masks = tree_masks(3, 64, 9)
    masks[0][0] = masks[1][5] = masks[2][40] = 0          # with no cache rows: nothing
    masks[1][3] = -1                                      # bits of rows that are not there count for nothing
    c = Paged("tree", 4, 2, d, 64, (0, 0, 45), dtype, counts=counts, mask=masks)
    c.run()
    c.check()


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64)])
def test_one_mask_for_all(dtype, d):
    c = Paged("tree", 4, 2, d, 21, (40, 300), dtype, mask=tree_masks(1, 21, 2) * 2)
    c.shape.mask_stride = 0
    c.run()
    c.check()


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
def test_what_is_not_seen_may_be_anything(dtype, d):
    # rows that only some of the tree see are not finite: those rows alone get them
    masks = tree_masks(2, 40, 1)

    def edit(k_pages, v_pages, c):
        c.v_blk[0, 0, 7, 3] = float("nan")
        c.v_blk[0, 1, 7, 5] = float("inf")
        c.v_blk[0, 1, 33, 5] = float("-inf")
        c.v_blk[1, 0, 20] = float("-inf")
        c.k_blk[1, 1, 11] = float("nan")
    c = Paged("tree", 4, 2, d, 40, (70, 0), dtype, mask=masks, edit=edit)
    c.run()
    c.check()


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 128)])
def test_one_key_takes_nearly_all(dtype, d):
    def edit(k_pages, v_pages, c):
        q = c.q[0, :, 3]
        page, row = c.table[0, 300 // 32], 300 % 32
        k_pages[page, :, row] = q * 3
    c = Paged("tree", 2, 2, d, 8, (700,), dtype, mask=tree_masks(1, 8, 1), edit=edit, scale=0.5)
    c.run()
    c.check()


def test_an_empty_pool_leaves_the_rows_themselves():
    c = Paged("tree", 4, 2, 128, 9, (0, 0), "bf16", spare=0, mask=tree_masks(2, 9, 4), table_pages=0)
    c.run()
    c.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_lengths_are_held_to_the_table_and_pages_to_the_pool(dtype):
    c = Paged("tree", 4, 2, 64, 5, (64, 64), dtype, mask=tree_masks(2, 5, 4), table_pages=2)
    c.lengths = ints([1000000, -5])
    c.run()
    c.check()
    pages = c.k_pages.shape[0]
    c.k_pages[:], c.v_pages[:] = torch.randn_like(c.k_pages), torch.randn_like(c.v_pages)
    c.lengths = ints([64, 40])
    c.table[0, 1], c.table[1, 0] = pages + 1000, -1000000
    c.out.fill_(float("nan"))
    c.run()
    c.check()
