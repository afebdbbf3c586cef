"""Attention with a window and first keys over the paged cache against the float64 oracle."""
import pytest
import torch

from tests.paged_util import DEV, Paged, ints

pytestmark = pytest.mark.gpu

WINDOWS = [(-1, 0, 0), (-1, -1, 0), (0, 0, 0), (31, 0, 4), (40, 17, 33), (100, 0, 1), (5, -1, 70), (-1, 3, 2), (63, 2000000000, 2000000000), (2147483647, 0, 0)]


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("window", WINDOWS)
@pytest.mark.parametrize("Hq,Hkv,n,lengths,page_rows", [(7, 1, 1, (0, 1, 200), 16), (4, 2, 45, (33, 0), 32), (3, 3, 130, (77,), 64), (8, 1, 70, (5, 260), 128)])
def test_against_the_oracle(dtype, d, window, Hq, Hkv, n, lengths, page_rows):
    left, right, sinks = window
    c = Paged("window", Hq, Hkv, d, n, lengths, dtype, page_rows=page_rows, left=left, right=right, sinks=sinks)
    c.run()
    c.check()


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("window", [(-1, 0, 0), (511, 0, 5), (2000, 30, 100)])
@pytest.mark.parametrize("Hq,Hkv,n,lengths", [(1, 1, 1, (4099,)), (28, 4, 1, (2500, 3, 900, 0)), (14, 2, 1, tuple(range(0, 700, 7))), (4, 1, 333, (3000,)),
                                              (64, 64, 2, (150,) * 9), (2, 1, 600, (0, 100))])
def test_splits_and_full_grids(dtype, d, window, Hq, Hkv, n, lengths):
    left, right, sinks = window
    c = Paged("window", Hq, Hkv, d, n, lengths, dtype, page_rows=64, layout="rows", left=left, right=right, sinks=sinks)
    c.run()
    c.check()


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("counts", [(0, 9, 80), (80, 0, 1), (-3, 90, 33)])
def test_counts(dtype, d, counts):
    c = Paged("window", 4, 2, d, 80, (0, 50, 45), dtype, counts=[min(max(x, 0), 80) for x in counts], left=20, right=5, sinks=3)
    c.counts = ints(counts)
    c.run()
    c.check()


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("page_rows", [16, 32, 64])
def test_pages_outside_the_window_may_be_gone(dtype, d, page_rows):
    # one token at place 300 sees 0-4 and 237-300: other pages are not in the table, rows of theirs that stayed hold NaN
    def edit(k_pages, v_pages, c):
        for j in range(5, 237):
            page = int(c.table[0, j // page_rows])
            k_pages[page, :, j % page_rows], v_pages[page, :, j % page_rows] = float("nan"), float("inf")
        for i in range(-(-5 // page_rows), 237 // page_rows):
            c.table[0, i] = -1
    c = Paged("window", 8, 2, d, 1, (300,), dtype, page_rows=page_rows, left=63, right=0, sinks=5, edit=edit)
    c.run()
    c.check()


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
def test_what_is_not_seen_may_be_anything(dtype, d):
    def edit(k_pages, v_pages, c):
        for j, x in ((130, float("nan")), (160, float("inf")), (161, float("-inf"))):
            page = int(c.table[0, j // 32])
            v_pages[page, 0, j % 32, j % 7] = x
        k_pages[int(c.table[0, 150 // 32]), 1, 150 % 32, 2] = float("nan")
    c = Paged("window", 4, 2, d, 90, (100,), dtype, left=9, right=0, sinks=2, edit=edit)
    c.run()
    c.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_past_the_table_see_what_there_is(dtype):
    c = Paged("window", 4, 2, 64, 40, (30, 64), dtype, counts=(2, 0), left=3, right=1, sinks=1, table_pages=2, page_rows=32)
    c.lengths, c.counts = ints([30, 1000]), ints([40, 40])
    c.k_pages.copy_(torch.randn_like(c.k_pages))
    c.v_pages.copy_(torch.randn_like(c.v_pages))
    c.q.copy_(torch.randn_like(c.q))
    c.table[:] = ints([[1, 0], [2, 0]])
    c.run()
    c.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_an_empty_pool_gives_zeros(dtype):
    c = Paged("window", 4, 2, 128, 3, (0, 0), dtype, spare=0, table_pages=0, counts=(0, 0))
    c.counts = None
    c.run()
    torch.cuda.synchronize()
    assert (c.out == 0).all()
