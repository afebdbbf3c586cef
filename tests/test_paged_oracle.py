"""The paged cache's oracle against hand-worked cases and plain torch."""
import numpy as np
import torch

from oracle import paged_oracle as pg


def test_rows_lie_where_the_table_says():
    pages = np.arange(3 * 1 * 16 * 2, dtype=float).reshape(3, 1, 16, 2)
    rows = pg.rows_of(pages, [2, 0], 18, 16)
    assert np.array_equal(rows[0, :16], pages[2, 0]) and np.array_equal(rows[0, 16:], pages[0, 0, :2])
    assert np.array_equal(pg.rows_of(pages, [9, -4], 17, 16)[0, 16], pages[0, 0, 0])


def test_windows_by_hand():
    show = lambda *a: ["".join("x" if v else "." for v in r) for r in pg.seen_window(*a)]
    assert show(2, 3, -1, 0, 0) == ["xxx..", "xxxx.", "xxxxx"]
    assert show(2, 3, 1, 0, 0) == [".xx..", "..xx.", "...xx"]
    assert show(2, 3, 0, 0, 1) == ["x.x..", "x..x.", "x...x"]
    assert show(0, 4, 1, 1, 0) == ["xx..", "xxx.", ".xxx", "..xx"]
    assert show(0, 3, 0, 0, 3) == ["x..", "xx.", "xxx"]          # first keys behind the row's limit stay hidden
    assert show(1, 2, 0, -1, 0) == [".xx", "..x"]


def test_trees_by_hand():
    show = lambda *a: ["".join("x" if v else "." for v in r) for r in pg.seen_tree(*a)]
    assert show(2, 3, [1, 3, 5]) == ["xxx..", "xxxx.", "xxx.x"]
    assert show(1, 2, None) == ["xxx", "xxx"]
    assert show(0, 2, [0, 6]) == ["..", ".x"]


def test_attention_is_the_softmax_of_what_is_seen():
    rng = np.random.default_rng(0)
    q, k, v = rng.standard_normal((5, 8)), rng.standard_normal((9, 8)), rng.standard_normal((9, 8))
    seen = rng.random((5, 9)) < 0.6
    seen[3] = False
    out, _ = pg.attention(q, k, v, seen, 0.3)
    bias = torch.where(torch.tensor(seen), 0.0, -torch.inf).double()
    want = torch.softmax(0.3 * torch.tensor(q) @ torch.tensor(k).T + bias, -1) @ torch.tensor(v)
    assert np.allclose(out[[0, 1, 2, 4]], want[[0, 1, 2, 4]].numpy(), atol=1e-14) and (out[3] == 0).all()
    v[2] = np.nan
    got, _ = pg.attention(q, k, v, seen, 0.3)
    assert np.array_equal(np.isnan(got).any(-1), seen[:, 2])


def test_appended_rows_by_hand():
    kp, vp = np.zeros((2, 1, 16, 64)), np.zeros((2, 1, 16, 64))
    k = np.ones((1, 1, 3, 64)) * np.array([1.0, 2, 3])[:, None]
    a, b = pg.append(kp, vp, k, -k, np.array([[1, 0]]), [15], [2], [[2, 0, 0]], None, page_rows=16, weight=None, inv_freq=np.zeros(0), rot=0, pairing=0, norm=False,
                     eps=0)
    assert (a[1, 0, 15] == 3).all() and (a[0, 0, 0] == 1).all() and (b == -a).all() and np.count_nonzero(a) == 128
