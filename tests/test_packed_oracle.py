"""The oracle of the packed cache against values worked out by hand, and against itself byte by byte."""
import numpy as np

from oracle import packed_oracle as po


def test_numbers_ties_and_the_choice_of_the_step():
    x = np.zeros(32)
    x[:16] = [6, 5, 3.5, 2.5, 1.75, 1.25, 0.75, 0.25, -5.01, -3.49, -2.51, -1.74, -1.26, -0.74, -0.26, 0.24]
    want = [6, 4, 4, 2, 2, 1, 1, 0, -6, -3, -3, -1.5, -1.5, -0.5, -0.5, 0]
    assert po.group_values(x)[:16].tolist() == want
    assert po.group_codes(x)[0] == 0
    for top, e in ((7.0, 1), (6.999, 0), (3.5, 0), (3.4999, -1), (14, 2), (0.0, -125), (2.0 ** -140, -125), (2.0 ** 127 * 1.9, 125)):
        y = np.zeros(32)
        y[3] = -top
        assert po.group_codes(y)[0] == e, top
    y = np.full(32, 6.9)
    assert (po.group_values(y) == 6).all()                       # past the last number
    for bad in (np.nan, np.inf, -np.inf):
        y[7] = bad
        assert np.isnan(po.group_values(y)).all()


def test_groups_are_channels_of_a_key_and_rows_of_a_channel():
    rng = np.random.RandomState(0)
    k, v = rng.randn(40, 64), rng.randn(40, 64)
    kc, vc = po.cache_values(k, v)
    k2, v2 = k.copy(), v.copy()
    k2[5, 40] *= 1000
    v2[35, 9] *= 1000
    kd, vd = po.cache_values(k2, v2)
    changed = kd != kc
    assert changed[5, 32:].any() and not changed[5, :32].any() and not np.delete(changed, 5, 0).any()
    changed = vd != vc
    assert changed[32:, 9].any() and not changed[:32].any() and not np.delete(changed, 9, 1).any()


def test_bytes_hold_what_the_values_are():
    rng = np.random.RandomState(1)
    for d in (64, 128):
        k, v = rng.randn(45, d), rng.randn(45, d)
        v[2, 3] = np.nan
        tiles = po.cache_bytes(k, v)
        assert tiles.shape == (2, 34 * d)
        kc, vc = po.cache_values(k, v)
        number = lambda code: (-1.0 if code & 8 else 1.0) * po.MAGNITUDES[int(code) & 7]
        step = lambda b: np.nan if b == 255 else 2.0 ** (int(b) - 127)
        for r, ch in ((0, 0), (13, 37), (31, d - 1), (32, 5), (44, 63)):
            t, row = tiles[r // 32], r % 32
            byte = t[(ch // 32 * 32 + row) * 16 + ch % 32 // 2]
            assert number(byte >> 4 * (ch % 2) & 15) * step(t[32 * d + row * (d // 32) + ch // 32]) == kc[r, ch]
            m, rest = divmod(ch, d // 32)
            a, h, p = row // 8, row // 4 % 2, row % 4
            byte = t[16 * d + (((rest // 2 * 2 + h) * 32 + m) * 2 + rest % 2) * 8 + (4 * a + p) // 2]
            assert number(byte >> 4 * (p % 2) & 15) * step(t[33 * d + ch]) == vc[r, ch]
        assert (tiles[0, 33 * d + 3] == 255) and np.isnan(vc[:32, 3]).all() and not np.isnan(vc[32:, 3]).any()
        assert not (tiles[1, 16 * 13:16 * 32].any())                     # rows past the end


def test_norm_and_rotation_by_hand():
    x = np.zeros((1, 64))
    x[0, 0], x[0, 1], x[0, 8] = 3.0, 4.0, 5.0
    quarter = np.full(8, np.pi / 2)
    y = po.norm_rope(x, None, quarter, [1], rot=16, pairing=po.HALVES, norm=False, eps=0)
    assert np.allclose(y[0, [0, 1, 8, 9]], [-5, 0, 3, 4])
    y = po.norm_rope(x, None, quarter, [1], rot=16, pairing=po.ADJACENT, norm=False, eps=0)
    assert np.allclose(y[0, [0, 1, 8, 9]], [-4, 3, 0, 5])
    y = po.norm_rope(x, np.full(64, 2.0), quarter, [0], rot=16, pairing=po.HALVES, norm=True, eps=0)
    assert np.allclose(y, x / np.sqrt(50 / 64) * 2)
    # turning by positions that differ by the same amount leaves products alone
    rng = np.random.RandomState(2)
    q, k, f = rng.randn(1, 64), rng.randn(1, 64), 10000.0 ** -(np.arange(32) / 32)
    dots = [float((po.norm_rope(q, None, f, [5 + s], rot=64, pairing=p, norm=True, eps=1e-6) *
                   po.norm_rope(k, None, f, [2 + s], rot=64, pairing=p, norm=True, eps=1e-6)).sum()) for s in (0, 1000) for p in (0, 1)]
    assert np.isclose(dots[0], dots[2]) and np.isclose(dots[1], dots[3]) and not np.isclose(dots[0], dots[1])
