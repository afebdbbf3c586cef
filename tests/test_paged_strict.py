"""The comparison of results that are no numbers, on results that are wrong."""
import numpy as np

from tests.paged_strict import same_classes


def test_what_is_told_apart():
    inf, nan = np.inf, np.nan
    want = np.array([1.0, inf, -inf, nan])
    assert same_classes(np.array([3.0, inf, -inf, nan]), want)
    for i, wrong in ((0, inf), (0, nan), (1, 2.0), (1, -inf), (1, nan), (2, -2.0), (2, inf), (3, 0.0), (3, inf)):
        got = want.copy()
        got[i] = wrong
        assert not same_classes(got, want), (i, wrong)
