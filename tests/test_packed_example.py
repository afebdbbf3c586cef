"""The example's command on the CPU: what it refuses before it looks for a GPU."""
import sys

import pytest

from examples import packed_block as ex


@pytest.mark.parametrize("steps", ["0", "1", "2", "-1"])
def test_a_block_that_never_reuses_its_cache_has_nothing_to_compare(monkeypatch, capsys, steps):
    monkeypatch.setattr(sys, "argv", ["packed_block", "--steps", steps])
    with pytest.raises(SystemExit) as end:
        ex.main()
    assert end.value.code == 2 and "--steps" in capsys.readouterr().err
