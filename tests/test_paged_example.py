"""The paged example's command on the CPU: what it refuses before it looks for a GPU."""
import sys

import pytest

from examples import paged_serving as ex


@pytest.mark.parametrize("args,name", [(["--prompts", "4,0"], "--prompts"), (["--tree", "65"], "--tree"), (["--tree", "0"], "--tree"), (["--tokens", "0"], "--tokens")])
def test_what_cannot_be_served(monkeypatch, capsys, args, name):
    monkeypatch.setattr(sys, "argv", ["paged_serving", *args])
    with pytest.raises(SystemExit) as end:
        ex.main()
    assert end.value.code == 2 and name in capsys.readouterr().err
