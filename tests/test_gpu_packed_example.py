"""Blocks of so few steps that none reads the cache."""
import pytest
import torch

from examples import packed_block as ex

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("steps", [1, 2])
def test_no_step_to_repeat(steps):
    layer = ex.Layer(256, 4, 4)
    x, x_steps = ex.inputs(1, 432, 400, 32, 256, steps)
    out, _, _, again = ex.decode_block(layer, x, x_steps, 400, 32)
    torch.cuda.synchronize()
    assert again is None and torch.isfinite(out).all()


def test_the_command(monkeypatch, capsys):
    monkeypatch.setattr("sys.argv", ["packed_block", "--prompt", "256", "--gen", "64", "--hidden", "256", "--q-heads", "4", "--kv-heads", "2", "--steps", "3"])
    ex.main()
    said = capsys.readouterr().out
    assert "4 bits: cache" in said and "bf16: cache" in said and "apart" in said
