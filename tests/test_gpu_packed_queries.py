"""Logits over the packed cache are those of the queries as they are given, however unlike their channels."""
import pytest
import torch

from tests.test_gpu_attn_packed import Call

pytestmark = pytest.mark.gpu


# one to three tiles of the cache to a wavefront, and more
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("heads,n", [(2, 200), (8, 700), (64, 1290)])
@pytest.mark.parametrize("power", [14, 18, 21, 60])
def test_a_channel_far_above_the_others(d, heads, n, power):
    # the keys are zero there, so that the others alone make the logits
    def edit(k, v, c):
        k[..., 5] = 0
        c.kb[..., 5] = 0
        c.q[..., 5] = 2.0 ** power
    c = Call(1, heads, heads, d, 32, n, "bf16", edit=edit, scale=0.5)
    c.run()
    c.check()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("heads,n", [(2, 200), (64, 1290)])
def test_queries_of_all_magnitudes_at_once(d, heads, n):
    # channels fall by powers of two, and the keys' groups grow so that each group of 32 has its part in the logits
    def edit(k, v, c):
        power = torch.arange(d, dtype=torch.float32) % 32
        c.q.mul_((2.0 ** -power).to(c.q.device))
        k.mul_(2.0 ** (power - 16))
        c.kb.mul_((2.0 ** (power - 16)).to(c.kb.device))
    c = Call(1, heads, heads, d, 32, n, "bf16", edit=edit, scale=2.0 ** 14)
    c.run()
    c.check()
