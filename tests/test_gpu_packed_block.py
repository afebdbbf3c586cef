"""The example that runs norm and rotation, the packed cache and its attention together, against float64 from the same projections."""
import numpy as np
import pytest
import torch

from examples import packed_block as ex
from oracle import packed_oracle as po
from tests.test_gpu_attn_packed import compare

pytestmark = pytest.mark.gpu


def host(t):
    return t.detach().cpu().double().numpy()


@pytest.mark.parametrize("q_heads,kv_heads,block", [(4, 4, 32), (7, 1, 32), (4, 2, 16)])
def test_a_block_of_a_layer(q_heads, kv_heads, block):
    prompt, hidden, steps, batch = 400, 256, 4, 2
    L, o = prompt + 2 * block, prompt
    layer = ex.Layer(hidden, q_heads, kv_heads)
    x, x_steps = ex.inputs(batch, L, o, block, hidden, steps)
    out, cache, idx, again = ex.decode_block(layer, x, x_steps, o, block)
    torch.cuda.synchronize()
    first = out.clone()
    again()
    torch.cuda.synchronize()
    assert torch.equal(out, first)                           # the last step's call, made once more
    dense, _, idx_dense, _ = ex.decode_block(layer, x, x_steps, o, block, packed=False)
    torch.cuda.synchronize()
    assert torch.equal(out[:2], dense[:2])                   # the steps that do not read the cache
    assert torch.equal(idx, idx_dense)
    # step 3 from its own projection, over the rows that step 1 retained
    d = layer.head_dim
    full = x.clone()
    full[:, o:o + block] = x_steps[1]
    _, k1, v1 = (host(t) for t in layer.qkv(full, 0))
    q3, k3, v3 = layer.qkv(x_steps[3], o)
    torch.cuda.synchronize()
    pick = idx.cpu().numpy().astype(int)[..., None]
    kc, vc = po.cache_values(np.take_along_axis(k1, pick, 2), np.take_along_axis(v1, pick, 2))
    compare(out[3], q3, kc, vc, k3, v3, d ** -0.5, "bf16")


def test_the_cache_is_a_quarter():
    layer = ex.Layer(256, 4, 4)
    x, x_steps = ex.inputs(1, 1120, 1024, 32, 256, 3)
    sizes = []
    for packed in (True, False):
        _, cache, _, _ = ex.decode_block(layer, x, x_steps, 1024, 32, packed=packed)
        sizes.append(sum(c.numel() * c.element_size() for c in cache))
    kept = 544
    assert sizes[0] == 4 * kept // 32 * 34 * 128 and sizes[1] == 2 * 2 * 4 * kept * 128
