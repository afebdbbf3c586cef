"""One decoding block of one layer with the cache of 4 bits a value, from projections to attention output.

Every denoising step projects its positions (all of them while the sequence is recomputed, the block's alone afterwards), normalises and
turns queries and keys in place in the projection, and hands views of it to the block step:

    x W  ->  sdllm_qk_norm_rope  ->  sdllm_block_step_packed   (state 0, state 1, then state 2 to the end)

Nothing is copied between the calls and nothing is allocated by them.  A decoder that replays its steps as a HIP graph records the same calls.

    python -m examples.packed_block [--prompt 4096 --gen 256 --q-heads 28 --kv-heads 4 --steps 32]

prints the bytes of the cache, the time of a step that reuses it beside the bf16 cache's, and how far the outputs of the two are apart.
"""
from __future__ import annotations

import argparse

import torch

from paper_2508_02558_amd import binding as B

DEV = "cuda"


class Layer:
    """Projection and norm weights of one attention layer, random; rotation by halves."""

    def __init__(self, hidden, q_heads, kv_heads, head_dim=128, base=1e6, seed=0):
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        rn = lambda *s: torch.randn(*s, generator=g, device=DEV)
        self.q_heads, self.kv_heads, self.head_dim = q_heads, kv_heads, head_dim
        self.w_qkv = (rn(hidden, (q_heads + 2 * kv_heads) * head_dim) * hidden ** -0.5).bfloat16()
        self.q_norm, self.k_norm = ((1 + 0.1 * rn(head_dim)).bfloat16() for _ in range(2))
        half = torch.arange(0, head_dim, 2, device=DEV, dtype=torch.float64)
        self.inv_freq = (base ** (-half / head_dim)).float()

    def qkv(self, x, first):
        """Queries, keys and values [B, H, n, d] of positions first, first + 1, ...: views of one projection."""
        batch, n, _ = x.shape
        hq, hkv, d = self.q_heads, self.kv_heads, self.head_dim
        p = (x @ self.w_qkv).view(batch, n, hq + 2 * hkv, d).permute(0, 2, 1, 3)
        q, k, v = p[:, :hq], p[:, hq:hq + hkv], p[:, hq + hkv:]
        st = B.strides_of(p)
        shape = B.make_qk_shape(batch=batch, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, rows=n, dtype=B.SDLLM_BF16, pos_begin=first,
                                q_in_stride=st, k_in_stride=st, q_out_stride=st, k_out_stride=st)
        B.sdllm_qk_norm_rope(shape, q, k, self.q_norm, self.k_norm, self.inv_freq, None, q, k)
        return q, k, v


def decode_block(layer, x_full, x_steps, block_off, block_len, *, packed=True, retention=0.5, delay=1):
    """Outputs [steps, B, Hq, b, d] of a block's denoising steps.  x_full [B, L, hidden]: the layer's input of the whole sequence;
    x_steps [steps, B, b, hidden]: that of the block, which a step changes.  Also the cache, the retained positions, and the call of the last
    step that read the cache (None if there was none)."""
    batch, L, _ = x_full.shape
    hq, hkv, d, o, b = layer.q_heads, layer.kv_heads, layer.head_dim, block_off, block_len
    row = (hq + 2 * hkv) * d
    make = lambda **kw: B.make_shape(batch=batch, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, seq_len=L, block_off=o, block_len=b, dtype=B.SDLLM_BF16,
                                     retention=retention, **kw)
    kept = B.sdllm_retained_count(make())[0]
    shapes = {}
    for rows in (L, b):                                     # q rows of the block, k and v of `rows` positions, all views of a projection
        st = (rows * row, d, row)
        shapes[rows] = make(q_stride=st, kv_stride=(L * row, d, row), blk_stride=(b * row, d, row), cache_rows=kept)
    out = torch.empty(len(x_steps), batch, hq, b, d, dtype=torch.bfloat16, device=DEV)
    idx = torch.empty(batch, hkv, kept, dtype=torch.int32, device=DEV)
    op = B.SDLLM_OP_BLOCK_STEP_PACKED if packed else B.SDLLM_OP_BLOCK_STEP
    ws = torch.empty(max(B.sdllm_workspace_bytes(s, op) for s in shapes.values()), dtype=torch.uint8, device=DEV)
    if packed:
        cache = [torch.empty(B.sdllm_packed_cache_bytes(shapes[b], kept), dtype=torch.uint8, device=DEV)]
    else:
        cache = [torch.empty(batch, hkv, kept, d, dtype=torch.bfloat16, device=DEV) for _ in range(2)]

    def step(t, q, k, v, shape):
        if packed:
            return B.sdllm_block_step_packed(shape, t, delay, q, k, v, idx, cache[0], kept, out[t], ws)
        return B.sdllm_block_step(shape, t, delay, q, k, v, idx, cache[0], cache[1], out[t], ws)

    last = None
    for t in range(len(x_steps)):
        if B.sdllm_cache_state(t, delay) == B.SDLLM_STATE_REUSE:
            q, k, v = layer.qkv(x_steps[t], o)
            step(t, q, k, v, shapes[b])
            last = (t, q, k, v, shapes[b])
        else:
            x = x_full.clone()
            x[:, o:o + b] = x_steps[t]
            q, k, v = layer.qkv(x, 0)
            step(t, q[:, :, o:o + b], k, v, shapes[L])
    return out, cache, idx, last and (lambda: step(*last))


def inputs(batch, seq_len, block_off, block_len, hidden, steps, seed=1):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    x = torch.randn(batch, seq_len, hidden, generator=g, device=DEV)
    blk = x[:, block_off:block_off + block_len]
    drift = torch.randn(steps, batch, block_len, hidden, generator=g, device=DEV)
    return x.bfloat16(), (0.9 * blk + 0.45 * drift).bfloat16()


def _time_us(call, n=200):
    for _ in range(20):
        call()
    a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    a.record()
    for _ in range(n):
        call()
    b.record()
    torch.cuda.synchronize()
    return a.elapsed_time(b) * 1e3 / n


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, default in (("batch", 1), ("prompt", 4096), ("gen", 256), ("block", 32), ("q-heads", 28), ("kv-heads", 4), ("hidden", 2048), ("steps", 32)):
        ap.add_argument("--" + name, type=int, default=default)
    a = ap.parse_args()
    if a.steps < 3:
        ap.error("--steps: the third is the first that reuses the cache")
    layer = Layer(a.hidden, a.q_heads, a.kv_heads)
    x, x_steps = inputs(a.batch, a.prompt + a.gen, a.prompt, a.block, a.hidden, a.steps)
    got = {}
    for packed in (False, True):
        out, cache, _, reuse = decode_block(layer, x, x_steps, a.prompt, a.block, packed=packed)
        got[packed] = out.float()
        held = sum(c.numel() * c.element_size() for c in cache)
        print(f"{'4 bits' if packed else 'bf16':>7}: cache {held / 2 ** 20:8.2f} MiB, step over it {_time_us(reuse):7.2f} us")
    diff = (got[True][2:] - got[False][2:]).norm() / got[False][2:].norm()
    print(f"outputs of the steps that reuse the cache: {diff:.3f} apart (relative, 2-norm)")


if __name__ == "__main__":
    main()
