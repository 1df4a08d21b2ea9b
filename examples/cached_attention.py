"""Attention sub-blocks whose linear layers run in 8 bits and whose outputs are cached between full-compute steps.

    python examples/cached_attention.py [--frames 2] [--height 32] [--width 32] [--text 128] [--heads 8] [--head-dim 128] [--rank 32] [--steps 12] [--interval 4]

The sequence is `text` text tokens, padded from `text_used` on, and frames x height x width tokens of a video.  The angles of their positions are made once (rotary_table: the
grid stays).  Every `interval`-th time step is computed: the residual stream takes the output F of the step before and is normed into 8 bits (rms_norm8), goes through the product
for queries, keys and values (matmul8), queries and keys are normed and turned by head in place (norm_rotate), attend to all keys but the padding (attention), and the result goes
in 8 bits (quantize8) through the product behind the attention (matmul8) as F, which the cache step keeps.  At the other steps F is forecast.  Random weights; the inputs turn
slowly, as a sampler's do.  Prints, for each time step, its time and how far the cached stream is from the computed one.
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2601_07396_amd as svdc  # noqa: E402


def grid_positions(text, frames, height, width, device):
    """[tokens, 3]: text at the origin, then (frame, row, column) of each token of the video."""
    i = torch.arange(frames * height * width, device=device)
    grid = torch.stack([i // (height * width), i // width % height, i % width], 1)
    return torch.cat([torch.zeros(text, 3, device=device, dtype=grid.dtype), grid]).to(torch.int32)


class CachedAttention:
    """One sub-block: attention of normed and turned heads of norm(H) W_qkv^T, times W_out^T, its basis and its cached state."""

    def __init__(self, W_qkv, W_out, gain, gain_q, gain_k, table, keep, heads, rank, alpha=0.1):
        tokens, dev = table.shape[0], W_qkv.device
        self.D, self.wide, self.heads, self.rank, self.alpha = W_qkv.shape[1], W_out.shape[1], heads, rank, alpha
        self.d = self.wide // heads
        self.W_qkv, self.W_out = svdc.quantize8(W_qkv, 128), svdc.quantize8(W_out, 128)      # (values, scales), once
        self.gain, self.gain_q, self.gain_k, self.table, self.keep = gain.float(), gain_q.float(), gain_k.float(), table, keep
        # what the calls below need, allocated once
        self.A, self.B = svdc.alloc_q8(tokens, self.D, dev), svdc.alloc_q8(tokens, self.wide, dev)
        self.qkv = torch.empty(tokens, 3 * self.wide, device=dev, dtype=torch.bfloat16)
        self.q, self.k, self.v = (t.unflatten(2, (heads, self.d)) for t in self.qkv[None].split(self.wide, 2))
        self.o = torch.empty(1, tokens, heads, self.d, device=dev, dtype=torch.bfloat16)
        self.F = torch.empty(1, tokens, self.D, device=dev, dtype=torch.bfloat16)
        self.into = svdc.make_matmul8(tokens, 3 * self.wide, self.D, torch.bfloat16)
        self.turn = svdc.make_norm_rotate(self.q, self.k, None, self.q, self.k, None, table)
        self.attend = svdc.make_attention(self.q, self.k, self.v, self.o)
        self.quant = svdc.make_quant8(self.o.view(tokens, self.wide))
        self.out = svdc.make_matmul8(tokens, self.D, self.wide, torch.bfloat16)
        self.workspaces = [svdc.alloc_matmul8_workspace(self.into, dev), svdc.alloc_attention_workspace(self.attend, dev), svdc.alloc_matmul8_workspace(self.out, dev)]
        self.shape = svdc.make_shape(self.F, rank)
        self.R, self.S, self.V = torch.empty_like(self.F), torch.empty(1, tokens, rank, device=dev), None

    def compute(self, H, F_before):
        """F for the stream H + F_before; H is updated in place."""
        svdc.svdcache_rms_norm8(svdc.make_norm8(H, F_before, H), H, F_before, self.gain, H, None, *self.A)
        svdc.svdcache_matmul8(self.into, *self.A, *self.W_qkv, None, self.qkv, None, self.workspaces[0])
        svdc.svdcache_norm_rotate(self.turn, self.q, self.k, None, self.gain_q, self.gain_k, self.table, self.q, self.k, None)
        svdc.svdcache_attention(self.attend, self.q, self.k, self.v, self.o, None, None, self.keep, self.workspaces[1])
        svdc.svdcache_quantize8(self.quant, self.o.view(-1, self.wide), *self.B)
        svdc.svdcache_matmul8(self.out, *self.B, *self.W_out, None, self.F[0], None, self.workspaces[2])
        return self.F

    def keep_step(self):
        """The cache step of a computed F; the basis is fitted once, to the first one."""
        first = self.V is None
        if first:
            self.V = svdc.fit_basis(self.F, self.rank)[0]
            self.packed = svdc.pack_basis(self.shape, self.V)
        svdc.svdcache_full_step(self.shape, self.F, self.V, self.packed, self.R, self.S, None, self.alpha, first)

    def add_forecast(self, H):
        """H += the forecast of F."""
        svdc.svdcache_forecast_combine(self.shape, [self.S], [1.0], self.V, self.packed, self.R, H, H)


def run(frames=2, height=32, width=32, text=128, text_used=40, heads=8, head_dim=128, rank=32, steps=12, interval=4, seed=0, say=print):
    """[relative distance of the cached stream from the computed one, for each time step]"""
    dev = torch.device("cuda:0")
    g = torch.Generator(device=dev).manual_seed(seed)

    def randn(*shape):
        return torch.randn(*shape, device=dev, generator=g)

    D, tokens = heads * head_dim, text + frames * height * width
    side = head_dim * 3 // 16 * 2                                                          # columns of the height and of the width; time has the others
    table = svdc.rotary_table(grid_positions(text, frames, height, width, dev), (head_dim - 2 * side, side, side))
    keep = torch.ones(1, tokens, device=dev, dtype=torch.uint8)
    keep[:, text_used:text] = 0
    block = CachedAttention(randn(3 * D, D) / math.sqrt(D), randn(D, D) / math.sqrt(D), 1 + 0.1 * randn(D), 1 + 0.1 * randn(head_dim), 1 + 0.1 * randn(head_dim), table, keep,
                            heads, rank)
    U, A, B = randn(tokens, 48), randn(48, D), randn(48, D)
    zero = torch.zeros(1, tokens, D, device=dev, dtype=torch.bfloat16)
    marks = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
    far = []
    for t in range(steps):
        angle = 0.05 * t
        X = ((U @ (math.cos(angle) * A + math.sin(angle) * B)) / 7).bfloat16()[None]       # a low-rank stream that turns slowly
        full = t % interval == 0
        H = X.clone()
        want = H + block.compute(H, zero)
        torch.cuda.synchronize()
        marks[0].record()
        out = X.clone()
        if full:
            out = out + block.compute(out, zero)
            block.keep_step()
        else:
            block.add_forecast(out)
        marks[1].record()
        torch.cuda.synchronize()
        far.append(float((out.float() - want.float()).norm() / want.float().norm()))
        say(f"step {t:2d} {'cached' if not full else 'computed' if t else 'first':8s} {1e3 * marks[0].elapsed_time(marks[1]):8.1f} us   distance {far[-1]:.4f}")
    return far


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("frames", 2), ("height", 32), ("width", 32), ("text", 128), ("text-used", 40), ("heads", 8), ("head-dim", 128), ("rank", 32), ("steps", 12), ("interval", 4)):
        ap.add_argument("--" + name, type=int, default=value)
    run(**vars(ap.parse_args()))
