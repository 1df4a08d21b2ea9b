"""Feed-forward sub-blocks in 8 bits whose outputs are cached between full-compute steps.

    python examples/cached_feed_forward.py [--tokens 4608] [--hidden 3072] [--blocks 2] [--rank 32] [--steps 12] [--interval 4]

Every `interval`-th time step is computed: each block takes the residual stream H with the output F of the block before it (rms_norm8: H += F, the norm in
8 bits), goes through its two linear layers in 8 bits (matmul8: up with GELU, the result in 8 bits again; down in bfloat16), and hands F to the cache step
(full step: coefficients, residual, running mean).  At the other steps each block's F is forecast and added to the stream in one call.  Random
weights; the inputs drift slowly, as a sampler's do.  Prints, for each time step, its time (of a computed one with its cache steps, of the first with the fit of the
bases too) and how far the cached stream is from the computed one.
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2601_07396_amd as svdc  # noqa: E402


class CachedFeedForward:
    """One block: act(norm(H) W1^T + b1) W2^T + b2 with W1 [4 D, D] and W2 [D, 4 D], its basis and its cached state."""

    def __init__(self, W1, b1, W2, b2, gain, tokens, rank, alpha=0.1):
        self.D, self.wide, self.rank, self.alpha = W1.shape[1], W1.shape[0], rank, alpha
        self.W1, self.W2 = svdc.quantize8(W1, 128), svdc.quantize8(W2, 128)      # (values, scales), once
        self.b1, self.b2, self.gain = b1.float(), b2.float(), gain.float()
        dev, D, wide = W1.device, self.D, self.wide
        # what the calls below need, allocated once
        self.Q, self.Z = svdc.alloc_q8(tokens, D, dev), svdc.alloc_q8(tokens, wide, dev)
        self.F = torch.empty(1, tokens, D, device=dev, dtype=torch.bfloat16)
        self.up = svdc.make_matmul8(tokens, wide, D, torch.float8_e4m3fn, "gelu")
        self.down = svdc.make_matmul8(tokens, D, wide, torch.bfloat16)
        self.workspaces = [svdc.alloc_matmul8_workspace(p, dev) for p in (self.up, self.down)]
        self.shape = svdc.make_shape(self.F, rank)
        self.R, self.S, self.V = torch.empty_like(self.F), torch.empty(1, tokens, rank, device=dev), None

    def compute(self, H, F_before):
        """F for the stream H + F_before; H is updated in place."""
        svdc.svdcache_rms_norm8(svdc.make_norm8(H, F_before, H), H, F_before, self.gain, H, None, *self.Q)
        svdc.svdcache_matmul8(self.up, *self.Q, *self.W1, self.b1, *self.Z, self.workspaces[0])
        svdc.svdcache_matmul8(self.down, *self.Z, *self.W2, self.b2, self.F[0], None, self.workspaces[1])
        return self.F

    def keep(self):
        """The cache step of a computed F; the basis is fitted once, to the first one."""
        first = self.V is None
        if first:
            self.V = svdc.fit_basis(self.F, self.rank)[0]
            self.packed = svdc.pack_basis(self.shape, self.V)
        svdc.svdcache_full_step(self.shape, self.F, self.V, self.packed, self.R, self.S, None, self.alpha, first)

    def add_forecast(self, H):
        """H += the forecast of F."""
        svdc.svdcache_forecast_combine(self.shape, [self.S], [1.0], self.V, self.packed, self.R, H, H)


def run(tokens=4608, hidden=3072, blocks=2, rank=32, steps=12, interval=4, seed=0, say=print):
    """[relative distance of the cached stream from the computed one, for each time step]"""
    dev = torch.device("cuda:0")
    g = torch.Generator(device=dev).manual_seed(seed)

    def randn(*shape):
        return torch.randn(*shape, device=dev, generator=g)

    D, wide = hidden, 4 * hidden
    layers = [CachedFeedForward(randn(wide, D) / math.sqrt(D), 0.1 * randn(wide), randn(D, wide) / math.sqrt(wide), 0.1 * randn(D), 1 + 0.1 * randn(D), tokens, rank)
              for _ in range(blocks)]
    U, A, B = randn(tokens, 48), randn(48, D), randn(48, D)
    zero = torch.zeros(1, tokens, D, device=dev, dtype=torch.bfloat16)
    marks = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
    far = []
    for t in range(steps):
        angle = 0.05 * t
        X = ((U @ (math.cos(angle) * A + math.sin(angle) * B)) / 7).bfloat16()[None]       # a low-rank stream that turns slowly

        def computed(keep):
            H, F = X.clone(), zero
            for layer in layers:
                F = layer.compute(H, F)
                if keep:
                    layer.keep()
            return H + F

        full = t % interval == 0
        want = computed(keep=False)
        torch.cuda.synchronize()
        marks[0].record()
        if full:
            out = computed(keep=True)
        else:
            out = X.clone()
            for layer in layers:
                layer.add_forecast(out)
        marks[1].record()
        torch.cuda.synchronize()
        far.append(float((out.float() - want.float()).norm() / want.float().norm()))
        kind = "cached" if not full else "computed" if t else "first"
        say(f"step {t:2d} {kind:8s} {1e3 * marks[0].elapsed_time(marks[1]):8.1f} us   distance {far[-1]:.4f}")
    return far


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("tokens", 4608), ("hidden", 3072), ("blocks", 2), ("rank", 32), ("steps", 12), ("interval", 4)):
        ap.add_argument("--" + name, type=int, default=value)
    run(**vars(ap.parse_args()))
