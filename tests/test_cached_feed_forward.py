"""The example of cached feed-forward sub-blocks: its block against float64, and the run as a whole."""
import math
import os
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))

pytestmark = pytest.mark.gpu


def test_block_against_float64():
    """One computed block.  Rounding to e4m3 (2^-4 of a value at most, about 0.026 in norm) enters three times of which two through sums of random signs: the
    activations (0.026 each way in norm) and the weights (0.026) of both layers: sqrt(4) * 0.026 = 0.05 of F, of which 0.08 is allowed."""
    from cached_feed_forward import CachedFeedForward
    M, D = 300, 512
    g = torch.Generator(device="cuda").manual_seed(1)

    def randn(*s):
        return torch.randn(*s, device="cuda", generator=g)

    W1, b1, W2, b2, gain = randn(4 * D, D) / math.sqrt(D), 0.1 * randn(4 * D), randn(D, 4 * D) / math.sqrt(4 * D), 0.1 * randn(D), 1 + 0.1 * randn(D)
    layer = CachedFeedForward(W1, b1, W2, b2, gain, M, 8)
    H, F0 = randn(1, M, D).bfloat16(), randn(1, M, D).bfloat16()
    h = H.double().cpu() + F0.double().cpu()
    F = layer.compute(H, F0).double().cpu()
    assert torch.equal(H.cpu(), h.float().bfloat16())
    y = h / (h.square().mean(-1, keepdim=True) + 1e-6).sqrt() * gain.double().cpu()
    z = torch.nn.functional.gelu(y @ W1.double().cpu().T + b1.double().cpu(), approximate="tanh")
    want = z @ W2.double().cpu().T + b2.double().cpu()
    assert float((F - want).norm() / want.norm()) < 0.08


def test_run():
    """Computed steps repeat themselves bit for bit, cached ones stay near the slowly turning stream: an angle of 0.05 a step moves it by 0.05 of its
    size a step, so by 0.15 after three; the forecast of the blocks' part is no further off than that."""
    from cached_feed_forward import run
    far = run(tokens=512, hidden=256, blocks=2, rank=32, steps=8, interval=4, say=lambda s: None)
    assert len(far) == 8 and far[0] == 0.0 and far[4] == 0.0
    assert all(0 < d < 0.3 for i, d in enumerate(far) if i % 4)
