"""The example of cached attention sub-blocks: its operators in a row against float64, and the run as a whole."""
import os
import sys

import pytest
import torch

import paper_2601_07396_amd as svdc

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))

pytestmark = pytest.mark.gpu


def make(tokens, D, heads, d, text, seed=1):
    from cached_attention import CachedAttention, grid_positions
    g = torch.Generator(device="cuda").manual_seed(seed)

    def randn(*s):
        return torch.randn(*s, device="cuda", generator=g)
    pos = grid_positions(text, 1, (tokens - text) // 10, 10, "cuda")
    table = svdc.rotary_table(pos, (d // 4, d // 4 + d // 8, d // 4 + d // 8))
    keep = torch.ones(1, tokens, device="cuda", dtype=torch.uint8)
    keep[:, text // 3:text] = 0
    W_qkv, W_out, gain = randn(3 * heads * d, D) / D ** 0.5, randn(D, heads * d) / (heads * d) ** 0.5, 1 + 0.1 * randn(D)
    block = CachedAttention(W_qkv, W_out, gain, 1 + 0.1 * randn(d), 1 + 0.1 * randn(d), table, keep, heads, 8)
    return block, W_qkv, W_out, pos, randn(1, tokens, D).bfloat16(), randn(1, tokens, D).bfloat16()


def test_block_against_float64():
    """One computed sub-block.  Rounding to e4m3 is 2^-4 of a value at most, about 0.026 in norm; through sums of random signs it stays that.  It enters by the activations and the weights of
    both products: 0.037 of queries, keys and values each, 0.037 of what comes out.  Logits are sums of products of unit size, so that errors of 0.037 of queries and keys move them by
    0.05 and the probabilities by 0.05 of themselves: in norm 0.05 of the values' part; in all sqrt(0.037^2 * 2 + 0.05^2) = 0.07 of F, of which 0.11 is allowed."""
    tokens, D, heads, d, text = 350, 512, 4, 128, 60
    block, W_qkv, W_out, pos, H, F0 = make(tokens, D, heads, d, text)
    h = H.double() + F0.double()
    F = block.compute(H, F0).double()
    y = h / (h.square().mean(-1, keepdim=True) + 1e-6).sqrt() * block.gain.double()
    q, k, v = (t.unflatten(-1, (heads, d)) for t in (y @ W_qkv.double().T.contiguous()).split(heads * d, -1))
    dims = (d // 4, d // 4 + d // 8, d // 4 + d // 8)
    angle = torch.cat([pos[:, a:a + 1].double() * 10000.0 ** (-torch.arange(0, n, 2, device="cuda").double() / n) for a, n in enumerate(dims)], 1)[None, :, None]

    def turned(x, gain):
        x = x / (x.square().mean(-1, keepdim=True) + 1e-6).sqrt() * gain.double()
        a, b = x[..., ::2], x[..., 1::2]
        return torch.stack([a * angle.cos() - b * angle.sin(), a * angle.sin() + b * angle.cos()], -1).flatten(-2)
    q, k, v = turned(q, block.gain_q).transpose(1, 2), turned(k, block.gain_k).transpose(1, 2), v.transpose(1, 2)
    s = q @ k.transpose(2, 3).contiguous() / d ** 0.5
    s = s.masked_fill(block.keep[:, None, None, :] == 0, -float("inf"))
    want = (s.softmax(-1) @ v).transpose(1, 2).flatten(2) @ W_out.double().T.contiguous()
    assert float((F - want).norm() / want.norm()) < 0.11


def test_padding_does_not_matter():
    """What the padded text holds changes no other token's F."""
    block, _, _, _, H, F0 = make(350, 512, 4, 128, 60)
    F = block.compute(H.clone(), F0).clone()
    other = H.clone()
    other[:, 20:60] = 3.0
    again = block.compute(other, F0)
    assert torch.equal(F[:, :20], again[:, :20]) and torch.equal(F[:, 60:], again[:, 60:])


def test_captured_together():
    """The whole sub-block in a graph, replayed on new inputs with eager work in between, gives the eager calls' bits."""
    block, _, _, _, H, F0 = make(350, 512, 4, 128, 60)
    g = torch.Generator(device="cuda").manual_seed(2)
    inputs = [torch.randn(H.shape, device="cuda", generator=g).bfloat16() for _ in range(3)]
    wants = [block.compute(x.clone(), F0).clone() for x in inputs]
    static = H.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        block.compute(static, F0)
    for turn in range(6):
        static.copy_(inputs[turn % 3])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(block.F, wants[turn % 3])
        assert torch.equal(block.compute(inputs[(turn + 1) % 3].clone(), F0), wants[(turn + 1) % 3])


def test_run():
    """Computed steps repeat themselves bit for bit, cached ones stay near the slowly turning stream: an angle of 0.05 a step moves it by 0.05 of its size a step, so by 0.15 after
    three; the forecast of the sub-block's part is no further off than that."""
    from cached_attention import run
    far = run(frames=1, height=16, width=16, text=64, text_used=20, heads=4, steps=8, say=lambda line: None)
    assert far[0] == 0.0 and far[4] == 0.0
    assert max(far) < 0.3
