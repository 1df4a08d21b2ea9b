"""How much of a product in 8 bits may be lost where its terms cancel: the documented bound for results in bfloat16 and in 8 bits, and float32 sums for results in float32.

The 8-bit matrix instructions add the products of 8 consecutive columns with 13 bits below the largest exponent among them.  Each of the 7 others loses less than 2^-13 of 2^(that
exponent), 7 * 2^-13 < 2^-10 in all.  The exponent is the sum of the operands' own, and a subnormal e4m3 value counts as 2^-6 there; so what is cut off is less than
2^-10 of sum max(|a|, 2^-6 of its scale) max(|w|, 2^-6 of its scale).  The rest is in float32: (blocks + 2) * 2^-21 of sum |a w| as derived in test_block8.py, and a value's rounding to its type.
"""
import numpy as np
import pytest
import torch

import paper_2601_07396_amd as svdc
from test_block8 import BLOCK, TABLE, bytes_of, spread, value_of

pytestmark = pytest.mark.gpu

F32, BF16, E4M3 = torch.float32, torch.bfloat16, torch.float8_e4m3fn
# few rows and tiles of 64, 128 and 256
SIZES = [(1, 130), (200, 700), (2000, 1000), (3000, 4400)]


def byte_of(v):
    b = int(np.argmin(np.abs(TABLE - abs(v))))
    assert TABLE[b] == abs(v)
    return b | (128 if v < 0 else 0)


def product(qa, qw, dtype):
    """The library's product of bytes with scales of 1, as float64 values, and the scales of an 8-bit result."""
    def matrix(q, block_rows):
        rows, K = q.shape
        Q = np.zeros((rows, -(-K // BLOCK) * BLOCK), dtype=np.uint8)
        Q[:, :K] = q
        s = torch.full((-(-rows // block_rows), (Q.shape[1] // BLOCK + 3) // 4 * 4), 127, dtype=torch.uint8)
        return torch.from_numpy(Q).cuda().view(E4M3), s.cuda().view(torch.float8_e8m0fnu)

    got = svdc.matmul8(*matrix(qa, 1), *matrix(qw, BLOCK), qa.shape[1], None, dtype)
    if dtype != E4M3:
        return got.double().cpu().numpy(), None
    M, N = qa.shape[0], qw.shape[0]
    scale = 2.0 ** spread(bytes_of(got[1])[:, :-(-N // BLOCK)].astype(np.float64) - 127, M, N)
    return value_of(bytes_of(got[0])[:, :N]) * scale, scale


@pytest.mark.parametrize("M,N", SIZES)
@pytest.mark.parametrize("dtype", [F32, BF16, E4M3])
def test_one_beside_cancelling_products(M, N, dtype):
    """448 * 448 - 448 * 448 + 1 * 1 in eight consecutive columns is 1 in float32, and off by no more than the bound elsewhere; with the 1 among other columns it is 1 everywhere."""
    K = 128
    for column in (2, 9):
        a, w = np.zeros((M, K), dtype=np.uint8), np.zeros((N, K), dtype=np.uint8)
        a[:, 0] = a[:, 1] = w[:, 0] = byte_of(448.0)
        w[:, 1] = byte_of(-448.0)
        a[:, column] = w[:, column] = byte_of(1.0)
        got, _ = product(a, w, dtype)
        assert got.shape == (M, N)
        if dtype == F32 or column == 9:
            assert (got == 1).all()
        else:
            assert (np.abs(got - 1) <= 2.0 ** -10 * (2 * 448.0 ** 2 + 1)).all()


def bound(qa, qw, z, dtype, scale):
    a, w = np.abs(value_of(qa)), np.abs(value_of(qw))
    off = (-(-a.shape[1] // BLOCK) + 2) * 2.0 ** -21 * (a @ w.T)
    if dtype == F32:
        return off
    off += 2.0 ** -10 * (np.maximum(a, 2.0 ** -6) @ np.maximum(w, 2.0 ** -6).T)
    return off + (2.0 ** -8 * (np.abs(z) + off) if dtype == BF16 else 2.0 ** -4 * (np.abs(z) + off) + 2.0 ** -10 * scale)


@pytest.mark.parametrize("M,N", SIZES)
@pytest.mark.parametrize("dtype", [F32, BF16, E4M3])
@pytest.mark.parametrize("kind", ["pairs", "subnormal"])
def test_the_bound_holds(M, N, dtype, kind):
    """Groups of eight columns whose large products cancel in pairs and leave small ones; and rows of subnormal values alone."""
    g = np.random.default_rng(M)
    K = 640
    signs = lambda *s: (g.integers(0, 2, s) << 7).astype(np.uint8)      # noqa: E731
    qa = (g.integers(1, 127, (M, K)).astype(np.uint8) | signs(M, K))
    qw = (g.integers(1, 127, (N, K)).astype(np.uint8) | signs(N, K))
    if kind == "pairs":
        qa[:, 1::2], qw[:, 1::2] = qa[:, 0::2], qw[:, 0::2] ^ 128
        qa[:, 7::8] = byte_of(1.0)                                      # of each group one pair does not cancel
    else:
        qa = (g.integers(1, 8, (M, K)).astype(np.uint8) | signs(M, K))
    z = value_of(qa) @ value_of(qw).T
    got, scale = product(qa, qw, dtype)
    assert (np.abs(got - z) <= bound(qa, qw, z, dtype, scale)).all()
