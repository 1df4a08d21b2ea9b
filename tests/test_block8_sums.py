"""Sums of the product in 8 bits where scales reach the ends of their range, against float64.

Tolerances are those derived in test_block8.py (product_bound there): 2^-21 of sum |a w| for each block of 128 columns and the bias, that of the 8-bit matrix instructions for results
in bfloat16 and in 8 bits, and the rounding to the result's type.  Nothing in their derivation depends on the size of a scale: products of a power of two and a
float32 are exact where the result is a normal float32, as all results here are.
"""
import numpy as np
import pytest
import torch

import paper_2601_07396_amd as svdc
from test_block8 import BLOCK, bytes_of, check_padding, product_bound, ref_act, ref_amax, ref_scale, spread, value_of

F32, BF16, E4M3 = torch.float32, torch.bfloat16, torch.float8_e4m3fn


def as_tensors(q, e):
    """Bytes [rows, K] and exponents of scales [rows or blocks of rows, blocks of columns] as a matrix in 8 bits."""
    rows, K = q.shape
    Q = np.zeros((rows, -(-K // BLOCK) * BLOCK), dtype=np.uint8)
    Q[:, :K] = q
    s = np.full((e.shape[0], -(-e.shape[1] // 4) * 4), 127, dtype=np.uint8)
    s[:, :e.shape[1]] = e + 127
    return torch.from_numpy(Q).cuda().view(E4M3), torch.from_numpy(s).cuda().view(torch.float8_e8m0fnu)


def multiply(qa, ea, qw, ew, bias, dtype, act):
    """The library's product as float64 values, and the exponents of its scales where it is in 8 bits."""
    (M, K), N = qa.shape, qw.shape[0] // (2 if act == "swiglu" else 1)
    tb = None if bias is None else torch.from_numpy(bias).cuda()
    got = svdc.matmul8(*as_tensors(qa, ea), *as_tensors(qw, ew), K, tb, dtype, act)
    if dtype != E4M3:
        assert got.shape == (M, N)
        return got.double().cpu().numpy(), None
    check_padding(*got, N)
    e = bytes_of(got[1])[:, :-(-N // BLOCK)].astype(np.int64) - 127
    return value_of(bytes_of(got[0])[:, :N]) * 2.0 ** spread(e, M, N).astype(np.float64), e


def check(qa, ea, qw, ew, bias, dtype, act):
    (M, K), N = qa.shape, qw.shape[0] // (2 if act == "swiglu" else 1)
    a = value_of(qa) * 2.0 ** spread(ea, M, K).astype(np.float64)
    w = value_of(qw) * 2.0 ** spread(ew, qw.shape[0], K, BLOCK).astype(np.float64)
    z = a @ w.T + (0 if bias is None else bias.astype(np.float64))
    out = ref_act(z, act, N)
    assert np.isfinite(out).all() and np.abs(out).max() < 1e30
    bound = product_bound(a, w, bias, z, out, act, N, K, dtype != F32)
    got, e = multiply(qa, ea, qw, ew, bias, dtype, act)
    if dtype == E4M3:
        slack, amax = ref_amax(bound), ref_amax(out)
        assert ((e >= ref_scale(np.maximum(amax - slack, 0))) & (e <= ref_scale(amax + slack)) | (slack >= amax)).all()
        bound = bound + 2.0 ** -4 * (np.abs(out) + bound) + 2.0 ** -10 * 2.0 ** spread(e, M, N)
    elif dtype == BF16:
        bound = bound + 2.0 ** -8 * (np.abs(out) + bound)
    off = np.abs(got - out)
    assert (off <= bound).all(), (int((~(off <= bound)).sum()), got.size)


def random_bytes(g, rows, K):
    return (g.integers(0, 127, (rows, K)) | g.integers(0, 2, (rows, K)) << 7).astype(np.uint8)


# Few rows in every width, tiles of 64 and 128, parts of a long axis; gates whose rows begin inside a block of 128 rows of W, inside a tile and inside four rows
SIZES = [(3, 105, 266, "none"), (3, 103, 264, "swiglu"), (161, 1372, 654, "none"), (225, 278, 260, "gelu"), (98, 1064, 516, "swiglu"), (17, 2066, 267, "none"),
         (456, 133, 385, "swiglu"), (552, 231, 661, "swiglu"), (402, 622, 778, "none"), (198, 609, 267, "none"), (344, 178, 263, "swiglu"), (525, 3654, 263, "none"),
         (2058, 459, 270, "swiglu"), (152, 405, 7681, "none"), (2, 102, 7917, "swiglu"), (1100, 1801, 260, "gelu")]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16, E4M3])
@pytest.mark.parametrize("M,N,K,act", SIZES)
def test_scales_at_both_ends_cancel(M, N, K, act, dtype):
    """Each block of columns of A lies near 2^126, 2^-126 or in between, and that of W as far on the other side: values that the operands' product in float32 holds although bfloat16
    (and, at the upper end, float32) does not hold the operands."""
    g = np.random.default_rng(M + N + K)
    wide, blocks = 2 * N if act == "swiglu" else N, -(-K // BLOCK)
    shift = np.resize([126, -126, 119, -118, 0, -124, 121, 60], blocks)
    if M % 2:
        shift = -shift
    ea = np.clip(shift + g.integers(-3, 4, (M, blocks)), -126, 126)
    ew = np.clip(-shift + g.integers(-3, 4, (-(-wide // BLOCK), blocks)), -126, 126)
    bias = g.standard_normal(wide).astype(np.float32) if N % 2 else None
    check(random_bytes(g, M, K), ea, random_bytes(g, wide, K), ew, bias, dtype, act)


@pytest.mark.gpu
@pytest.mark.parametrize("M", [3, 70, 700])
@pytest.mark.parametrize("size,back", [(3.4e38, -100.0), (1e-38, 100.0), (1e-40, 120.0)])
def test_values_at_the_ends_of_float32(M, size, back):
    """Rows near the largest and the smallest float32 values, quantised by the library, against weights that bring the product back: float32 results as of the same 8-bit values
    in float64."""
    g = np.random.default_rng(M)
    K, N = 300, 260
    x = np.clip(g.uniform(0.1, 1.0, (M, K)), None, 1.0) * size * g.choice([-1, 1], (M, K))
    X = torch.from_numpy(x.astype(np.float32)).cuda()
    Wf = torch.from_numpy((g.standard_normal((N, K)) * 2.0 ** back).astype(np.float32)).cuda()
    (A, As), (W, Ws) = svdc.quantize8(X), svdc.quantize8(Wf, BLOCK)
    a = value_of(bytes_of(A)[:, :K]) * 2.0 ** spread(bytes_of(As)[:, :3].astype(np.float64) - 127, M, K)
    w = value_of(bytes_of(W)[:, :K]) * 2.0 ** spread(bytes_of(Ws)[:, :3].astype(np.float64) - 127, N, K, BLOCK)
    assert np.abs(a).max() > 0
    out = a @ w.T
    got = svdc.matmul8(A, As, W, Ws, K, dtype=F32).double().cpu().numpy()
    assert (np.abs(got - out) <= product_bound(a, w, None, out, out, "none", N, K, False) + 2.0 ** -140).all()
