"""The operators of a block in 8 bits against plain implementations in float64 that share no code with the library, and their refusals.

Tolerances, derived:
  8-bit values of given inputs are exact: bytes are compared.
  8-bit values y of sums: float32 sums leave a relative error of at most e = 1e-5 in y here, so a value may round the other way next to the middle of two
  neighbours, and a block's scale may be the neighbouring one if amax lies within e of a step.  Each value is at most half a step of e4m3 off: 2^-4 of itself, or
  2^-10 scales for subnormal ones, plus e.
  Products: sums of 128 columns at a time; each of the `blocks` additions rounds to float32 or, with the terms aligned to the largest first, to a few bits
  less: 2^-21 of S = sum |a w| a block, and the bias.  The activations' slopes are at most 1.13 (GELU) and 1.1 (silu), their own rounding 2^-18 of the
  result, as the exponential's argument is rounded to float32 first.  Results in bfloat16 are half a step (2^-8 of the value at most) off more.
  Products for results in bfloat16 and in 8 bits add 8 products at a time with 13 bits below the largest: each of 7 loses less than 2^-13 of the largest,
  7 * 2^-13 * sum of the largest <= 2^-10 S in all.  These losses have the signs of their products, so that far less is likely: with T^2 = sum (a w)^2 their
  standard deviation is at most 2^-13 sqrt(7 / 3) T, of which 7 are allowed.
"""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import paper_2601_07396_amd as svdc

E_REL = 1e-5
BLOCK = 128


# ---- oracle ---------------------------------------------------------------------------------------------------------

def _e4m3_table():
    """Values of the 128 bytes without sign, NaN last."""
    v = []
    for byte in range(127):
        e, m = byte >> 3, byte & 7
        v.append(m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10))
    return np.array(v)


TABLE = _e4m3_table()


def ref_e4m3(x):
    """Bytes of float64 values rounded to nearest, ties to even; what is not finite is NaN."""
    a = np.abs(np.where(np.isfinite(x), x, 0.0))
    hi = np.clip(np.searchsorted(TABLE, a), 1, 126)
    lo = hi - 1
    down, up = a - TABLE[lo], TABLE[hi] - a
    byte = np.where((down < up) | ((down == up) & (lo % 2 == 0)), lo, hi)
    return np.where(np.isfinite(x), byte | (np.signbit(x) << 7), 0x7F).astype(np.uint8)


def value_of(byte):
    a = np.append(TABLE, np.nan)[byte & 0x7F]
    return np.where(byte & 0x80, -a, a)


def ref_scale(amax):
    """Exponents of the scales."""
    a = np.minimum(amax, float(np.finfo(np.float32).max))
    e = np.zeros(a.shape, dtype=np.int64)
    for i in np.ndindex(a.shape):
        if a[i] > 0:
            e[i] = math.frexp(a[i])[1] - 9
            e[i] += a[i] > 448 * 2.0 ** float(e[i])
            e[i] = max(-126, min(126, e[i]))
    return e


def ref_amax(v, block_rows=1):
    rows, D = v.shape
    full = np.zeros((-(-rows // block_rows) * block_rows, -(-D // BLOCK) * BLOCK))
    full[:rows, :D] = np.where(np.isnan(v), 0.0, np.abs(v))
    return full.reshape(full.shape[0] // block_rows, block_rows, -1, BLOCK).max(axis=(1, 3))


def spread(s, rows, D, block_rows=1):
    return np.repeat(np.repeat(s, block_rows, 0)[:rows], BLOCK, 1)[:, :D]


def ref_quantize(v, block_rows=1):
    """(bytes [rows, D], scale exponents)."""
    e = ref_scale(ref_amax(v, block_rows))
    with np.errstate(over="ignore"):
        return ref_e4m3(v * 2.0 ** -spread(e, *v.shape, block_rows).astype(np.float64)), e


def ref_norm(x, f, gain, eps):
    h = x if f is None else x + f
    with np.errstate(all="ignore"):
        y = h / np.sqrt((h * h).mean(axis=1, keepdims=True) + eps)
        return h, y if gain is None else y * gain


def ref_act(z, act, N):
    with np.errstate(over="ignore", invalid="ignore"):
        if act == "gelu":
            return 0.5 * z * (1 + np.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
        if act == "swiglu":
            return z[:, :N] / (1 + np.exp(-z[:, :N])) * z[:, N:]
    return z


# ---- helpers --------------------------------------------------------------------------------------------------------

def bytes_of(t):
    return t.view(torch.uint8).cpu().numpy()


def check_padding(Q, scales, D):
    q, s = bytes_of(Q), bytes_of(scales)
    assert not q[:, D:].any()
    assert (s[:, -(-D // BLOCK):] == 127).all()


def check_near_q8(Q, scales, y, what):
    """Q and scales stand for y up to the rounding, with sums that are E_REL off."""
    rows, D = y.shape
    check_padding(Q, scales, D)
    nb = -(-D // BLOCK)
    e = bytes_of(scales)[:, :nb].astype(np.int64) - 127
    amax = ref_amax(y)
    low, high = ref_scale(amax * (1 - E_REL)), ref_scale(amax * (1 + E_REL))
    assert ((e >= low) & (e <= high)).all(), what
    got = value_of(bytes_of(Q)[:, :D]) * 2.0 ** spread(e, rows, D).astype(np.float64)
    finite = np.isfinite(y)
    assert np.isnan(got[~finite]).all() and np.isfinite(got[finite]).all(), what
    bound = 2.0 ** -4 * np.abs(y) * (1 + E_REL) + 2.0 ** -10 * 2.0 ** spread(e, rows, D) + E_REL * np.abs(y)
    assert (np.abs(got - y)[finite] <= bound[finite]).all(), what


def make_rows(rows, D, dtype, pad=0, offset=0, seed=0, planted=True):
    """A view [rows, D] of a wider buffer, starting `offset` elements in; a row of zeros, tiny and huge rows, and (planted) NaN and infinities."""
    g = np.random.default_rng(seed)
    v = g.standard_normal((rows, D)) * np.exp(g.standard_normal(D))
    if rows > 3:
        v[1] = 0
        v[2] *= 1e-6
        v[3] *= 1e4
    if planted and rows > 6:
        v[4, D // 2] = np.nan
        v[5, D - 1] = np.inf
        v[6, 0] = -np.inf
    ld = D + pad
    buf = torch.zeros(offset + rows * ld, dtype=dtype)
    view = buf[offset:].view(rows, ld)[:, :D]
    view.copy_(torch.from_numpy(v).to(dtype))
    dev = buf.cuda()
    return dev[offset:].view(rows, ld)[:, :D], view.double().numpy()


# ---- quantisation ---------------------------------------------------------------------------------------------------

@pytest.mark.gpu
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,D,pad,offset", [(1, 1, 0, 0), (1, 128, 0, 0), (7, 129, 0, 0), (130, 515, 5, 1), (257, 1024, 8, 0), (300, 4100, 0, 3), (64, 20000, 0, 0)])
def test_quantize8_is_exact(rows, D, pad, offset, dtype, block_rows):
    X, v = make_rows(rows, D, dtype, pad, offset, seed=rows + D)
    Q, scales = svdc.quantize8(X, block_rows)
    q, e = ref_quantize(v, block_rows)
    check_padding(Q, scales, D)
    assert np.array_equal(bytes_of(scales)[:, :e.shape[1]].astype(np.int64) - 127, e)
    got = bytes_of(Q)[:, :D]
    nan = ~np.isfinite(v)
    assert (got[nan] & 0x7F == 0x7F).all()
    assert np.array_equal(got[~nan], q[~nan])


@pytest.mark.gpu
def test_quantize8_at_the_ends_of_the_range():
    """Scales at amax = 448 * 2^e exactly, just above it, at the smallest and largest float32 and for a block of zeros; ties and subnormals of e4m3."""
    amax = [448.0, np.nextafter(np.float32(448), np.float32(1e3)), 447.9, 1.75, 3.4028235e38, 1e-45, 1.2e-38, 3e-36, 0.0, 224.0, 225.0]
    v = np.zeros((len(amax), BLOCK), dtype=np.float32)
    steps = np.append(TABLE, [(a + b) / 2 for a, b in zip(TABLE, TABLE[1:])])
    for i, m in enumerate(amax):
        e = float(ref_scale(np.array([float(np.float32(m))]))[0])
        v[i] = np.float32(np.minimum(np.random.default_rng(i).choice(steps, BLOCK) * 2.0 ** e, m)) if m else 0
        v[i, ::2] *= -1
        v[i, 77] = m
    X = torch.from_numpy(v).cuda()
    Q, scales = svdc.quantize8(X)
    q, e = ref_quantize(v.astype(np.float64))
    assert np.array_equal(bytes_of(scales)[:, :1].astype(np.int64) - 127, e)
    assert np.array_equal(bytes_of(Q), q)


# ---- norm -----------------------------------------------------------------------------------------------------------

@pytest.mark.gpu
@pytest.mark.parametrize("dtype,dtype_f", [(torch.bfloat16, torch.bfloat16), (torch.float32, torch.float32), (torch.float32, torch.bfloat16),
                                           (torch.bfloat16, torch.float32)])
@pytest.mark.parametrize("rows,D,pad,offset", [(1, 1, 0, 0), (1, 3072, 0, 0), (9, 100, 0, 1), (33, 512, 8, 0), (130, 1157, 3, 1), (20, 3076, 0, 0),
                                               (1500, 640, 0, 0), (7, 5000, 1, 0), (40, 9000, 0, 0), (300, 12288, 0, 0), (3, 20001, 0, 0), (2, 70000, 0, 0)])
def test_rms_norm8(rows, D, pad, offset, dtype, dtype_f):
    X, x = make_rows(rows, D, dtype, pad, offset, seed=1)
    F, f = make_rows(rows, D, dtype_f, 0, 0, seed=2, planted=False)
    gain = torch.randn(D, generator=torch.Generator().manual_seed(3)).cuda()
    H = torch.full((rows, D + 2), 7.0, device="cuda", dtype=dtype)[:, :D]
    Y = torch.full((rows, D), 7.0, device="cuda", dtype=dtype)
    Q, scales = svdc.alloc_q8(rows, D, "cuda")
    eps = 1e-5
    p = svdc.make_norm8(X, F, H, Y, eps)
    svdc.svdcache_rms_norm8(p, X, F, gain, H, Y, Q, scales)
    h, y = ref_norm(x, f, gain.double().cpu().numpy(), eps)
    # the sum is one float32 addition, then rounded to the stream's type
    with np.errstate(over="ignore"):
        want_h = torch.from_numpy((x.astype(np.float32) + f.astype(np.float32))).to(dtype)
    got_h = H.cpu()
    assert torch.equal(torch.nan_to_num(got_h, nan=123.0), torch.nan_to_num(want_h, nan=123.0))
    got = Y.double().cpu().numpy()
    step = 2.0 ** -8 if dtype == torch.bfloat16 else 0.0
    finite = np.isfinite(y)
    assert np.isnan(got[~finite]).all()
    assert (np.abs(got - y)[finite] <= (E_REL + step) * np.abs(y)[finite]).all()
    check_near_q8(Q, scales, y, (rows, D))
    assert not (H.stride(0) > D and (torch.as_strided(H, (rows, 2), (H.stride(0), 1), D) != 7).any())      # nothing beyond the rows


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,dtype_f", [(torch.bfloat16, torch.bfloat16), (torch.float32, torch.bfloat16)])
@pytest.mark.parametrize("rows,D", [(8195, 1000), (8195, 1101), (8193, 2040), (8194, 2501), (8195, 3001), (8195, 3100), (1030, 1025)])
def test_rms_norm8_many_rows(rows, D, dtype, dtype_f):
    """A row each for a wave or a workgroup of a full grid, and several rows for each of a small one."""
    test_rms_norm8(rows, D, 3, 1, dtype, dtype_f)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,D", [(5, 3072), (2000, 1000)])
def test_rms_norm8_outputs_on_their_own(rows, D):
    """Without F, gain, H; only Y; only Q; in place of X and of F: the same bits as with everything."""
    X, x = make_rows(rows, D, torch.bfloat16, seed=4)
    F, f = make_rows(rows, D, torch.bfloat16, seed=5, planted=False)
    gain = torch.rand(D, device="cuda") + 0.5
    H, Y = torch.empty_like(X), torch.empty_like(X)
    Q, scales = svdc.alloc_q8(rows, D, "cuda")
    svdc.svdcache_rms_norm8(svdc.make_norm8(X, F, H, Y), X, F, gain, H, Y, Q, scales)

    def same(a, b):
        return np.array_equal(bytes_of(a.contiguous()), bytes_of(b.contiguous()))

    H2, Q2, s2 = svdc.rms_norm8(X, F, gain)
    assert same(H, H2) and same(Q, Q2) and same(scales, s2)
    Y2 = torch.empty_like(X)
    svdc.svdcache_rms_norm8(svdc.make_norm8(X, F, None, Y2), X, F, gain, None, Y2, None, None)
    assert same(Y, Y2)
    for name in ("X", "F"):
        Xc, Fc = X.clone(), F.clone()
        into = Xc if name == "X" else Fc
        Q2.view(torch.uint8).zero_()
        svdc.svdcache_rms_norm8(svdc.make_norm8(Xc, Fc, into), Xc, Fc, gain, into, None, Q2, s2)
        assert same(into, H) and same(Q, Q2), name
    # no F, no gain: the norm of H as stored
    Y3, Q3 = torch.empty_like(X), Q2
    svdc.svdcache_rms_norm8(svdc.make_norm8(X, None, None, Y3), X, None, None, None, Y3, Q3, s2)
    _, y = ref_norm(x, None, None, 1e-6)
    finite = np.isfinite(y)
    assert (np.abs(Y3.double().cpu().numpy() - y)[finite] <= (E_REL + 2.0 ** -8) * np.abs(y)[finite]).all()
    check_near_q8(Q3, s2, y, "no gain")


# ---- product --------------------------------------------------------------------------------------------------------

def make_product(M, wide, K, seed=0, planted=False):
    """A and W in 8 bits made by the oracle (numpy), as tensors and as the values they stand for."""
    g = np.random.default_rng(seed)
    a = g.standard_normal((M, K)) * np.exp(g.standard_normal(K)) * np.exp(3 * g.standard_normal((M, 1)))
    w = g.standard_normal((wide, K)) / math.sqrt(K) * np.exp(g.standard_normal((wide, 1)))
    if M > 3:
        a[1] = 0
    if planted:
        a[M // 2, K // 3] = np.nan
    made = []
    for v, block_rows in ((a, 1), (w, BLOCK)):
        q, e = ref_quantize(v, block_rows)
        rows, D = v.shape
        Q = np.zeros((rows, -(-D // BLOCK) * BLOCK), dtype=np.uint8)
        Q[:, :D] = q
        s = np.full((e.shape[0], -(-e.shape[1] // 4) * 4), 127, dtype=np.uint8)
        s[:, :e.shape[1]] = e + 127
        made.append((torch.from_numpy(Q).cuda().view(torch.float8_e4m3fn), torch.from_numpy(s).cuda().view(torch.float8_e8m0fnu),
                     value_of(q) * 2.0 ** spread(e, rows, D, block_rows)))
    return made


def product_bound(a, w, bias, z, out, act, N, K, eight_bit_sums):
    """How far a result may be from the oracle's."""
    S = np.abs(np.nan_to_num(a)) @ np.abs(w).T + (0 if bias is None else np.abs(bias))
    off = (-(-K // BLOCK) + 2) * 2.0 ** -21 * S
    if eight_bit_sums:
        T = np.sqrt(np.square(np.nan_to_num(a)) @ np.square(w).T)
        off = off + np.minimum(2.0 ** -10 * S, 7 * 2.0 ** -13 * math.sqrt(7 / 3) * T)
    if act == "swiglu":
        gate, up = np.abs(ref_act(z[:, :N], "gelu", N)) + 0.3, np.abs(z[:, N:])
        off = 1.1 * off[:, :N] * up + gate * off[:, N:] + 1.1 * off[:, :N] * off[:, N:]
    elif act == "gelu":
        off = 1.13 * off
    return off + 2.0 ** -18 * np.abs(out)


def check_product(M, N, K, dtype, act, with_bias, seed=0, planted=False, ldo_pad=0):
    wide = 2 * N if act == "swiglu" else N
    (A, As, a), (W, Ws, w) = make_product(M, wide, K, seed, planted)
    bias = np.random.default_rng(seed + 1).standard_normal(wide).astype(np.float32) if with_bias else None
    tb = torch.from_numpy(bias).cuda() if with_bias else None
    z = a @ w.T + (0 if bias is None else bias.astype(np.float64))
    out = ref_act(z, act, N)
    bound = product_bound(a, w, bias, np.nan_to_num(z), out, act, N, K, dtype != torch.float32)
    p = svdc.make_matmul8(M, N, K, dtype, act, N + ldo_pad)
    ws = svdc.alloc_matmul8_workspace(p, "cuda")
    if ws is not None:
        ws.fill_(0xFF)                                   # what a workspace holds before the call does not matter
    finite = np.isfinite(out)
    what = (M, N, K, dtype, act)
    if dtype == torch.float8_e4m3fn:
        Q, scales = svdc.alloc_q8(M, N, "cuda")
        Q.view(torch.uint8).fill_(0x55)
        scales.view(torch.uint8).fill_(0x55)
        svdc.svdcache_matmul8(p, A, As, W, Ws, tb, Q, scales, ws)
        check_padding(Q, scales, N)
        e = bytes_of(scales)[:, :-(-N // BLOCK)].astype(np.int64) - 127
        slack = ref_amax(np.where(finite, bound, 0))
        amax = ref_amax(out)
        assert ((e >= ref_scale(np.maximum(amax - slack, 0))) & (e <= ref_scale(amax + slack)) | (slack >= amax)).all(), what
        got = value_of(bytes_of(Q)[:, :N]) * 2.0 ** spread(e, M, N).astype(np.float64)
        bound = bound + 2.0 ** -4 * (np.abs(out) + bound) + 2.0 ** -10 * 2.0 ** spread(e, M, N)
    else:
        buf = torch.full((M, N + ldo_pad), 7.0, device="cuda", dtype=dtype)
        svdc.svdcache_matmul8(p, A, As, W, Ws, tb, buf[:, :N], None, ws)
        got = buf[:, :N].double().cpu().numpy()
        assert (buf[:, N:] == 7).all(), what
        if dtype == torch.bfloat16:
            bound = bound + 2.0 ** -8 * (np.abs(out) + bound)
    assert np.isnan(got[~finite]).all(), what
    bad = np.abs(got - out)[finite] > bound[finite]
    assert not bad.any(), (what, int(bad.sum()), float(np.max(np.abs(got - out)[finite] / bound[finite])))


DTYPES_OUT = [torch.float32, torch.bfloat16, torch.float8_e4m3fn]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES_OUT)
@pytest.mark.parametrize("act", ["none", "gelu", "swiglu"])
@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (1, 300, 128), (3, 128, 1000), (16, 257, 512), (17, 64, 640), (40, 384, 1157), (130, 200, 130), (300, 520, 260)])
def test_matmul8(M, N, K, act, dtype):
    check_product(M, N, K, dtype, act, with_bias=(M + N) % 2 == 0, seed=M + N + K, ldo_pad=3 if M % 2 else 0)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES_OUT)
@pytest.mark.parametrize("M,N,K,act", [(1, 2000, 3000, "none"), (64, 1024, 4096, "gelu"), (256, 512, 2048, "none"), (200, 300, 8192, "swiglu"), (513, 1030, 700, "gelu"),
                                       (1025, 640, 384, "none"), (31, 100, 16384, "none"), (2100, 768, 256, "swiglu"), (777, 1921, 1157, "swiglu")])
def test_matmul8_larger(M, N, K, act, dtype):
    check_product(M, N, K, dtype, act, with_bias=True, seed=M)


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", [(5, 140, 300), (300, 300, 1000), (200, 256, 6000)])
@pytest.mark.parametrize("dtype", DTYPES_OUT)
def test_matmul8_nan_stays_in_its_row(M, N, K, dtype):
    check_product(M, N, K, dtype, "gelu", True, seed=2, planted=True)


@pytest.mark.gpu
def test_matmul8_at_the_ends_of_the_scales():
    """Scales near both ends cancel: 2^100 in A against 2^-100 in W."""
    for M in (2, 200):
        (A, As, a), (W, Ws, w) = make_product(M, 130, 300, 5)
        a64, w64 = a, w
        As = (As.view(torch.uint8).to(torch.int32) + torch.where(As.view(torch.uint8) == 127, 0, 100)).to(torch.uint8).view(torch.float8_e8m0fnu)
        Ws = (Ws.view(torch.uint8).to(torch.int32) - torch.where(Ws.view(torch.uint8) == 127, 0, 100)).to(torch.uint8).view(torch.float8_e8m0fnu)
        blocks = 3
        sa = 2.0 ** (As.view(torch.uint8).cpu().numpy()[:, :blocks].astype(np.float64) - 127)
        sw = 2.0 ** (Ws.view(torch.uint8).cpu().numpy()[:, :blocks].astype(np.float64) - 127)
        a64 = value_of(bytes_of(A)[:, :300]) * spread(sa, M, 300)
        w64 = value_of(bytes_of(W)[:, :300]) * spread(sw, 130, 300, BLOCK)
        out = svdc.matmul8(A, As, W, Ws, 300, dtype=torch.float32).double().cpu().numpy()
        S = np.abs(a64) @ np.abs(w64).T
        assert (np.abs(out - a64 @ w64.T) <= 5 * 2.0 ** -21 * S).all()


@pytest.mark.gpu
def test_same_bits_on_every_call_and_on_another_stream():
    (A, As, _), (W, Ws, _) = make_product(200, 700, 5000, 7)
    X, _ = make_rows(333, 2001, torch.bfloat16, seed=8)
    F, _ = make_rows(333, 2001, torch.bfloat16, seed=9)

    def everything():
        return [svdc.matmul8(A, As, W, Ws, 5000, dtype=torch.float32), *svdc.matmul8(A, As, W, Ws, 5000, dtype=torch.float8_e4m3fn, act="gelu"),
                *svdc.rms_norm8(X, F), *svdc.quantize8(X), *svdc.quantize8(X, 128)]

    first = everything()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        with torch.cuda.stream(side):
            again = everything()
        side.synchronize()
        for a, b in zip(first, again):
            assert np.array_equal(bytes_of(a), bytes_of(b))


@pytest.mark.gpu
def test_graph_replay():
    """Captured once, replayed on new inputs, with eager work in between."""
    M, N, K = 150, 520, 4000
    (A, As, _), (W, Ws, _) = make_product(M, N, K, 3)
    X, F = torch.randn(M, K, device="cuda"), torch.randn(M, K, device="cuda").bfloat16()
    Q, s = svdc.alloc_q8(M, K, "cuda")
    H, out = torch.empty_like(X), torch.empty(M, N, device="cuda")
    pn, pm = svdc.make_norm8(X, F, H), svdc.make_matmul8(M, N, K, torch.float32)
    ws = svdc.alloc_matmul8_workspace(pm, "cuda")

    def step():
        svdc.svdcache_rms_norm8(pn, X, F, None, H, None, Q, s)
        svdc.svdcache_matmul8(pm, Q, s, W, Ws, None, out, None, ws)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        X.normal_(generator=torch.Generator("cuda").manual_seed(i))
        step()
        want = out.clone()
        out.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


@pytest.mark.gpu
def test_no_rows():
    X = torch.empty(0, 300, device="cuda", dtype=torch.bfloat16)
    H, Q, s = svdc.rms_norm8(X, X)
    assert H.shape == (0, 300) and Q.shape == (0, 384) and s.shape == (0, 4)
    Q, s = svdc.quantize8(X)
    (_, _, _), (W, Ws, _) = make_product(1, 20, 300)
    assert svdc.matmul8(Q, s, W, Ws, 300).shape == (0, 20)


@pytest.mark.gpu
def test_offsets_beyond_32_bits():
    """Rows whose elements and bytes lie beyond 2^32: the last ones against the same rows in a small tensor."""
    rows, D = 1_100_000, 4096                                         # 4.5e9 elements
    X = torch.zeros(rows, D, device="cuda", dtype=torch.bfloat16)
    tail = torch.randn(300, D, device="cuda").bfloat16()
    X[-300:] = tail
    Q, s = svdc.quantize8(X)
    q, t = svdc.quantize8(tail)
    assert torch.equal(Q.view(torch.uint8)[-300:], q.view(torch.uint8)) and torch.equal(s.view(torch.uint8)[-300:], t.view(torch.uint8))
    del X
    W, Ws = svdc.quantize8(torch.randn(64, D, device="cuda"), 128)
    out = svdc.matmul8(Q, s, W, Ws, D, dtype=torch.float32)
    assert torch.allclose(out[-300:], svdc.matmul8(q, t, W, Ws, D, dtype=torch.float32), rtol=1e-4, atol=1e-3) and not out[:1000].any()


# ---- refusals (no GPU) ----------------------------------------------------------------------------------------------

def fake(n=4096):
    return C.c_void_p(n)


def norm8(**kw):
    return svdc.Norm8(**{**dict(rows=4, D=256, dtype=0, dtype_f=0, eps=1e-6, ldx=256, ldf=256, ldh=256, ldy=256), **kw})


@pytest.mark.parametrize("kw,code", [(dict(dtype=2), -3), (dict(dtype_f=7), -3), (dict(eps=-1.0), -5), (dict(eps=float("nan")), -5), (dict(eps=float("inf")), -5),
                                     (dict(rows=-1), -2), (dict(rows=1 << 31), -2), (dict(D=0), -2), (dict(D=(1 << 20) + 1, ldx=1 << 21), -2), (dict(ldx=255), -2),
                                     (dict(ldf=0), -2), (dict(ldh=255), -2), (dict(ldy=-256), -2), (dict(ldx=1 << 47), -2)])
def test_norm_refusals(kw, code):
    lib = svdc.load_library()
    p = norm8(**kw)
    a = [fake(i << 12) for i in range(1, 9)]
    assert lib.svdcache_rms_norm8(C.byref(p), *a[:7], None) == code


def test_norm_refuses_pointers():
    lib = svdc.load_library()
    x, f, g, h, y, q, s = (fake(i << 12) for i in range(1, 8))

    def call(*a, **kw):
        return lib.svdcache_rms_norm8(C.byref(norm8(**kw)), *a, None)

    assert lib.svdcache_rms_norm8(None, x, f, g, h, y, q, s, None) == -1
    assert call(None, f, g, h, y, q, s) == -1
    assert call(x, f, g, h, None, None, None) == -1                      # nothing to compute
    assert call(x, f, g, h, y, q, None) == -1 and call(x, f, g, h, y, None, s) == -1
    assert call(fake(4098), f, g, h, y, q, s) == -4 and call(x, fake(4097), g, h, y, q, s, dtype_f=1) == -4
    assert call(x, f, fake(4098), h, y, q, s) == -4 and call(x, f, g, h, y, fake(4104), s) == -4 and call(x, f, g, h, y, q, fake(4098)) == -4
    assert call(x, f, g, x, y, q, s, ldh=512) == -5                       # in place with another stride
    assert call(x, f, g, f, y, q, s, dtype_f=1) == -5                     # in place of a tensor of another type
    assert call(x, f, g, h, x, q, s) == -5 and call(x, f, g, h, h, q, s) == -5
    assert call(None, None, None, None, None, None, None, rows=0) == 0   # no rows: nothing is needed


def test_quantize_refusals():
    lib = svdc.load_library()

    def call(x=fake(), q=fake(8192), s=fake(12288), **kw):
        p = svdc.Quant8(**{**dict(rows=4, D=256, dtype=0, ldx=256, block_rows=1, reserved=0), **kw})
        return lib.svdcache_quantize8(C.byref(p), x, q, s, None)

    assert lib.svdcache_quantize8(None, fake(), fake(), fake(), None) == -1
    for kw, code in [(dict(dtype=2), -3), (dict(block_rows=2), -5), (dict(block_rows=0), -5), (dict(reserved=1), -5), (dict(rows=-1), -2), (dict(D=0), -2), (dict(ldx=0), -2),
                     (dict(x=None), -1), (dict(q=None), -1), (dict(s=None), -1), (dict(x=fake(4098)), -4), (dict(q=fake(4104)), -4), (dict(s=fake(4098)), -4)]:
        assert call(**kw) == code, kw
    assert call(x=None, q=None, s=None, rows=0) == 0


def test_matmul_refusals():
    lib = svdc.load_library()

    def call(a=fake(1 << 12), sa=fake(2 << 12), w=fake(3 << 12), sw=fake(4 << 12), b=None, o=fake(5 << 12), so=fake(6 << 12), ws=None, n=0, **kw):
        p = svdc.Matmul8(**{**dict(M=4, N=256, K=256, dtype=0, act=0, ldo=256), **kw})
        return lib.svdcache_matmul8(C.byref(p), a, sa, w, sw, b, o, so, ws, n, None)

    assert lib.svdcache_matmul8(None, *[fake()] * 8, 0, None) == -1
    for kw, code in [(dict(dtype=3), -3), (dict(act=3), -5), (dict(act=-1), -5), (dict(M=-1), -2), (dict(M=1 << 31), -2), (dict(N=0), -2), (dict(N=(1 << 24) + 1, ldo=1 << 25), -2),
                     (dict(N=(1 << 20) + 1, dtype=2), -2), (dict(K=0), -2), (dict(K=(1 << 20) + 1), -2), (dict(ldo=255), -2), (dict(ldo=1 << 47), -2), (dict(a=None), -1),
                     (dict(sa=None), -1), (dict(w=None), -1), (dict(sw=None), -1), (dict(o=None), -1), (dict(so=None, dtype=2), -1), (dict(a=fake(4104)), -4),
                     (dict(sa=fake(4098)), -4), (dict(w=fake(4100)), -4), (dict(sw=fake(4097)), -4), (dict(b=fake(4098)), -4), (dict(o=fake(4098)), -4),
                     (dict(o=fake(4104), dtype=2), -4), (dict(so=fake(4098), dtype=2), -4)]:
        assert call(**kw) == code, kw
    assert call(a=None, M=0) == 0


def test_workspace_refusals():
    """A product that keeps partial sums needs the workspace it asks for."""
    lib = svdc.load_library()
    for M, N, K in [(256, 256, 16384), (64, 512, 1 << 18), (4608, 3072, 12288), (1, 1, 1)]:
        p = svdc.make_matmul8(M, N, K)
        need = svdc.svdcache_matmul8_workspace_bytes(p)
        a = [fake(i << 12) for i in range(1, 8)]
        if need:
            assert lib.svdcache_matmul8(C.byref(p), *a[:4], None, *a[4:6], None, need, None) == -1
            assert lib.svdcache_matmul8(C.byref(p), *a[:4], None, *a[4:6], fake(4100), need, None) == -4
            assert lib.svdcache_matmul8(C.byref(p), *a[:4], None, *a[4:6], fake(4096), need - 1, None) == -6
    assert svdc.svdcache_matmul8_workspace_bytes(svdc.Matmul8(4, 0, 4, 0, 0, 4)) == 0


def test_sizes_of_the_8_bit_form():
    assert svdc.svdcache_q8_bytes(3, 129) == 3 * 256 and svdc.svdcache_q8_scale_bytes(3, 129) == 3 * 4
    assert svdc.svdcache_q8_scale_bytes(129, 1025, 128) == 2 * 12 and svdc.svdcache_q8_bytes(0, 5) == 0
    for bad in [(-1, 5), (1 << 31, 5), (1, 0), (1, (1 << 20) + 1)]:
        assert svdc.svdcache_q8_bytes(*bad) == 0 and svdc.svdcache_q8_scale_bytes(*bad) == 0
    assert svdc.svdcache_q8_scale_bytes(4, 128, 64) == 0
    with pytest.raises(svdc.SvdcError):
        svdc.alloc_q8(3, 0, "cpu")


def test_binding_refuses_layouts():
    """Tensors that are not what the descriptor says, before any pointer is taken."""
    X = torch.zeros(4, 256)
    with pytest.raises(ValueError, match="contiguous last"):
        svdc.make_norm8(X.t())
    with pytest.raises(ValueError, match="one stride"):
        svdc.make_quant8(torch.zeros(3, 4, 256)[:, :2])
    with pytest.raises(ValueError, match="float32 or bfloat16"):
        svdc.make_quant8(X.half())
    with pytest.raises(ValueError, match="rows of"):
        svdc.make_norm8(X, torch.zeros(4, 128))
    with pytest.raises(ValueError):
        svdc.make_matmul8(4, 4, 4, torch.float16)
    p = svdc.make_norm8(X, X)
    Q, s = svdc.alloc_q8(4, 256, "cpu")
    with pytest.raises(ValueError, match="dtype"):
        svdc.svdcache_rms_norm8(p, X, X.bfloat16(), None, None, None, Q, s)
    with pytest.raises(ValueError, match="row stride"):
        svdc.svdcache_rms_norm8(p, torch.zeros(4, 300)[:, :256], X, None, None, None, Q, s)
    with pytest.raises(ValueError, match="gain"):
        svdc.svdcache_rms_norm8(p, X, X, torch.zeros(255), None, None, Q, s)
    with pytest.raises(ValueError, match="bytes"):
        svdc.svdcache_rms_norm8(p, X, X, None, None, None, Q[:2], s)
    with pytest.raises(ValueError, match="go together"):
        svdc.svdcache_rms_norm8(p, X, X, None, None, X, Q, None)
    with pytest.raises(RuntimeError, match="GPU"):
        svdc.svdcache_rms_norm8(p, X, X, None, None, None, Q, s)
    with pytest.raises(RuntimeError, match="GPU"):
        svdc.svdcache_quantize8(svdc.make_quant8(X), X, Q, s)
    m = svdc.make_matmul8(4, 128, 256, torch.float8_e4m3fn)
    W, Ws = svdc.alloc_q8(128, 256, "cpu", 128)
    O, Os = svdc.alloc_q8(4, 128, "cpu")
    with pytest.raises(ValueError, match="Out_scales"):
        svdc.svdcache_matmul8(m, Q, s, W, Ws, None, O)
    with pytest.raises(ValueError, match="W"):
        svdc.svdcache_matmul8(svdc.make_matmul8(4, 128, 256, act="swiglu"), Q, s, W, Ws, None, torch.zeros(4, 128).bfloat16())
    with pytest.raises(RuntimeError, match="GPU"):
        svdc.svdcache_matmul8(m, Q, s, W, Ws, None, O, Os)


# Sizes that between them take every way in which a product is made on a whole card, with odd ends: groups of 16 and 32 rows by 16, 32, 64 (and 128) columns, tiles of 64, 128
# and 256, long axes in 2, 4, 8 and 16 parts.
WAYS = {
    torch.float32: {
        "none": [(1178, 1668, 130), (90, 3, 15866), (132, 5571, 7117), (4108, 3, 17709), (91, 5, 15003), (12, 3, 300), (203, 306, 260), (166, 1356, 666), (674, 166, 257),
                 (388, 323, 392), (4311, 33, 846), (291, 209, 300)],
        "swiglu": [(1897, 1754, 130), (95, 3, 8043), (138, 2077, 9579), (124, 3, 17596), (95, 3, 7665), (12, 3, 129), (166, 691, 535), (371, 163, 385), (457, 278, 644), (45, 3, 300)]},
    torch.bfloat16: {
        "none": [(1411, 1409, 131), (102, 3, 16148), (130, 4212, 8011), (4127, 3, 13753), (99, 3, 14365), (12, 3, 257), (215, 295, 131), (301, 815, 391), (3014, 4137, 514), (579, 204, 137),
                 (324, 395, 257), (2092, 97, 670), (211, 290, 300)],
        "swiglu": [(2306, 2196, 100), (92, 4, 8038), (4198, 65, 6144), (93, 3, 13982), (90, 3, 7383), (163, 682, 435), (3499, 1732, 536), (407, 146, 267), (211, 585, 536), (45, 3, 300)]},
    torch.float8_e4m3fn: {
        "gelu": [(2877, 3587, 130), (101, 3, 7768), (132, 4126, 6029), (90, 3, 3215), (90, 3, 3743), (12, 3, 907), (2773, 4388, 535), (45, 3, 300)],
        "swiglu": [(3736, 2719, 100), (91, 3, 7789), (92, 3, 3040), (90, 3, 3359), (90, 3, 3889), (5846, 641, 2898), (45, 3, 300)]}}


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,act,M,N,K", [(d, a, *s) for d, by in WAYS.items() for a, sizes in by.items() for s in sizes])
def test_matmul8_every_way(dtype, act, M, N, K):
    check_product(M, N, K, dtype, act, with_bias=N % 2 == 1, seed=N, planted=M % 2 == 0, ldo_pad=5 if M % 3 == 0 else 0)


# Few tiles and more than 8 blocks of columns: four blocks in flight instead of two.  9 to 13 blocks, so that every remainder of four ends the sums; tiles of 64, of 128, and
# of 128 in parts.
@pytest.mark.gpu
@pytest.mark.parametrize("dtype,act", [(torch.bfloat16, "none"), (torch.bfloat16, "gelu"), (torch.bfloat16, "swiglu"), (torch.float8_e4m3fn, "none"),
                                       (torch.float8_e4m3fn, "gelu"), (torch.float8_e4m3fn, "swiglu")])
@pytest.mark.parametrize("M,N,K", [(200, 1500, 1100), (130, 1031, 1157), (250, 1300, 1300), (190, 1411, 1537), (200, 1500, 1600), (1000, 3000, 1100), (1000, 1501, 1250),
                                   (900, 2900, 1408), (1001, 3001, 1500), (255, 1100, 12000), (100, 8000, 6100)])
def test_matmul8_few_tiles_of_long_sums(M, N, K, dtype, act):
    check_product(M, N, K, dtype, act, with_bias=N % 2 == 1, seed=K, planted=M % 2 == 0, ldo_pad=3 if M % 3 == 0 else 0)
