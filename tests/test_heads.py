"""Angles of a rotation with several position axes, and norm and rotation of heads, against plain implementations in float64; their refusals.

Tolerances, derived:
  angles  are made in float64: each of the frequency, its product with the position and the division by 2 pi is off by at most 2 steps of float64, so an angle x by
          2^-50 |x|; what is left of it by 2^-28 of a turn (2 pi 2^-28 < 2^-25), its cosine and sine by a step of float32 more (2^-23): 2^-22 + 2^-50 |x|.
  heads   the sum of d squares, its mean, square root and division are off by less than (d + 8) 2^-24 of the result, half of it under the root; each product of y by 2^-24:
          a column y = a c - b s of (d + 16) 2^-24 (|a c| + |b s|), and half a step of the result's type (2^-24 or 2^-8).
"""
import ctypes as C
import math
from decimal import Decimal, localcontext

import numpy as np
import pytest
import torch

import paper_2601_07396_amd as svdc

F32, BF16 = torch.float32, torch.bfloat16
gpu = pytest.mark.gpu


# ---- angles ---------------------------------------------------------------------------------------------------------

def ref_angles(pos, dims, theta):
    """Angles [rows, pairs] in float64."""
    pos = pos.cpu().numpy().astype(np.float64)
    return np.concatenate([pos[:, a:a + 1] * np.array([theta[a] ** (-2.0 * i / n) for i in range(n // 2)]) for a, n in enumerate(dims)], axis=1)


def check_table(table, pos, dims, theta):
    x = ref_angles(pos, dims, theta)
    got = table.cpu().double().numpy()
    tol = 2.0 ** -22 + 2.0 ** -50 * np.abs(x)
    assert (np.abs(got[..., 0] - np.cos(x)) <= tol).all() and (np.abs(got[..., 1] - np.sin(x)) <= tol).all()


@gpu
@pytest.mark.parametrize("whole", [False, True])
@pytest.mark.parametrize("rows", [1, 2, 257, 4608])
@pytest.mark.parametrize("dims", [(16, 56, 56), (128,), (2,), (44, 42, 42), (2, 4, 6, 8), (64, 64, 64, 64), (30, 34)])
def test_angles(dims, rows, whole):
    g = torch.Generator().manual_seed(1)
    pos = torch.randint(-300, 5000, (rows, len(dims)), generator=g)
    pos = pos.to(torch.int32) if whole else pos.float() / 3
    theta = [10000.0, 256.0, 10000.0, 1.5][:len(dims)]
    pos = pos.cuda()
    table = svdc.rotary_table(pos, dims, theta)
    assert table.shape == (rows, sum(dims) // 2, 2)
    check_table(table, pos, dims, theta)


@gpu
def test_far_positions_strides_and_no_rows():
    whole = torch.tensor([[2 ** 31 - 1, 1], [-2 ** 31, 2 ** 30], [2 ** 24 + 1, 0]], dtype=torch.int32, device="cuda")
    check_table(svdc.rotary_table(whole, (8, 6)), whole, (8, 6), (10000.0, 10000.0))
    wide = torch.randn(50, 7, device="cuda")
    check_table(svdc.rotary_table(wide[:, 2:5], (8, 6, 4)), wide[:, 2:5], (8, 6, 4), (10000.0,) * 3)
    bad = torch.tensor([[math.inf], [math.nan], [1.0]], device="cuda")
    t = svdc.rotary_table(bad, (4,))
    assert t[:2].isnan().all() and torch.isfinite(t[2]).all()
    assert svdc.rotary_table(torch.empty(0, 2, device="cuda"), (2, 2)).shape == (0, 2, 2)


def test_angles_refused():
    lib, p = svdc.load_library(), svdc.make_rotary(torch.zeros(4, 2), (8, 6))

    def status(pos=1 << 20, table=1 << 21, **fields):
        q = svdc.Rotary.from_buffer_copy(p)
        for name, value in fields.items():
            setattr(q, name, value)
        return lib.svdcache_rotary_table(C.byref(q), pos, table, None)
    four, thetas = C.c_int32 * 4, C.c_double * 4
    assert lib.svdcache_rotary_table(None, 1 << 20, 1 << 21, None) == -1
    assert status(pos=0) == -1 and status(table=0) == -1 and status(pos=(1 << 20) + 2) == -4 and status(table=(1 << 20) + 4) == -4
    for fields in (dict(rows=-1), dict(rows=2 ** 31), dict(axes=0), dict(axes=5), dict(ld=1), dict(ld=2 ** 24 + 1), dict(dims=four(8, 7)), dict(dims=four(8, 0)),
                   dict(dims=four(-2, 8)), dict(dims=four(200, 58))):
        assert status(**fields) == -2
    for fields in (dict(whole=2), dict(theta=thetas(0.0, 1.0)), dict(theta=thetas(1.0, -1.0)), dict(theta=thetas(math.inf, 1.0)), dict(theta=thetas(math.nan, 1.0))):
        assert status(**fields) == -5
    assert status(rows=0, pos=0) == 0
    for bad in (lambda: svdc.make_rotary(torch.zeros(4, 2), (8,)), lambda: svdc.make_rotary(torch.zeros(4, 2).double(), (8, 6)),
                lambda: svdc.make_rotary(torch.zeros(4, 5), (2,) * 5), lambda: svdc.svdcache_rotary_table(p, torch.zeros(3, 2), torch.zeros(4, 7, 2)),
                lambda: svdc.svdcache_rotary_table(p, torch.zeros(4, 2), torch.zeros(4, 6, 2)),
                lambda: svdc.svdcache_rotary_table(p, torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 7, 2))):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(RuntimeError, match="GPU"):
        svdc.svdcache_rotary_table(p, torch.zeros(4, 2), torch.zeros(4, 7, 2))


# ---- norm and rotation ----------------------------------------------------------------------------------------------

def ref_heads(x, gain, table, halves, norm, eps):
    """(y, the sum of the sizes of its terms); x [batch, rows, heads, d], table [rows, pairs, 2] or [batch, rows, pairs, 2]"""
    x = x.cpu().double()
    if norm:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
        if gain is not None:
            x = x * gain.cpu().double()
    y, size = x.clone(), x.abs()
    if table is not None:
        n = table.shape[-2]
        t = table.cpu().double()
        t = t if t.dim() == 4 else t[None]
        c, s = t[:, :, None, :, 0], t[:, :, None, :, 1]
        at = [(j, n + j) if halves else (2 * j, 2 * j + 1) for j in range(n)]
        one, two = [i for i, _ in at], [j for _, j in at]
        a, b = x[..., one], x[..., two]
        y[..., one], y[..., two] = a * c - b * s, a * s + b * c
        size[..., one], size[..., two] = (a * c).abs() + (b * s).abs(), (a * s).abs() + (b * c).abs()
    return y, size


def check_heads(got, x, gain, table, halves, norm, eps):
    y, size = ref_heads(x, gain, table, halves, norm, eps)
    half_step = 2.0 ** -8 if got.dtype == BF16 else 2.0 ** -24
    tol = 1.01 * (half_step * y.abs() + (x.shape[-1] + 16) * 2.0 ** -24 * size)
    off = (got.cpu().double() - y).abs()
    assert (off <= tol).all(), f"off by {float((off - tol).max()):.3e} more than allowed"


def inputs(batch, rows, heads, kv, d, pairs, dtype, per_seq=False, seed=2):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(batch, rows, (heads + 2 * kv) * d, generator=g) * torch.exp(torch.randn((heads + 2 * kv) * d, generator=g))
    x[:, ::5] = 0
    x = x.to(dtype).cuda()
    q, k, v = (t.unflatten(2, (-1, d)) for t in x.split([heads * d, kv * d, kv * d], 2))
    gains = [(1 + 0.3 * torch.randn(d, generator=g)).cuda() for _ in range(2)]
    angle = torch.rand(*((batch,) if per_seq else ()), rows, pairs, generator=g) * 50
    table = torch.stack([angle.cos(), angle.sin()], -1).cuda() if pairs else None
    return q, k, v, gains, table


@gpu
@pytest.mark.parametrize("dtype,dtype_out", [(BF16, BF16), (F32, BF16), (F32, F32), (BF16, F32)])
@pytest.mark.parametrize("layout", ["neighbours", "halves"])
@pytest.mark.parametrize("size", [  # batch, rows, heads, heads of keys, head_dim, pairs
    (1, 1, 24, 24, 128, 64), (2, 37, 5, 5, 128, 64), (1, 9, 16, 8, 72, 36), (1, 9, 16, 8, 72, 27), (3, 4, 7, 1, 64, 32), (1, 3, 3, 2, 64, 20), (1, 5, 2, 2, 256, 128),
    (1, 5, 2, 1, 256, 100), (1, 4, 3, 3, 33, 16), (1, 4, 3, 3, 33, 0), (2, 3, 2, 2, 1, 0), (1, 2, 50, 7, 8, 4), (1, 3, 2, 2, 130, 65), (1, 2, 2, 2, 24, 12),
    (1, 2, 130, 3, 2, 1), (1, 700, 2, 2, 96, 48), (3, 531, 1, 3, 128, 64), (2, 301, 5, 1, 8, 4), (5, 67, 3, 2, 40, 18)], ids=lambda s: "x".join(map(str, s)))
def test_heads(size, layout, dtype, dtype_out):
    batch, rows, heads, kv, d, pairs = size
    q, k, v, (gq, gk), table = inputs(batch, rows, heads, kv, d, pairs, dtype)
    qo, ko, vo = svdc.norm_rotate(q, k, v, gq, gk, table, layout, dtype=dtype_out)
    check_heads(qo, q, gq, table, layout == "halves", True, 1e-6)
    check_heads(ko, k, gk, table, layout == "halves", True, 1e-6)
    assert torch.equal(vo, v.to(dtype_out))


@gpu
@pytest.mark.parametrize("layout", ["neighbours", "halves"])
@pytest.mark.parametrize("d,pairs", [(128, 64), (72, 27)])
def test_parts_of_the_operator(d, pairs, layout):
    """Without a norm, without a table, gains missing, queries or keys or values alone, a table for each sequence."""
    halves = layout == "halves"
    q, k, v, (gq, gk), table = inputs(2, 11, 4, 2, d, pairs, BF16, per_seq=True)
    qo, ko, vo = svdc.norm_rotate(q, k, None, None, None, table, layout, norm=False)
    assert vo is None
    check_heads(qo, q, None, table, halves, False, 0.0)
    check_heads(ko, k, None, table, halves, False, 0.0)
    qo, ko, _ = svdc.norm_rotate(q, k, None, gq, None, None, layout, eps=0.5)
    check_heads(qo, q, gq, None, halves, True, 0.5)
    check_heads(ko, k, None, None, halves, True, 0.5)
    qo, none, _ = svdc.norm_rotate(q, None, None, gq, None, table[0], layout)
    assert none is None
    check_heads(qo, q, gq, table[0], halves, True, 1e-6)
    _, ko, vo = svdc.norm_rotate(None, k, v, None, gk, table[1], layout)
    check_heads(ko, k, gk, table[1], halves, True, 1e-6)
    assert torch.equal(vo, v)
    _, _, vo = svdc.norm_rotate(None, None, v, dtype=F32)
    assert torch.equal(vo, v.float())
    qo, ko, _ = svdc.norm_rotate(q, k, norm=False)
    assert torch.equal(qo, q) and torch.equal(ko, k)


@gpu
@pytest.mark.parametrize("layout", ["neighbours", "halves"])
@pytest.mark.parametrize("d,pairs,pad", [(128, 64, 0), (128, 64, 1), (72, 27, 3), (64, 32, 8)])
def test_in_place_and_joint_buffers(d, pairs, pad, layout):
    """In place, and into rows and columns of wider buffers, whose other elements stay."""
    q, k, v, (gq, gk), table = inputs(2, 13, 4, 2, d, pairs, BF16)
    wide = [torch.full((2, 13 + 6, h + 1, d + pad), 7.0, device="cuda", dtype=BF16) for h in (4, 2, 2)]
    out = [w[:, 5:-1, 1:, pad:] for w in wide]
    p = svdc.make_norm_rotate(q, k, v, *out, table, layout)
    svdc.svdcache_norm_rotate(p, q, k, v, gq, gk, table, *out)
    want = svdc.norm_rotate(q, k, v, gq, gk, table, layout)
    assert all(torch.equal(o, w) for o, w in zip(out, want))
    for w, o in zip(wide, out):
        o.fill_(7.0)
        assert (w == 7.0).all()
    by_head = [t.transpose(1, 2).contiguous().transpose(1, 2) for t in (q, k)]
    svdc.svdcache_norm_rotate(svdc.make_norm_rotate(*by_head, None, *by_head, None, table, layout), *by_head, None, gq, gk, table, *by_head, None)
    assert torch.equal(by_head[0], want[0]) and torch.equal(by_head[1], want[1])
    p = svdc.make_norm_rotate(q, k, None, q, k, None, table, layout)
    before = v.clone()
    svdc.svdcache_norm_rotate(p, q, k, None, gq, gk, table, q, k, None)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(v, before)


@gpu
def test_numbers_that_are_not_finite():
    """A NaN or an infinity stays in its head, and in the columns of its pair where there is no norm."""
    q, _, _, (gq, _), table = inputs(1, 4, 6, 6, 128, 30, F32)
    q = q.contiguous()
    q[0, 1, 2, 7], q[0, 2, 3, 100] = math.nan, math.inf
    qo, _, _ = svdc.norm_rotate(q, gain_q=gq, table=table)
    bad = torch.zeros(1, 4, 6, dtype=torch.bool)
    bad[0, 1, 2] = bad[0, 2, 3] = True
    assert torch.isfinite(qo[~bad.cuda()]).all() and qo[0, 1, 2].isnan().all() and qo[0, 2, 3, 100].isnan()
    qo, _, _ = svdc.norm_rotate(q, table=table, norm=False)
    assert qo[0, 1, 2, 6:8].isnan().all() and torch.isfinite(qo[0, 1, 2, :6]).all() and torch.isfinite(qo[0, 1, 2, 8:]).all()
    assert qo[0, 2, 3, 100] == math.inf and torch.isfinite(qo[0, 2, 3, :100]).all() and torch.isfinite(qo[0, 2, 3, 101:]).all()


@gpu
def test_many_rows_streams_and_graphs():
    """More rows than workgroups; the same bits on another stream and from a captured graph on new inputs."""
    q, k, v, (gq, gk), table = inputs(3, 3000, 3, 3, 64, 32, BF16)
    want = svdc.norm_rotate(q, k, v, gq, gk, table)
    check_heads(want[0], q, gq, table, False, True, 1e-6)
    out = [torch.empty_like(t) for t in want]
    p = svdc.make_norm_rotate(q, k, v, *out, table)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        svdc.svdcache_norm_rotate(p, q, k, v, gq, gk, table, *out)
    side.synchronize()
    assert all(torch.equal(o, w) for o, w in zip(out, want))
    pos = torch.zeros(3000, 2, device="cuda")
    pr = svdc.make_rotary(pos, (20, 44))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        svdc.svdcache_rotary_table(pr, pos, table)
        svdc.svdcache_norm_rotate(p, q, k, v, gq, gk, table, *out)
    for turn in range(4):
        pos.copy_(torch.randn(3000, 2, device="cuda") * 100)
        for o in out:
            o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        want = svdc.norm_rotate(q, k, v, gq, gk, svdc.rotary_table(pos, (20, 44)))
        assert all(torch.equal(o, w) for o, w in zip(out, want))


def test_heads_refused():
    lib, s = svdc.load_library(), svdc.Heads(1000, 100, 64)
    base = svdc.NormRotate(2, 10, 4, 2, 64, 1, 1, 1, 32, 0, 1e-6, 0, 0, s, s, s, s, s, s)
    at = {n: (i + 1) << 20 for i, n in enumerate(("Q", "K", "V", "gain_q", "gain_k", "table", "Qo", "Ko", "Vo"))}

    def status(where=None, **fields):
        q = svdc.NormRotate.from_buffer_copy(base)
        for name, value in fields.items():
            setattr(q, name, value)
        return lib.svdcache_norm_rotate(C.byref(q), *{**at, **(where or {})}.values(), None)
    assert lib.svdcache_norm_rotate(None, *at.values(), None) == -1
    for fields, code in ((dict(dtype=2), -3), (dict(dtype_out=7), -3), (dict(eps=-1.0), -5), (dict(eps=math.nan), -5), (dict(norm=2), -5), (dict(layout=2), -5),
                         (dict(reserved=1), -5), (dict(batch=-1), -2), (dict(rows=2 ** 31), -2), (dict(batch=2 ** 16, rows=2 ** 16), -2), (dict(heads=0), -2),
                         (dict(kv_heads=2 ** 16 + 1), -2), (dict(head_dim=0), -2), (dict(head_dim=257), -2), (dict(pairs=33), -2), (dict(pairs=-1), -2),
                         (dict(table_seq=-1), -2), (dict(q=svdc.Heads(0, -1, 0)), -2), (dict(ko=svdc.Heads(0, 2 ** 22 + 1, 0)), -2), (dict(vo=svdc.Heads(-1, 0, 0)), -2)):
        assert status(**fields) == code, fields
    for name in ("Q", "K", "V", "Qo", "Ko", "Vo", "table"):
        assert status({name: 0}) == -1
    for name in ("Q", "K", "V", "Qo", "Ko", "Vo"):
        assert status({name: (20 << 20) + 1}) == -4
    assert status({"table": (20 << 20) + 4}) == -4 and status({"gain_q": (20 << 20) + 2}) == -4
    # in place with other strides or another type, and outputs that are each other's or another's input
    assert status({"Qo": at["Q"]}, qo=svdc.Heads(1000, 101, 64)) == -5 and status({"Vo": at["V"]}, dtype=0) == -5
    for one, other in (("Qo", "Ko"), ("Ko", "Vo"), ("Qo", "K"), ("Ko", "Q"), ("Vo", "K"), ("Qo", "V")):
        assert status({one: at[other]}) == -5
    assert status(batch=0) == 0 and status({"Q": 0}, rows=0) == 0
    q = torch.zeros(2, 8, 4, 64)
    table = torch.zeros(8, 32, 2)
    p = svdc.make_norm_rotate(q, None, None, q, None, None, table)
    with pytest.raises(RuntimeError, match="GPU"):
        svdc.svdcache_norm_rotate(p, q, None, None, None, None, table, q, None, None)
    for bad in (lambda: svdc.make_norm_rotate(q, Ko=q), lambda: svdc.make_norm_rotate(), lambda: svdc.make_norm_rotate(q, Qo=q, layout="other"),
                lambda: svdc.svdcache_norm_rotate(p, q, None, None, None, None, None, q, None, None),
                lambda: svdc.svdcache_norm_rotate(p, q, None, None, None, None, table[:7], q, None, None),
                lambda: svdc.svdcache_norm_rotate(p, q, None, None, torch.zeros(63), None, table, q, None, None),
                lambda: svdc.svdcache_norm_rotate(p, q[:, :7], None, None, None, None, table, q, None, None),
                lambda: svdc.svdcache_norm_rotate(p, q, None, None, None, None, table, q.transpose(1, 2).contiguous().transpose(1, 2), None, None)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(ValueError, match="share memory"):
        one = torch.zeros(2, 1, 4, 64).expand(2, 8, 4, 64)
        svdc.svdcache_norm_rotate(svdc.make_norm_rotate(q, None, None, one, None, None, table), q, None, None, None, None, table, one, None, None)


# ---- angles of any base ---------------------------------------------------------------------------------------------------

PI = Decimal("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899")


def exact_turns(pos, n, theta):
    """Angles [rows, n / 2] less whole turns, from the definition with 120 digits, and the angles themselves, as float64."""
    with localcontext() as c:
        c.prec = 120
        freq = [Decimal(theta) ** (Decimal(-2 * i) / n) for i in range(n // 2)]
        x = [[Decimal(p) * f for f in freq] for p in pos]
        left = [[a - (a / (2 * PI)).to_integral_value() * 2 * PI for a in row] for row in x]
    return np.array(left, dtype=np.float64), np.array(x, dtype=np.float64)


@gpu
@pytest.mark.parametrize("theta", [1.5, 10000.0, 5e5, 1e30, 1e300])
def test_angles_from_exact_frequencies(theta):
    """The bound 2^-22 + 2^-50 |x| with x from exponents that are not rounded, at any base, and at positions where the second term counts."""
    n = 254
    pos = [0.0, 1.0, -3.0, 12345.0, 2.0 ** 31, -(2.0 ** 40), 2.0 ** 52, 2.0 ** 60, 2.0 ** 80, -(2.0 ** 100)]
    left, x = exact_turns(pos, n, theta)
    got = svdc.rotary_table(torch.tensor(pos, device="cuda").unsqueeze(1), (n,), theta).cpu().double().numpy()
    tol = 2.0 ** -22 + 2.0 ** -50 * np.abs(x)
    assert (np.abs(got[..., 0] - np.cos(left)) <= tol).all() and (np.abs(got[..., 1] - np.sin(left)) <= tol).all()


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [128, 72, 33, 8, 256])
def test_small_heads_without_eps(d, dtype):
    """mean + eps counts as 2^-126 at least: with eps = 0 heads of numbers below 2^-63 are multiplied by 2^63, zeros stay zeros; from there on the formula holds."""
    g = torch.Generator().manual_seed(30)
    signs = (torch.randint(0, 2, (1, 6, 1, d), generator=g) * 2 - 1).float()
    sizes = torch.tensor([0.0, 2.0 ** -100, 2.0 ** -70, 2.0 ** -64, 2.0 ** -62, 2.0 ** -40]).view(1, 6, 1, 1)
    x = (signs * sizes).to(dtype).cuda()
    got = svdc.norm_rotate(x, eps=0.0)[0].cpu().double()
    want = torch.where(sizes < 2.0 ** -63, signs * sizes * 2.0 ** 63, signs).double()
    assert ((got - want).abs() <= 1.01 * ((2.0 ** -8 if dtype == BF16 else 2.0 ** -24) + (d + 16) * 2.0 ** -24) * want.abs()).all()
