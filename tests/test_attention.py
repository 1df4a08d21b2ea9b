"""Attention against a plain implementation in float64 that shares no code with the library, and its refusals.

Tolerances, derived for every element.  With p the exact probabilities (they sum to 1), A = sum p |v|, d columns and n keys:
  products   a sum of d float32 products is off by at most (d + 1) 2^-24 B with B = scale max sum |q k|; scaling, subtracting the maximum and the hardware's power of
             two add less than 7 * 2^-24 B + 2^-22 to that, so that a probability is off by at most e = (d + 8) 2^-24 B + 2^-22 of itself, their sum as much.
  sums       of n terms in float32, numerator and denominator: n 2^-24 each; rescaled and joined in parts: 2^-20 is far more than these steps add.
  bfloat16   a probability is rounded by at most 2^-8 of itself, the result by 2^-8 of itself; float32: 2^-24 of the result.
  So |got - want| <= u |want| + (2 e + 2 n 2^-24 + 2^-20 + [2^-8 for bfloat16]) A, u = 2^-8 or 2^-24, and the product of both terms, which 1.01 covers.
"""
import ctypes as C
import math

import pytest
import torch

import paper_2601_07396_amd as svdc

F32, BF16 = torch.float32, torch.bfloat16
gpu = pytest.mark.gpu


def ref(q, k, v, scale):
    """(o, A, B) of one sequence: q [rows, heads, d], k and v [keys, kv_heads, d], in float64."""
    q, k, v = (t.detach().cpu().double().transpose(0, 1) for t in (q, k, v))
    share = q.shape[0] // max(1, k.shape[0])
    k, v = k.repeat_interleave(share, 0), v.repeat_interleave(share, 0)
    if k.shape[1] == 0:
        z = torch.zeros(q.shape[1], q.shape[0], q.shape[2], dtype=torch.float64)
        return z, z, 0.0
    s = scale * q @ k.transpose(1, 2)
    p = torch.exp(s - s.amax(2, keepdim=True))
    p = p / p.sum(2, keepdim=True)
    B = float((scale * q.abs() @ k.abs().transpose(1, 2)).max()) if s.numel() else 0.0
    return (p @ v).transpose(0, 1), (p @ v.abs()).transpose(0, 1), B


def check(got, q, k, v, scale, dtype):
    o, A, B = ref(q, k, v, scale)
    d, n = q.shape[-1], k.shape[0]
    e = (d + 8) * 2.0 ** -24 * B + 2.0 ** -22
    u, rounded = (2.0 ** -8, 2.0 ** -8) if dtype == BF16 else (2.0 ** -24, 0.0)
    tol = 1.01 * (u * o.abs() + (2 * e + 2 * n * 2.0 ** -24 + 2.0 ** -20 + rounded) * A)
    off = (got.detach().cpu().double() - o).abs()
    assert torch.isfinite(got).all()
    assert (off <= tol).all(), f"off by {float((off - tol).max()):.3e} more than allowed, at most {float((off / (tol + 1e-300)).max()):.2f} of it"


def heads(g, batch, rows, n, d, dtype, layout="rows", scale=1.0):
    """[batch, rows, n, d]: "rows" as a product gives them, "heads" with a head's rows together, "slice" out of a wider result, "odd" at odd strides"""
    def normal(*shape):
        return (scale * torch.randn(*shape, generator=g)).to(dtype).cuda()
    if layout == "heads":
        return normal(batch, n, rows, d).transpose(1, 2)
    if layout == "slice":
        return normal(batch, rows, 3 * n * d)[:, :, n * d:2 * n * d].unflatten(2, (n, d))
    if layout == "odd":
        return normal(batch, rows + 1, n + 1, d + 3)[:, 1:, 1:, 1:d + 1]
    return normal(batch, rows, n, d)


def like(t):
    """An output of t's layout, NaN everywhere beforehand."""
    return torch.full_like(t, float("nan")) if t.is_contiguous() else torch.full(t.shape, float("nan"), device=t.device, dtype=t.dtype)


def call(q, k, v, out, q_span=None, k_span=None, key_mask=None, scale=None, **most):
    p = svdc.make_attention(q, k, v, out, q_span, k_span, scale, **most)
    svdc.svdcache_attention(p, q, k, v, out, q_span, k_span, key_mask, svdc.alloc_attention_workspace(p, "cuda"))
    return p


SIZES = [  # batch, queries, keys, heads, heads of keys, head_dim
    (1, 1, 1, 1, 1, 128), (1, 1, 512, 24, 24, 128), (2, 33, 65, 3, 3, 128), (1, 128, 64, 2, 2, 128), (1, 129, 191, 2, 1, 128), (2, 257, 300, 4, 2, 64),
    (1, 40, 1000, 6, 2, 72), (3, 31, 97, 5, 5, 80), (1, 300, 200, 2, 2, 96), (1, 70, 130, 2, 2, 256), (1, 300, 90, 1, 1, 256), (2, 64, 64, 4, 4, 8),
    (1, 50, 77, 3, 1, 33), (1, 17, 40, 2, 2, 1), (1, 140, 333, 2, 2, 130), (1, 9, 5000, 2, 2, 128), (1, 3, 9000, 1, 1, 40), (2, 513, 700, 2, 2, 128),
    (2, 7, 300, 41, 1, 72), (1, 1, 2000, 24, 3, 128), (1, 200, 260, 6, 2, 128), (2, 127, 90, 9, 3, 64), (1, 5, 130, 130, 1, 33),
]


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_sizes(size, dtype):
    batch, n, m, h, hk, d = size
    g = torch.Generator().manual_seed(7)
    q, k, v = heads(g, batch, n, h, d, dtype, scale=1.5), heads(g, batch, m, hk, d, dtype), heads(g, batch, m, hk, d, dtype)
    out = like(q)
    call(q, k, v, out)
    for b in range(batch):
        check(out[b], q[b], k[b], v[b], d ** -0.5, dtype)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("layout", ["heads", "slice", "odd"])
@pytest.mark.parametrize("size", [(2, 150, 210, 4, 2, 128), (2, 5, 800, 3, 3, 64), (1, 260, 100, 2, 2, 72)], ids=lambda s: "x".join(map(str, s)))
def test_layouts(size, layout, dtype):
    batch, n, m, h, hk, d = size
    g = torch.Generator().manual_seed(8)
    q, k, v = heads(g, batch, n, h, d, dtype, layout), heads(g, batch, m, hk, d, dtype, layout), heads(g, batch, m, hk, d, dtype, layout)
    whole = torch.full((batch, n + 2, h + 1, d + 5), 3.0, device="cuda", dtype=dtype)
    out = whole[:, 1:-1, 1:, 2:-3]
    call(q, k, v, out, scale=0.3)
    for b in range(batch):
        check(out[b], q[b], k[b], v[b], 0.3, dtype)
    out.fill_(3.0)
    assert (whole == 3.0).all(), "written beside the result"


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,m", [(200, 300), (3, 3000)])
def test_masks(n, m, dtype):
    """Scattered keys, runs over whole tiles, one key, none; what lies in masked rows does not matter."""
    batch, h, d = 6, 2, 128
    g = torch.Generator().manual_seed(9)
    q, k, v = (heads(g, batch, rows, h, d, dtype) for rows in (n, m, m))
    keep = torch.zeros(batch, m, dtype=torch.bool)
    keep[0] = torch.rand(m, generator=g) < 0.5
    keep[1, :70] = True
    keep[2, -1] = True
    keep[3, 130:] = True
    keep[5] = True
    for bad, of in ((float("nan"), k), (float("inf"), k), (float("nan"), v), (-float("inf"), v), (torch.finfo(dtype).min, k)):
        kk, vv = k.clone(), v.clone()
        (kk if of is k else vv)[~keep.cuda()] = bad
        out = like(q)
        call(q, kk, vv, out, key_mask=keep.to(torch.uint8).cuda() if of is k else keep.cuda())
        for b in range(batch):
            check(out[b], q[b], k[b][keep[b].cuda()], v[b][keep[b].cuda()], d ** -0.5, dtype)
        assert (out[4] == 0).all()


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("m", [40, 2000])
def test_numbers_at_the_ends(m, dtype):
    """Logits far apart, equal ones, a NaN in one query, one key, one value; products of -infinity."""
    h, d, n = 1, 64, 40
    g = torch.Generator().manual_seed(10)
    q, k, v = (heads(g, 1, rows, h, d, dtype) for rows in (n, m, m))
    out = like(q)
    call(100 * q, k, v, out)
    check(out[0], 100 * q[0], k[0], v[0], d ** -0.5, dtype)
    rising = k * torch.linspace(0.01, 40, m, device="cuda").to(dtype)[None, :, None, None]      # the maximum moves on and on
    call(q, rising, v, out)
    check(out[0], q[0], rising[0], v[0], d ** -0.5, dtype)
    call(torch.zeros_like(q), k, v, out)
    check(out[0], 0 * q[0], k[0], v[0], d ** -0.5, dtype)
    bad = q.clone()
    bad[0, 5, 0, 3] = float("nan")
    call(bad, k, v, out)
    assert out[0, 5].isnan().all() and torch.isfinite(out[0, :5]).all() and torch.isfinite(out[0, 6:]).all()
    bad = k.clone()
    bad[0, m // 2, 0, 3] = float("nan")
    call(q, bad, v, out)
    assert out.isnan().all()
    bad = v.clone()
    bad[0, m // 2, 0, 3] = float("nan")
    call(q, k, bad, out)
    assert out[..., 3].isnan().all() and torch.isfinite(out[..., :3]).all() and torch.isfinite(out[..., 4:]).all()
    low = torch.full_like(k, -float("inf"))
    call(q.abs() + 1, low, v, out)
    assert (out == 0).all()


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("cross", [False, True])
def test_spans(cross, masked, dtype):
    """Packed and padded sequences, empty ones, a single row, spans that leave the tensors: rows of no span stay as they were."""
    h, hk, d, total, k_total = 6, 2, 64, 700, 900 if cross else 700
    g = torch.Generator().manual_seed(11)
    q, k, v = heads(g, 1, total, h, d, dtype)[0], heads(g, 1, k_total, hk, d, dtype)[0], heads(g, 1, k_total, hk, d, dtype)[0]
    q_of = [(0, 129), (129, 1), (130, 0), (140, 200), (690, 300), (400, 77), (-20, 0), (900, 5), (350, 50), (2 ** 31 - 1, 2 ** 31 - 1), (-3, -4)]
    k_of = [(5, 300), (1, 64), (0, 10), (0, 0), (890, 2 ** 31 - 1), (300, 63), (0, 9), (3, 3), (-10, 75), (7, 7), (0, 1)] if cross else q_of
    q_span, k_span = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (q_of, k_of))
    mask = (torch.rand(k_total, generator=g) < 0.7).cuda() if masked else None
    out = torch.full_like(q, 5.0)
    call(q, k, v, out, q_span, k_span, mask, q_most=250, k_most=250)
    seen = torch.zeros(total, dtype=torch.bool)

    def rows(first, n, all_rows):
        lo, hi = max(0, first), min(all_rows, first + max(0, n))
        return lo, min(hi, lo + 250)
    for (qa, qn), (ka, kn) in zip(q_of, k_of):
        lo, hi = rows(qa, qn, total)
        if lo >= hi:
            continue
        klo, khi = rows(ka, kn, k_total)
        keys = torch.arange(klo, max(klo, khi), device="cuda")
        if masked:
            keys = keys[mask[keys]]
        check(out[lo:hi], q[lo:hi], k[keys], v[keys], d ** -0.5, dtype)
        seen[lo:hi] = True
    assert (out[~seen.cuda()] == 5.0).all()


@gpu
def test_spans_of_queries_alone():
    """Padded queries over keys of equal length."""
    g = torch.Generator().manual_seed(12)
    q, k, v = heads(g, 1, 100, 2, 128, BF16)[0], heads(g, 3, 90, 2, 128, BF16), heads(g, 3, 90, 2, 128, BF16)
    span = torch.tensor([[0, 30], [40, 0], [60, 33]], dtype=torch.int32, device="cuda")
    out = torch.zeros_like(q)
    call(q, k, v, out, q_span=span)
    for b, (a, n) in enumerate(span.tolist()):
        check(out[a:a + n], q[a:a + n], k[b], v[b], 128 ** -0.5, BF16)
    assert (out[30:60] == 0).all() and (out[93:] == 0).all()


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_offsets_beyond_32_bits(dtype):
    """Keys, values and rows that lie more than 2^32 bytes (bfloat16: 2^31 elements) into their tensors."""
    step, n, d = 1 << 16, 40000 if dtype == BF16 else 20000, 64
    g = torch.Generator().manual_seed(13)
    wide = torch.empty(n, step, device="cuda", dtype=dtype)
    k, v, q = wide[:, :d].unsqueeze(1), wide[:, d:2 * d].unsqueeze(1), wide[:, 2 * d:3 * d].unsqueeze(1)
    for t in (k, v, q):
        t.copy_(torch.randn(n, 1, d, generator=g).to(dtype))
    out = wide[:, 3 * d:4 * d].unsqueeze(1)
    rows = torch.tensor([[n - 50, 50]], dtype=torch.int32, device="cuda")
    call(q, k, v, out, rows, rows, q_most=64, k_most=64)
    check(out[n - 50:], q[n - 50:], k[n - 50:], v[n - 50:], d ** -0.5, dtype)
    call(q[n - 8:], k, v, out[n - 8:])
    check(out[n - 8:], q[n - 8:], k, v, d ** -0.5, dtype)


@gpu
def test_no_rows_and_no_keys():
    q, none = torch.ones(2, 5, 3, 64, device="cuda"), torch.ones(2, 0, 3, 64, device="cuda")
    out = like(q)
    call(q, none, none, out)
    assert (out == 0).all()
    call(none, q, q, torch.empty_like(none))


@gpu
def test_spans_of_nothing():
    """Tensors without rows: nothing to write, or no keys for anybody."""
    q, none = torch.ones(6, 3, 64, device="cuda"), torch.ones(0, 3, 64, device="cuda")
    span, out = torch.tensor([[0, 4], [4, 9]], dtype=torch.int32, device="cuda"), torch.full((6, 3, 64), 7.0, device="cuda")
    call(q, none, none, out, span, span, q_most=9, k_most=9)
    assert (out == 0).all()
    call(none, q, q, torch.empty_like(none), span, span, q_most=9, k_most=9)


@gpu
@pytest.mark.parametrize("dtype,m", [(BF16, 4100), (BF16, 130), (F32, 2050)])
def test_more_units_than_compute_units(dtype, m):
    """360 units of work: a workgroup each for the first ones, parts of the keys for the last ones where there are many keys."""
    batch, n, h, d = 3, 640, 24, 128
    g = torch.Generator().manual_seed(15)
    q, k, v = heads(g, batch, n, h, d, dtype), heads(g, batch, m, h, d, dtype), heads(g, batch, m, h, d, dtype)
    out = like(q)
    p = call(q, k, v, out)
    assert (svdc.svdcache_attention_workspace_bytes(p) > 0) == (m > 1000)
    assert torch.isfinite(out).all()
    for b, head in ((0, 0), (1, 13), (2, 7), (2, 15), (2, 16), (2, 23)):
        check(out[b][:, head:head + 1], q[b][:, head:head + 1], k[b][:, head:head + 1], v[b][:, head:head + 1], d ** -0.5, dtype)


@gpu
@pytest.mark.parametrize("size", [(1, 300, 400, 2, 2, 128), (1, 4, 3000, 2, 2, 128), (2, 700, 4100, 24, 24, 64)], ids=["whole", "parts", "last_round"])
def test_streams_graphs_and_repeats(size):
    """The same bits on other streams at once (a workspace each), when repeated, and from a captured graph on new inputs with eager work in between."""
    batch, n, m, h, hk, d = size
    g = torch.Generator().manual_seed(14)
    inputs = [[heads(g, batch, rows, x, d, BF16) for rows, x in ((n, h), (m, hk), (m, hk))] for _ in range(3)]
    wants = []
    for x in inputs:
        out = like(x[0])
        p = call(*x, out)
        wants.append(out)
    for x, want in zip(inputs, wants):
        again = like(want)
        call(*x, again)
        assert torch.equal(again, want)
    sides = [(torch.cuda.Stream(), svdc.alloc_attention_workspace(p, "cuda"), like(wants[0])) for _ in range(2)]
    for _ in range(3):
        for i, (stream, ws, out) in enumerate(sides):
            if ws is not None:
                ws.fill_(0xFF)
            stream.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(stream):
                for _ in range(3):
                    svdc.svdcache_attention(p, *inputs[i], out, None, None, None, ws)
        for i, (stream, _, out) in enumerate(sides):
            stream.synchronize()
            assert torch.equal(out, wants[i])
            out.zero_()
        torch.cuda.synchronize()
    static, out, ws = [t.clone() for t in inputs[0]], like(wants[0]), svdc.alloc_attention_workspace(p, "cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        svdc.svdcache_attention(p, *static, out, None, None, None, ws)
    for turn in range(6):
        for s, x in zip(static, inputs[turn % 3]):
            s.copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, wants[turn % 3])
        call(*inputs[(turn + 1) % 3], like(out))
        out.zero_()


# ---- refusals (no GPU) ----------------------------------------------------------------------------------------------

POINTER = 1 << 20      # aligned, never read


def descriptor(**other):
    s = svdc.Heads(1000, 128, 64)
    p = svdc.Attention(2, 100, 100, 200, 200, 4, 2, 64, 1, 0.125, 0, s, s, s, s)
    for name, value in other.items():
        setattr(p, name, value)
    return p


def status(p, Q=POINTER, K=2 * POINTER, V=3 * POINTER, q_span=0, k_span=0, mask=0, Out=4 * POINTER, ws=5 * POINTER, bytes=1 << 40):
    return svdc.load_library().svdcache_attention(C.byref(p) if p is not None else None, Q, K, V, q_span, k_span, mask, Out, ws, bytes, None)


@pytest.mark.parametrize("fields,code", [
    (dict(dtype=2), -3), (dict(dtype=-1), -3), (dict(scale=0.0), -5), (dict(scale=-1.0), -5), (dict(scale=math.inf), -5), (dict(scale=math.nan), -5),
    (dict(reserved=1), -5), (dict(batch=-1), -2), (dict(batch=65536), -2), (dict(q_rows=-1), -2), (dict(k_rows=2 ** 31), -2), (dict(batch=3, q_rows=2 ** 30), -2),
    (dict(heads=0), -2), (dict(heads=3), -2), (dict(kv_heads=0), -2), (dict(heads=2 ** 16 + 2), -2), (dict(head_dim=0), -2), (dict(head_dim=257), -2),
    (dict(heads=2 ** 16, q_rows=2 ** 20), -2), (dict(batch=1, heads=2 ** 14, kv_heads=1, q_rows=2 ** 16 + 1), -2), (dict(q=svdc.Heads(-1, 0, 0)), -2), (dict(k=svdc.Heads(0, 2 ** 22 + 1, 0)), -2),
    (dict(v=svdc.Heads(0, 0, 2 ** 40 + 1)), -2), (dict(o=svdc.Heads(2 ** 40 + 1, 0, 0)), -2), (dict(k=svdc.Heads(0, -5, 0)), -2)])
def test_refused_descriptors(fields, code):
    p = descriptor(**fields)
    assert status(p) == code
    assert svdc.svdcache_attention_workspace_bytes(p) == 0 or "q" in fields or "k" in fields or "v" in fields or "o" in fields


def test_refused_pointers():
    p = descriptor()
    assert status(None) == -1
    assert svdc.load_library().svdcache_attention_workspace_bytes(None) == 0
    for name in ("Q", "K", "V", "Out"):
        assert status(p, **{name: 0}) == -1
        assert status(p, **{name: POINTER * 9 + 1}) == -4
    assert status(p, q_span=POINTER + 4) == -4 and status(p, k_span=POINTER + 4) == -4
    for name in ("Q", "K", "V"):
        assert status(p, **{name: 4 * POINTER}) == -5
    assert status(descriptor(q_total=-1), q_span=POINTER) == -2 and status(descriptor(k_total=2 ** 31), k_span=POINTER) == -2
    assert status(descriptor(batch=0), Q=0) == 0 and status(descriptor(q_rows=0), Q=0) == 0
    assert status(descriptor(q_total=0), Q=0, q_span=POINTER) == 0


def test_workspace_is_checked():
    p = descriptor(batch=1, q_rows=1, k_rows=10000)
    need = svdc.svdcache_attention_workspace_bytes(p)
    assert need > 0
    assert status(p, ws=0) == -1 and status(p, ws=POINTER + 16) == -4 and status(p, bytes=need - 1) == -6


def test_binding_refuses():
    q, k = torch.zeros(2, 8, 4, 64), torch.zeros(2, 9, 2, 64)
    p = svdc.make_attention(q, k, k, q)
    with pytest.raises(RuntimeError, match="GPU"):
        svdc.svdcache_attention(p, q, k, k.clone(), q.clone())
    for bad in (q[:, :7], q[..., :32], q.double(), q[:1], q.transpose(1, 2).contiguous().transpose(1, 2)):
        with pytest.raises(ValueError, match="Q"):
            svdc.svdcache_attention(p, bad, k, k, q)
    with pytest.raises(ValueError, match="share memory"):
        one = torch.zeros(2, 8, 1, 64).expand(2, 8, 4, 64)
        svdc.svdcache_attention(svdc.make_attention(q, k, k, one), q, k, k, one)
    with pytest.raises(ValueError, match="key_mask"):
        svdc.svdcache_attention(p, q, k, k, q, key_mask=torch.zeros(2, 8, dtype=torch.uint8))
    with pytest.raises(ValueError, match="key_mask"):
        svdc.svdcache_attention(p, q, k, k, q, key_mask=torch.zeros(2, 9, dtype=torch.int32))
    span = torch.zeros(3, 2, dtype=torch.int32)
    with pytest.raises(ValueError, match="span"):
        svdc.make_attention(q, k, k, q, q_span=span)
    p = svdc.make_attention(q[0], k[0], k[0], q[0], span, span)
    with pytest.raises(ValueError, match="span"):
        svdc.svdcache_attention(p, q[0], k[0], k[0], q[0], span[:2], span)
    with pytest.raises(ValueError, match="span"):
        svdc.svdcache_attention(p, q[0], k[0], k[0], q[0], span.long(), span)


# ---- logits whose float32 steps pass the probabilities' range ---------------------------------------------------------
#
# Whole numbers times a power of two: float32 products and sums of them are exact, equal logits are equal bits, and logits that differ lie at least 2^16 apart, a probability of zero.  So
# e of the tolerances above is 2^-22 whatever the logits are, and ref's softmax of the exact products says how many keys share the probability.

def check_exact_products(got, q, k, v, scale, dtype):
    o, A, _ = ref(q, k, v, scale)
    u, rounded = (2.0 ** -8, 2.0 ** -8) if dtype == BF16 else (2.0 ** -24, 0.0)
    tol = 1.01 * (u * o.abs() + (2 * 2.0 ** -22 + 2 * k.shape[0] * 2.0 ** -24 + 2.0 ** -20 + rounded) * A)
    assert torch.isfinite(got).all()
    assert ((got.detach().cpu().double() - o).abs() <= tol).all()


def whole_numbers(n, m, d, dtype, seed=20):
    """Queries, and keys of which many are alike."""
    g = torch.Generator().manual_seed(seed)
    q, few = torch.randint(-3, 4, (1, n, 2, d), generator=g), torch.randint(-3, 4, (7, 2, d), generator=g)
    k = few[torch.randint(0, 7, (m,), generator=g)][None]
    return q.to(dtype).cuda(), k.to(dtype).cuda(), heads(g, 1, m, 2, d, dtype)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("steps,scale", [((8, 8), 2.0 ** 0), ((13, 14), 2.0 ** -3), ((20, 14), 2.0 ** -3), ((20, 20), 2.0 ** 0), ((60, 50), 2.0 ** 20), ((0, 0), 2.0 ** 126), ((60, 57), 2.0 ** -3)])
@pytest.mark.parametrize("n,m,d", [(150, 300, 64), (40, 1000, 128), (3, 3000, 128), (33, 260, 74), (70, 200, 256), (3, 2500, 200)])
def test_large_logits(n, m, d, steps, scale, dtype):
    """Logits of 2^16 and far more, keys with the same one in many tiles and parts; larger and larger ones; none but negative ones."""
    q, k, v = whole_numbers(n, m, d, dtype)
    q, k = q * 2.0 ** steps[0], k * 2.0 ** steps[1]
    out = like(q)
    call(q, k, v, out, scale=scale)
    check_exact_products(out[0], q[0], k[0], v[0], scale, dtype)
    if n == 3:                                                  # 256 units, a whole one each
        many = [t.expand(128, *t.shape[1:]) for t in (q, k, v)]
        all_out = torch.full(many[0].shape, float("nan"), device="cuda", dtype=dtype)
        assert svdc.svdcache_attention_workspace_bytes(call(*many, all_out, scale=scale)) == 0
        check_exact_products(all_out[77], q[0], k[0], v[0], scale, dtype)
    call(-q.abs(), k.abs() + 2.0 ** steps[1], v, out, scale=scale)
    check_exact_products(out[0], -q[0].abs(), k[0].abs() + 2.0 ** steps[1], v[0], scale, dtype)
    rising = k * (torch.arange(m, device="cuda") // 50 % 8).to(dtype)[None, :, None, None]
    if steps != (60, 57):                                       # eight times as much passes float32
        call(q, rising, v, out, scale=scale)
        check_exact_products(out[0], q[0], rising[0], v[0], scale, dtype)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("size", [1e8, 1e9, 1e11, 1e20])
@pytest.mark.parametrize("n,m,d", [(200, 300, 128), (3, 3000, 64)])
def test_large_random_logits(n, m, d, size, dtype):
    """Numbers that are not exact: the best key takes all wherever the others are further below it than the products' rounding."""
    g = torch.Generator().manual_seed(21)
    q, k, v = (heads(g, 1, rows, 2, d, dtype) for rows in (n, m, m))
    q = q * size ** 0.5
    k = k * size ** 0.5
    out = like(q)
    call(q, k, v, out)
    check(out[0], q[0], k[0], v[0], d ** -0.5, dtype)
    for head in range(2):
        s = d ** -0.5 * q[0, :, head].cpu().double() @ k[0, :, head].cpu().double().T
        B = d ** -0.5 * float((q[0, :, head].cpu().double().abs() @ k[0, :, head].cpu().double().abs().T).max())
        two = s.topk(2, dim=1)
        alone = (two.values[:, 0] - two.values[:, 1] > 2 * (d + 8) * 2.0 ** -24 * B + 40).nonzero()[:, 0]
        assert len(alone) >= 1
        want = v[0, two.indices[alone, 0].cuda(), head].double()
        tol = 1.01 * (2.0 ** -8 * 2 + 2.0 ** -20 if dtype == BF16 else 2.0 ** -20 + 2.0 ** -22) * want.abs() + 2.0 ** -40 * v.abs().max().double()
        assert ((out[0, alone.cuda(), head].double() - want).abs() <= tol).all()


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,m", [(64, 500), (9, 3000)])
def test_large_logits_beside_ordinary_ones(n, m, dtype):
    """One query of a tile with large logits, with infinite ones, or without a number: the others are as near as ever."""
    g = torch.Generator().manual_seed(22)
    q, k, v = (heads(g, 1, rows, 2, 128, dtype) for rows in (n, m, m))
    out, others = like(q), [i for i in range(n) if i != 5]
    for bad in (1e9, 1e30, float("inf"), float("nan")):
        q[:, 5] = bad
        call(q, k, v, out)
        check(out[0, others], q[0, others], k[0], v[0], 128 ** -0.5, dtype)
        assert torch.isfinite(out[0, 5]).all() if math.isfinite(bad) else out[0, 5].isnan().all()


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("steps,scale", [((20, 14), 2.0 ** -3), ((60, 50), 2.0 ** 20)])
@pytest.mark.parametrize("n,m,d", [(150, 300, 128), (3, 3000, 128), (40, 700, 74)])
def test_large_logits_under_a_mask(n, m, d, steps, scale, dtype):
    """The largest logits left out, whole tiles and parts without keys among the others, one key, none; heads that share keys."""
    q, k, v = whole_numbers(n, m, d, dtype, seed=26)
    q, k, v = (q * 2.0 ** steps[0]).expand(4, -1, -1, -1), (k * 2.0 ** steps[1])[:, :, :1].repeat(4, 1, 1, 1), v[:, :, :1].repeat(4, 1, 1, 1)
    keep = torch.zeros(4, m, dtype=torch.bool)
    keep[0] = torch.rand(m, generator=torch.Generator().manual_seed(27)) < 0.5
    keep[1, 130:250] = True
    keep[2, -2] = True
    keep = keep.cuda()
    k[~keep], v[~keep] = torch.finfo(dtype).max, float("nan")
    out = torch.full(q.shape, float("nan"), device="cuda", dtype=dtype)
    call(q, k, v, out, key_mask=keep, scale=scale)
    for b in range(3):
        check_exact_products(out[b], q[b], k[b][keep[b]], v[b][keep[b]], scale, dtype)
    assert (out[3] == 0).all()


# ---- what lies in the tensors reaches the result, whole and in parts ---------------------------------------------------

@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [64, 74, 128, 200])
def test_no_number_behind_a_small_probability(d, dtype):
    """A NaN or an infinity among the values of a key whose probability is zero in float32 gives no number, whether the keys are cut into parts or not; other columns do not change."""
    m, n = 3000, 3
    g = torch.Generator().manual_seed(23)
    q = torch.ones(1, n, 1, d, device="cuda", dtype=dtype)
    k = torch.full((1, m, 1, d), -16.0, device="cuda", dtype=dtype)
    k[:, 10] = 16.0
    v = heads(g, 1, m, 1, d, dtype)
    for at in (m - 1, m // 2):
        bad = v.clone()
        bad[0, at, 0, 3], bad[0, at, 0, 5] = float("nan"), float("inf")
        for batch in (1, 256):                                   # a few parts each; 256 units, a whole one each
            qq, kk, vv, clean = (t.expand(batch, *t.shape[1:]) for t in (q, k, bad, v))
            out, want = torch.zeros(batch, n, 1, d, device="cuda", dtype=dtype), torch.zeros(batch, n, 1, d, device="cuda", dtype=dtype)
            p = call(qq, kk, vv, out, scale=1.0)
            assert (svdc.svdcache_attention_workspace_bytes(p) > 0) == (batch == 1)
            call(qq, kk, clean, want, scale=1.0)
            assert out[..., 3].isnan().all() and out[..., 5].isnan().all()
            keep = [c for c in range(d) if c not in (3, 5)]
            assert torch.equal(out[..., keep], want[..., keep]) and torch.isfinite(want).all()


# ---- sizes of the workspace ------------------------------------------------------------------------------------------

@pytest.mark.parametrize("fields,spans", [
    (dict(q=svdc.Heads(-1, 128, 64), o=svdc.Heads(2 ** 41, 128, 64), k_total=-1), dict(q_span=POINTER)),
    (dict(k=svdc.Heads(-1, 128, 64), v=svdc.Heads(2 ** 41, 128, 64), q_total=2 ** 31), dict(k_span=POINTER)),
    (dict(q=svdc.Heads(-1, 128, 64), v=svdc.Heads(-1, 128, 64)), dict(q_span=POINTER, k_span=POINTER)),
    (dict(q_total=-1, k_total=2 ** 40), dict())])
def test_workspace_size_reads_what_the_call_reads(fields, spans):
    """Strides of a sequence where spans are given, and totals where none are, may hold anything."""
    sizes = dict(batch=1, q_rows=1, k_rows=10000)
    need = svdc.svdcache_attention_workspace_bytes(descriptor(**sizes))
    p = descriptor(**sizes, **fields)
    assert need > 0 and svdc.svdcache_attention_workspace_bytes(p) == need
    assert status(p, ws=0, **spans) == -1 and status(p, bytes=need - 1, **spans) == -6


# ---- masks over every kernel -----------------------------------------------------------------------------------------

@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("layout", ["rows", "heads", "odd"])
@pytest.mark.parametrize("d", [8, 64, 72, 96, 128, 200, 256, 33, 74, 130])
@pytest.mark.parametrize("n,m", [(140, 190), (3, 2100)])
def test_masks_at_every_width(n, m, d, layout, dtype):
    """Left-out keys through both ways of loading, at every width that the kernels have, whole and in parts: scattered ones, whole tiles, all but the last, all."""
    batch, h, hk = 5, 2, 1
    g = torch.Generator().manual_seed(24)
    q, k, v = heads(g, batch, n, h, d, dtype, layout), heads(g, batch, m, hk, d, dtype, layout), heads(g, batch, m, hk, d, dtype, layout)
    keep = torch.zeros(batch, m, dtype=torch.bool)
    keep[0] = torch.rand(m, generator=g) < 0.6
    keep[1, 70:131] = True
    keep[2, -1] = True
    keep[4, 64:] = True
    mask = keep.cuda()
    for bad, of in ((float("nan"), k), (float("inf"), v), (torch.finfo(dtype).min, k)):
        before = of[~mask].clone()
        of[~mask] = bad
        out = like(q)
        call(q, k, v, out, key_mask=mask)
        of[~mask] = before
        for b in range(batch):
            check(out[b], q[b], k[b][mask[b]], v[b][mask[b]], d ** -0.5, dtype)
        assert (out[3] == 0).all()


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("layout", ["rows", "odd"])
@pytest.mark.parametrize("d", [40, 72, 128, 136, 75])
@pytest.mark.parametrize("most", [90, 2000])
def test_masked_spans_at_every_width(most, d, layout, dtype):
    """Packed sequences with masks and shared key heads through both ways of loading; rows of no span stay as they were."""
    total = 2 * most + 50
    g = torch.Generator().manual_seed(25)
    q, k, v = heads(g, 1, total, 4, d, dtype, layout)[0], heads(g, 1, total, 2, d, dtype, layout)[0], heads(g, 1, total, 2, d, dtype, layout)[0]
    q_of, k_of = [(0, 3), (3, 0), (5, 77), (90, 1), (100, 40)], [(0, most), (7, 9), (most, most), (most, 1), (2 * most, 50)]
    mask = (torch.rand(total, generator=g) < 0.6).cuda()
    mask[most] = False
    k[~mask] = float("nan")
    v[~mask] = float("inf")
    out = torch.full((total, 4, d), 5.0, device="cuda", dtype=dtype)
    call(q, k, v, out, *(torch.tensor(x, dtype=torch.int32, device="cuda") for x in (q_of, k_of)), mask, q_most=80, k_most=most)
    seen = torch.zeros(total, dtype=torch.bool, device="cuda")
    for (qa, qn), (ka, kn) in zip(q_of, k_of):
        at = torch.arange(ka, ka + kn, device="cuda")
        at = at[mask[at]]
        check(out[qa:qa + qn], q[qa:qa + qn], k[at], v[at], d ** -0.5, dtype)
        seen[qa:qa + qn] = True
    assert (out[~seen] == 5.0).all()
