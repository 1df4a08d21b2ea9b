"""The operators of a block that runs in 8 bits on the time steps on which its output is computed, and their plain forms.

  norm    the residual stream takes a block's output F (computed or forecast), and the sum's root-mean-square norm goes on in 8 bits:
          H = X + F;  y = H rsqrt(mean(H^2) + eps) gain;  outputs H, optionally Y = y, and Q, scales = y in 8 bits.
  quant   a matrix in 8 bits: one scale for each row and 128 columns (activations) or for each 128 x 128 (weights).
  matmul  Out = act(A W^T + bias) with A and W in 8 bits; Out in float32, bfloat16 or in 8 bits again.
          act: none; "gelu" (tanh form); "swiglu": W holds N gate rows, then N rows that the gates multiply.

8 bits: values in e4m3 (four bits of exponent, three of mantissa, no infinity) times a scale that is a power of two, 2^e for the least e with
amax <= 448 * 2^e (e in -126..126; 0 for a block of zeros).  amax leaves out NaN and counts an infinity as the largest float32; NaN and
infinities become NaN.  A matrix of D columns is held in rows of D rounded up to 128, the tail zero.

listed() gives the fixed cases, draw(rng) more of the same ranges; prepare(case, seed) makes what a program holds before the call, run(state) is one
pass, work(case) what it cannot do without, exact(case, seed) the outputs in 64 bits.
"""
import math

import torch

own = False

EPS = 1e-6
BLOCK = 128
_DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
_SIZE = {"f32": 4, "bf16": 2, "fp8": 1}


def _norm(rows, D, x="bf16", f="bf16", y=False, pad=0, name=None):
    return _named({"kind": "norm", "rows": rows, "D": D, "x": x, "f": f, "y": y, "pad": pad}, name)


def _quant(rows, D, x="bf16", block_rows=1, pad=0, name=None):
    return _named({"kind": "quant", "rows": rows, "D": D, "x": x, "block_rows": block_rows, "pad": pad}, name)


def _matmul(M, N, K, out="bf16", act="none", bias=True, name=None):
    return _named({"kind": "matmul", "M": M, "N": N, "K": K, "out": out, "act": act, "bias": bias}, name)


def _named(case, name):
    return {**case, "name": name} if name else case


def listed():
    return [
        # one token (a conditioning vector, a decode step) at the image model's width: launches only
        _norm(1, 3072, name="norm_token"),
        # one block of the image model (4096 image + 512 text tokens)
        _norm(4608, 3072, name="norm_block"),
        # a long video sequence whose residual stream is kept in float32 while the blocks answer in bfloat16
        _norm(119056, 3072, "f32", "bf16", name="norm_video_f32_stream"),
        # widths that nothing is tuned for, rows inside a wider buffer, the norm wanted unrounded too
        _norm(1001, 1157, "f32", "f32", y=True, pad=3, name="norm_ragged_f32"),
        # the attention's output on its way into the projection behind it
        _quant(4608, 3072, name="quant_rows"),
        # a feed-forward weight as it is loaded
        _quant(12288, 3072, block_rows=128, name="quant_weight"),
        # one token through a wide layer (the six modulation vectors of a block): the weights' bytes are all there is
        _matmul(1, 18432, 3072, name="matmul_token"),
        # 256 text tokens, square layer, float32 result: few tiles, a short product
        _matmul(256, 3072, 3072, "f32", bias=False, name="matmul_text_f32"),
        # 512 text tokens into the feed-forward, which stays in 8 bits
        _matmul(512, 12288, 3072, "fp8", "gelu", name="matmul_text_up"),
        # one image block out of the feed-forward: a long axis of products
        _matmul(4608, 3072, 12288, name="matmul_down"),
        # four stacked prompts into the feed-forward: the largest
        _matmul(18432, 12288, 3072, "fp8", "gelu", name="matmul_up_4_prompts"),
        # nothing a multiple of anything, gated
        _matmul(777, 1921, 1157, "bf16", "swiglu", name="matmul_ragged_gated"),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def _size(rng, low, high):
    """Spread over the logarithm; every second one a multiple of 64, as widths mostly are, where that stays in the range."""
    n = _log(rng, low, high)
    return n if rng.random() < 0.5 or n < 128 else n // 64 * 64


def draw(rng):
    kind = rng.choice(["norm", "quant", "matmul", "matmul"])
    if kind == "norm":
        D = _size(rng, 64, 12288)
        rows = _log(rng, 1, min(119056, 119056 * 3072 // D))
        x, f = rng.choice([("bf16", "bf16"), ("f32", "f32"), ("f32", "bf16")])
        return _norm(rows, D, x, f, rng.random() < 0.3, rng.choice([0, 0, 8, 3]))
    if kind == "quant":
        D = _size(rng, 64, 12288)
        rows = _log(rng, 1, min(119056, 119056 * 3072 // D))
        return _quant(rows, D, rng.choice(["bf16", "f32"]), rng.choice([1, 128]), rng.choice([0, 0, 8, 3]))
    M, N, K = _log(rng, 1, 18432), _size(rng, 64, 12288), _size(rng, 64, 12288)
    M = min(M, max(1, 18432 * 12288 * 3072 // (N * K)))
    act = rng.choice(["none", "none", "gelu", "swiglu"])
    return _matmul(M, max(16, N // 2) if act == "swiglu" else N, K, rng.choice(["f32", "bf16", "bf16", "fp8"]), act, rng.random() < 0.5)


# ---- inputs ---------------------------------------------------------------------------------------------------------

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _activations(g, rows, D, dtype, pad, scale):
    """Rows of a residual stream: channels of different size, a few of them large, and now and then a row of zeros (padding); inside a
    buffer of D + pad columns."""
    size = torch.exp(0.5 * torch.randn(D, device="cuda", generator=g))
    size = torch.where(torch.rand(D, device="cuda", generator=g) < 0.004, 20.0 * size, size)
    x = torch.empty(rows, D + pad, device="cuda", dtype=dtype)
    x.normal_(generator=g)
    x[:, :D] *= (scale * size).to(dtype)
    x[96::97] = 0
    return x[:, :D]


def prepare(case, seed):
    g = _generator(seed)
    s = {"case": case}
    if case["kind"] == "norm":
        rows, D, dtype = case["rows"], case["D"], _DTYPES[case["x"]]
        s["X"] = _activations(g, rows, D, dtype, case["pad"], 2.0)
        s["F"] = _activations(g, rows, D, _DTYPES[case["f"]], 0, 0.5)
        s["gain"] = 1.0 + 0.2 * torch.randn(D, device="cuda", generator=g)
        if own:
            import paper_2601_07396_amd as svdc
            s["H"] = torch.empty(rows, D, device="cuda", dtype=dtype)
            s["Y"] = torch.empty_like(s["H"]) if case["y"] else None
            s["Q"], s["scales"] = svdc.alloc_q8(rows, D, "cuda")
            s["p"] = svdc.make_norm8(s["X"], s["F"], s["H"], s["Y"], eps=EPS)
    elif case["kind"] == "quant":
        rows, D = case["rows"], case["D"]
        s["X"] = _activations(g, rows, D, _DTYPES[case["x"]], case["pad"], 1.0 if case["block_rows"] == 1 else 0.02)
        if own:
            import paper_2601_07396_amd as svdc
            s["Q"], s["scales"] = svdc.alloc_q8(rows, D, "cuda", case["block_rows"])
            s["p"] = svdc.make_quant8(s["X"], case["block_rows"])
    else:
        M, N, K = case["M"], case["N"], case["K"]
        wide = 2 * N if case["act"] == "swiglu" else N
        s["A"], s["A_scales"] = _quantize(_activations(g, M, K, torch.float32, 0, 1.0))
        W = torch.randn(wide, K, device="cuda", generator=g) / math.sqrt(K)
        s["W"], s["W_scales"] = _quantize(W, BLOCK)
        s["bias"] = 0.1 * torch.randn(wide, device="cuda", generator=g) if case["bias"] else None
        if own:
            import paper_2601_07396_amd as svdc
            out = case["out"]
            s["p"] = svdc.make_matmul8(M, N, K, torch.float8_e4m3fn if out == "fp8" else _DTYPES[out], case["act"])
            s["Out_scales"] = None
            if out == "fp8":
                s["Out"], s["Out_scales"] = svdc.alloc_q8(M, N, "cuda")
            else:
                s["Out"] = torch.empty(M, N, device="cuda", dtype=_DTYPES[out])
            s["workspace"] = svdc.alloc_matmul8_workspace(s["p"], "cuda")
    return s


# ---- plain forms ----------------------------------------------------------------------------------------------------

def _up(n, m):
    return (n + m - 1) // m * m


def _quantize(v, block_rows=1):
    """v in e4m3 [rows, D rounded up to 128] and its scales as e8m0 [blocks of rows, D / 128 rounded up to 4]."""
    rows, D = v.shape
    tall, wide = _up(rows, block_rows), _up(D, BLOCK)
    full = torch.zeros(tall, wide, device=v.device, dtype=torch.float32)
    full[:rows, :D] = v
    blocks = full.view(tall // block_rows, block_rows, wide // BLOCK, BLOCK)
    size = blocks.abs()
    amax = torch.where(size.isnan(), 0.0, size).amax(dim=(1, 3)).clamp(max=torch.finfo(torch.float32).max)
    mantissa, exponent = torch.frexp(amax)
    e = exponent - 9 + (mantissa > 0.875)                      # 448 = 0.875 * 2^9
    e = torch.where(amax == 0, torch.zeros_like(e), e).clamp(-126, 126)
    inverse = ((127 - e) << 23).to(torch.int32).view(torch.float32)
    q = (blocks * inverse[:, None, :, None]).view(tall, wide)[:rows].to(torch.float8_e4m3fn)
    scales = torch.full((tall // block_rows, _up(wide // BLOCK, 4)), 127, device=v.device, dtype=torch.uint8)
    scales[:, :wide // BLOCK] = (e + 127).to(torch.uint8)
    return q, scales.view(torch.float8_e8m0fnu)


def _values(q, scales, D, block_rows=1):
    rows = q.shape[0]
    s = scales.to(torch.float32).repeat_interleave(block_rows, 0)[:rows].repeat_interleave(BLOCK, 1)[:, :D]
    return q[:, :D].to(torch.float32) * s


def _activated(z, act, N):
    if act == "gelu":
        return z / (1 + torch.exp(-2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))
    if act == "swiglu":
        return z[:, :N] / (1 + torch.exp(-z[:, :N])) * z[:, N:]
    return z


def _eight(q, scales, rows, D, block_rows=1):
    """The 8-bit outputs without their padding."""
    return {"Q": q[:, :D], "scales": scales[:, :_up(D, BLOCK) // BLOCK]}


def run(state):
    case = state["case"]
    if own:
        return _run_own(state, case)
    if case["kind"] == "norm":
        h = state["X"].to(torch.float32) + state["F"].to(torch.float32)
        y = h * torch.rsqrt((h * h).mean(dim=1, keepdim=True) + EPS) * state["gain"]
        dtype = _DTYPES[case["x"]]
        out = {"H": h.to(dtype), **_eight(*_quantize(y), case["rows"], case["D"])}
        if case["y"]:
            out["Y"] = y.to(dtype)
        return out
    if case["kind"] == "quant":
        return _eight(*_quantize(state["X"].to(torch.float32), case["block_rows"]), case["rows"], case["D"], case["block_rows"])
    K = case["K"]
    z = _values(state["A"], state["A_scales"], K) @ _values(state["W"], state["W_scales"], K, BLOCK).T
    if state["bias"] is not None:
        z = z + state["bias"]
    z = _activated(z, case["act"], case["N"])
    if case["out"] == "fp8":
        return _eight(*_quantize(z), case["M"], case["N"])
    return {"Out": z.to(_DTYPES[case["out"]])}


def _run_own(s, case):
    import paper_2601_07396_amd as svdc
    if case["kind"] == "norm":
        svdc.svdcache_rms_norm8(s["p"], s["X"], s["F"], s["gain"], s["H"], s["Y"], s["Q"], s["scales"])
        out = {"H": s["H"], **_eight(s["Q"], s["scales"], case["rows"], case["D"])}
        if case["y"]:
            out["Y"] = s["Y"]
        return out
    if case["kind"] == "quant":
        svdc.svdcache_quantize8(s["p"], s["X"], s["Q"], s["scales"])
        return _eight(s["Q"], s["scales"], case["rows"], case["D"], case["block_rows"])
    svdc.svdcache_matmul8(s["p"], s["A"], s["A_scales"], s["W"], s["W_scales"], s["bias"], s["Out"], s["Out_scales"], s["workspace"])
    if case["out"] == "fp8":
        return _eight(s["Out"], s["Out_scales"], case["M"], case["N"])
    return {"Out": s["Out"]}


def work(case):
    """Each input read once, each output written once; scales count one byte each, the padding does not count."""
    if case["kind"] == "norm":
        n = case["rows"] * case["D"]
        each = 2 * _SIZE[case["x"]] + _SIZE[case["f"]] + (_SIZE[case["x"]] if case["y"] else 0) + 1
        return {"bytes": n * each + 4 * case["D"] + case["rows"] * _up(case["D"], BLOCK) // BLOCK, "flops": 6 * n}
    if case["kind"] == "quant":
        n = case["rows"] * case["D"]
        scales = _up(case["rows"], case["block_rows"]) // case["block_rows"] * (_up(case["D"], BLOCK) // BLOCK)
        return {"bytes": n * (_SIZE[case["x"]] + 1) + scales, "flops": 2 * n}
    M, N, K = case["M"], case["N"], case["K"]
    wide = 2 * N if case["act"] == "swiglu" else N
    blocks = _up(K, BLOCK) // BLOCK
    moved = (M + wide) * K + (M + _up(wide, BLOCK) // BLOCK) * blocks + M * N * _SIZE[case["out"]]
    if case["out"] == "fp8":
        moved += M * (_up(N, BLOCK) // BLOCK)
    return {"bytes": moved + (4 * wide if case["bias"] else 0), "flops": 2 * M * wide * K}


# ---- 64 bits --------------------------------------------------------------------------------------------------------

def _exact_eight(v, block_rows, with_scales):
    """What the rounding to e4m3 starts from, and the scales.  Where v comes out of sums, a block whose amax lies within a rounding of the
    step may take either scale: then there is no one value for them."""
    rows, D = v.shape
    tall, wide = _up(rows, block_rows), _up(D, BLOCK)
    padded = torch.nn.functional.pad(v, (0, wide - D, 0, tall - rows))
    top = padded.abs().reshape(tall // block_rows, block_rows, wide // BLOCK, BLOCK).amax(3).amax(1)
    e = torch.ceil(torch.log2(top / 448))
    e = torch.where(top > 448 * torch.exp2(e), e + 1, e)       # the logarithm may round across a power of two
    e = torch.where(top <= 448 * torch.exp2(e - 1), e - 1, e)
    scale = torch.where(top > 0, torch.exp2(e.clamp(-126, 126)), torch.ones_like(top))
    each = scale.repeat_interleave(block_rows, 0)[:rows].repeat_interleave(BLOCK, 1)[:, :D]
    return {"Q": v / each, "scales": scale if with_scales else None}


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "norm":
        h = s["X"].double() + s["F"].double()
        y = h / torch.sqrt(h.square().sum(1, keepdim=True) / case["D"] + EPS) * s["gain"].double()
        out = {"H": h, **_exact_eight(y, 1, False)}
        if case["y"]:
            out["Y"] = y
        return out
    if case["kind"] == "quant":
        return _exact_eight(s["X"].double(), case["block_rows"], True)
    M, N, K = case["M"], case["N"], case["K"]
    blocks = _up(K, BLOCK) // BLOCK
    wide = 2 * N if case["act"] == "swiglu" else N

    def rows_of(q, scales, each):
        n = q.shape[0]
        v = q.double().reshape(n, blocks, BLOCK)
        which = torch.arange(n, device=v.device) // each
        return (v * scales.double()[which, :blocks, None]).reshape(n, blocks * BLOCK)[:, :K]

    z = torch.matmul(rows_of(s["A"], s["A_scales"], 1), rows_of(s["W"], s["W_scales"], BLOCK).t())
    if case["bias"]:
        z += s["bias"].double()
    if case["act"] == "gelu":
        z = 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    elif case["act"] == "swiglu":
        z = z[:, :N] * torch.sigmoid(z[:, :N]) * z[:, N:wide]
    return _exact_eight(z, 1, False) if case["out"] == "fp8" else {"Out": z}
