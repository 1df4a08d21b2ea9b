"""The operators between a block's product for queries, keys and values and the product behind its attention, and their plain forms.

  angles     (cos, sin) of every row's pairs of a rotation with several position axes (time, height, width): axis a turns dim_a / 2 pairs of columns,
             pair i of them by pos[row][a] theta^(-2 i / dim_a).  The axes' pairs follow one another.
  heads      queries and keys, a root-mean-square norm for each head and the rotation of its pairs:  y = x rsqrt(mean(x^2) + eps) gain,
             (a, b) -> (a cos - b sin, a sin + b cos).  Pairs are neighbours (columns 2 j and 2 j + 1) or halves (columns j and pairs + j); columns
             behind the last pair stay.  Values may be taken along (another type, a joint buffer).
  attention  softmax(scale Q K^T) V for each head; several heads of queries may share one of keys and values; sequences of a batch of equal length or
             packed one behind the other (rows that belong to none stay as they were); keys may be left out by a mask.  No key left: zeros.

listed() gives the fixed cases, draw(rng) more of the same ranges; prepare(case, seed) makes what a program holds before the call, run(state) is one
pass, work(case) what it cannot do without, exact(case, seed) the outputs in 64 bits.
"""
import math

import torch

own = False

EPS = 1e-6
_DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
_SIZE = {"f32": 4, "bf16": 2}


def _angles(rows, text, height, width, dims="16,56,56", theta=10000.0, whole=False, name=None):
    return _named({"kind": "angles", "rows": rows, "text": text, "height": height, "width": width, "dims": dims, "theta": theta, "whole": whole}, name)


def _heads(batch, rows, heads, kv_heads, d, x="bf16", out="bf16", norm=True, pairs=-1, halves=False, values=False, front=0, name=None):
    """pairs: of a head's columns that are turned, -1 for all and 0 for none; front: rows of the joint buffers before these (the other stream's)."""
    return _named({"kind": "heads", "batch": batch, "rows": rows, "heads": heads, "kv_heads": kv_heads, "d": d, "x": x, "out": out, "norm": norm,
                   "pairs": d // 2 if pairs < 0 else pairs, "halves": halves, "values": values, "front": front}, name)


def _attention(batch, q, k, heads, kv_heads, d, dtype="bf16", masked=0, q_lengths="", k_lengths="", by_head=False, name=None):
    """masked: leading keys of a sequence (padded text) of which sequence b keeps the first b / batch; q_lengths, k_lengths: packed sequences, with
    q and k the longest; by_head: rows of a head lie together, not heads of a row."""
    return _named({"kind": "attention", "batch": batch, "q": q, "k": k, "heads": heads, "kv_heads": kv_heads, "d": d, "dtype": dtype, "masked": masked,
                   "q_lengths": q_lengths, "k_lengths": k_lengths, "by_head": by_head}, name)


def _named(case, name):
    return {**case, "name": name} if name else case


def listed():
    return [
        # the joint sequence of the image model: 512 text tokens, a grid of 64 x 64
        _angles(4608, 512, 64, 64, name="angles_image"),
        # a long video: frames of 68 x 45 behind 256 text tokens, whole positions
        _angles(119056, 256, 68, 45, theta=256.0, whole=True, name="angles_video"),
        # one token: launches only
        _heads(1, 1, 24, 24, 128, name="heads_token"),
        # one block of the image model, straight from the product's bfloat16 result
        _heads(1, 4608, 24, 24, 128, name="heads_block"),
        # four stacked prompts from a float32 result, into joint buffers behind the text's rows, values too
        _heads(4, 4096, 24, 24, 128, "f32", "bf16", values=True, front=512, name="heads_4_prompts"),
        # nothing a multiple of anything: 16 heads of 72 columns, fewer of keys, halves, part of the columns turned, float32
        _heads(3, 1001, 16, 8, 72, "f32", "f32", pairs=27, halves=True, name="heads_ragged_f32"),
        # one token over a text's keys: launches only
        _attention(1, 1, 512, 24, 24, 128, name="attention_token"),
        # 64 tokens computed anew over all keys of a long video: its keys and values are read once
        _attention(1, 64, 119056, 24, 24, 128, name="attention_few_rows"),
        # one block of the image model
        _attention(1, 4608, 4608, 24, 24, 128, name="attention_block"),
        # four stacked prompts, their text padded to 512 tokens
        _attention(4, 4608, 4608, 24, 24, 128, masked=512, name="attention_4_prompts"),
        # a quarter of the long video, its heads spread over eight cards: the largest
        _attention(1, 29764, 29764, 3, 3, 128, by_head=True, name="attention_video"),
        # packed sequences of any length, one of them empty, narrow heads that share keys, float32
        _attention(5, 1301, 1301, 16, 8, 72, "f32", q_lengths="1301,77,0,1,640", k_lengths="1301,77,0,1,640", name="attention_packed_f32"),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    kind = rng.choice(["angles", "heads", "attention", "attention"])
    if kind == "angles":
        rows = _log(rng, 1, 119056)
        dims = [2 * rng.randint(1, 32) for _ in range(rng.randint(1, 4))]
        return _angles(rows, rng.randint(0, rows), rng.randint(1, 90), rng.randint(1, 90), ",".join(map(str, dims)), rng.choice([256.0, 10000.0, 500000.0]),
                       rng.random() < 0.5)
    d = rng.choice([64, 72, 80, 96, 128, 128, 256, rng.randint(1, 128) * 2])
    kv_heads = _log(rng, 1, max(1, 4096 // d))
    heads = kv_heads * (1 if rng.random() < 0.6 else rng.randint(1, max(1, 6144 // (d * kv_heads))))
    batch = rng.choice([1, 1, 2, 3, 5])
    if kind == "heads":
        x, out = rng.choice([("bf16", "bf16"), ("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32")])
        rows = max(1, min(_log(rng, 1, 119056), 16384 * 9216 // (batch * (heads + 2 * kv_heads) * d)))
        return _heads(batch, rows, heads, kv_heads, d, x, out, rng.random() < 0.8, rng.choice([-1, -1, -1, 0, rng.randint(1, d // 2)]), rng.random() < 0.4,
                      rng.random() < 0.4, rng.choice([0, 0, 77, 512]))
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    q, k = _log(rng, 1, 20000), _log(rng, 1, 20000)
    if rng.random() < 0.6:
        k = q
    elif rng.random() < 0.3:
        q, k = rng.randint(1, 64), _log(rng, 1000, 119056)
    most = 3 * 29764 * 29764 if dtype == "bf16" else 4608 * 4608
    while batch * heads * q * k * max(d, 128) > most * 128:                    # no dearer than the largest
        if batch * heads > 3:
            batch, heads, kv_heads = 1, max(1, heads // kv_heads // 2) * max(1, kv_heads // 2), max(1, kv_heads // 2)
        else:
            q, k = max(1, q * 7 // 8), max(1, k * 7 // 8)
    same = q == k
    if batch > 1 and rng.random() < 0.4:
        q_of = [q] + [rng.choice([0, 1, rng.randint(0, q)]) for _ in range(batch - 1)]
        k_of = q_of if same else [k] + [rng.choice([0, 1, rng.randint(0, k)]) for _ in range(batch - 1)]
        return _attention(batch, q, k, heads, kv_heads, d, dtype, 0, ",".join(map(str, q_of)), ",".join(map(str, k_of)))
    return _attention(batch, q, k, heads, kv_heads, d, dtype, rng.choice([0, 0, rng.randint(0, k - 1), k if batch > 1 else 0]), by_head=rng.random() < 0.3)


# ---- inputs ---------------------------------------------------------------------------------------------------------

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _normal(g, shape, dtype, scale=1.0):
    t = torch.empty(shape, device="cuda", dtype=dtype).normal_(generator=g)
    return t.mul_(scale) if scale != 1.0 else t


def _dims(case):
    return [int(n) for n in case["dims"].split(",")]


def _lengths(text):
    return [int(n) for n in text.split(",")]


def _spans(text):
    lengths = _lengths(text)
    starts = [sum(lengths[:b]) for b in range(len(lengths))]
    return torch.tensor(list(zip(starts, lengths)), device="cuda", dtype=torch.int32)


def _kept(case, b):
    """Leading keys of sequence b that the mask keeps; it leaves out the rest of the first `masked`."""
    return case["masked"] * b // case["batch"]


def prepare(case, seed):
    g = _generator(seed)
    s = {"case": case}
    if case["kind"] == "angles":
        # text tokens at the corner, then frames of height x width, all from an offset that the seed gives (another window of the video); the third
        # and further axes count columns
        n = torch.arange(case["rows"], device="cuda") - case["text"]
        area = case["height"] * case["width"]
        of_axis = [n // area, n % area // case["width"]] + [n % case["width"]] * 2
        pos = torch.stack(of_axis[:len(_dims(case))], 1)
        pos = torch.where((n >= 0)[:, None], pos, torch.zeros_like(pos)) + int(seed) % 997
        s["positions"] = pos.to(torch.int32) if case["whole"] else pos.to(torch.float32) * 0.5
        if own:
            import paper_2601_07396_amd as svdc
            s["p"] = svdc.make_rotary(s["positions"], _dims(case), case["theta"])
            s["table"] = torch.empty(case["rows"], sum(_dims(case)) // 2, 2, device="cuda")
    elif case["kind"] == "heads":
        batch, rows, heads, kv, d = (case[n] for n in ("batch", "rows", "heads", "kv_heads", "d"))
        # the result of the product: queries, keys and values of a row one behind the other; channels of different size; a row of zeros now and then
        x = _normal(g, (batch, rows, (heads + 2 * kv) * d), _DTYPES[case["x"]])
        x *= torch.exp(0.5 * torch.randn(x.shape[-1], device="cuda", generator=g)).to(x.dtype)
        x[:, 96::97] = 0
        s["Q"], s["K"], s["V"] = (t.unflatten(2, (-1, d)) for t in x.split([heads * d, kv * d, kv * d], 2))
        s["gain_q"], s["gain_k"] = (1.0 + 0.2 * torch.randn(d, device="cuda", generator=g) for _ in range(2)) if case["norm"] else (None, None)
        s["table"] = None
        if case["pairs"]:
            angle = 100.0 * torch.rand(rows, case["pairs"], device="cuda", generator=g)
            s["table"] = torch.stack([angle.cos(), angle.sin()], 2)
        if not case["values"]:
            s["V"] = None
        if own:
            import paper_2601_07396_amd as svdc

            def joint(n):
                return torch.empty(batch, case["front"] + rows, n, d, device="cuda", dtype=_DTYPES[case["out"]])[:, case["front"]:]
            s["Qo"], s["Ko"], s["Vo"] = joint(heads), joint(kv), joint(kv) if case["values"] else None
            s["p"] = svdc.make_norm_rotate(s["Q"], s["K"], s["V"], s["Qo"], s["Ko"], s["Vo"], s["table"], layout="halves" if case["halves"] else "neighbours",
                                           norm=case["norm"], eps=EPS)
    else:
        batch, heads, kv, d, dtype = case["batch"], case["heads"], case["kv_heads"], case["d"], _DTYPES[case["dtype"]]

        def rows_of(n, lengths, per_row):
            # packed sequences lie in a buffer with room to spare
            if lengths:
                return _normal(g, (sum(_lengths(lengths)) + 5, per_row, d), dtype)
            if case["by_head"]:
                return _normal(g, (batch, per_row, n, d), dtype).transpose(1, 2)
            return _normal(g, (batch, n, per_row, d), dtype)
        # normed heads: unit columns with gains, some keys that draw much of the attention; values as the product leaves them, beside queries and keys
        s["Q"] = rows_of(case["q"], case["q_lengths"], heads).mul_(1.2)
        s["K"] = rows_of(case["k"], case["k_lengths"], kv).mul_(1.2)
        s["K"][..., ::61, :, :] *= 1.5
        s["V"] = rows_of(case["k"], case["k_lengths"], kv)
        s["V"] += 0.3 * torch.randn(d, device="cuda", generator=g).to(dtype)
        s["q_span"] = _spans(case["q_lengths"]) if case["q_lengths"] else None
        s["k_span"] = _spans(case["k_lengths"]) if case["k_lengths"] else None
        s["key_mask"] = None
        if case["masked"]:
            kept = torch.tensor([_kept(case, b) for b in range(batch)], device="cuda")[:, None]
            key = torch.arange(case["k"], device="cuda")
            s["key_mask"] = ((key < kept) | (key >= case["masked"])).to(torch.uint8)
        if own:
            import paper_2601_07396_amd as svdc
            s["Out"] = torch.zeros(s["Q"].shape, device="cuda", dtype=dtype)
            s["p"] = svdc.make_attention(s["Q"], s["K"], s["V"], s["Out"], s["q_span"], s["k_span"], q_most=case["q"], k_most=case["k"])
            s["workspace"] = svdc.alloc_attention_workspace(s["p"], "cuda")
    return s


# ---- plain forms ----------------------------------------------------------------------------------------------------

def _frequencies(case):
    """Of every pair, and the axis it belongs to."""
    dims = torch.tensor(_dims(case), device="cuda")
    axis = torch.repeat_interleave(torch.arange(len(dims), device="cuda"), dims // 2, output_size=sum(_dims(case)) // 2)
    i = torch.arange(len(axis), device="cuda") - (dims.cumsum(0) - dims)[axis] // 2
    return torch.pow(torch.tensor(case["theta"], device="cuda", dtype=torch.float64), -2.0 * i / dims[axis]), axis


def _turned(x, table, pairs, halves):
    c, s = table[:, None, :, 0], table[:, None, :, 1]
    a, b = (x[..., :pairs], x[..., pairs:2 * pairs]) if halves else (x[..., 0:2 * pairs:2], x[..., 1:2 * pairs:2])
    a, b = a * c - b * s, a * s + b * c
    turned = torch.cat([a, b], -1) if halves else torch.stack([a, b], -1).flatten(-2)
    return torch.cat([turned, x[..., 2 * pairs:]], -1)


def _gathered(t, span, most):
    """Packed rows as a padded batch, and where each of them came from; rows behind a sequence's end come from anywhere."""
    i = torch.arange(most, device=t.device)
    there = i < span[:, 1:]
    at = (span[:, :1] + i).clamp(0, t.shape[0] - 1)
    return t[at], at, there


def run(state):
    case = state["case"]
    if own:
        return _run_own(state, case)
    if case["kind"] == "angles":
        frequency, axis = _frequencies(case)
        angle = state["positions"].to(torch.float64)[:, axis] * frequency
        return torch.stack([angle.cos(), angle.sin()], 2).to(torch.float32)
    if case["kind"] == "heads":
        out = {}
        for name, gain in (("Q", "gain_q"), ("K", "gain_k")):
            x = state[name].to(torch.float32)
            if case["norm"]:
                x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * state[gain]
            if case["pairs"]:
                x = _turned(x, state["table"], case["pairs"], case["halves"])
            out[name] = x.to(_DTYPES[case["out"]])
        if case["values"]:
            out["V"] = state["V"].to(_DTYPES[case["out"]])
        return out
    q, k, v = state["Q"], state["K"], state["V"]
    left_out = None
    if case["q_lengths"]:
        q, at, there = _gathered(q, state["q_span"], case["q"])
    if case["k_lengths"]:
        k, _, key_there = _gathered(k, state["k_span"], case["k"])
        v, _, _ = _gathered(v, state["k_span"], case["k"])
        left_out = ~key_there
    if state["key_mask"] is not None:
        left_out = state["key_mask"] == 0
    q, k, v = (t.transpose(1, 2).to(torch.float32).contiguous() for t in (q, k, v))
    share = case["heads"] // case["kv_heads"]
    k, v = k.repeat_interleave(share, 1), v.repeat_interleave(share, 1)
    scores = torch.matmul(q, k.transpose(2, 3)).mul_(1 / math.sqrt(case["d"]))
    if left_out is not None:
        scores.masked_fill_(left_out[:, None, None, :], -math.inf)
    top = scores.amax(3, keepdim=True)
    scores.sub_(torch.where(top == -math.inf, torch.zeros_like(top), top)).exp_()
    total = scores.sum(3, keepdim=True)
    o = torch.matmul(scores, v) / torch.where(total == 0, torch.ones_like(total), total)
    o = o.transpose(1, 2).to(_DTYPES[case["dtype"]])
    if not case["q_lengths"]:
        return o
    rows = state["Q"].shape[0]
    out = torch.zeros(rows + 1, *o.shape[2:], device=o.device, dtype=o.dtype)      # the last row takes what belongs to no sequence
    out[torch.where(there, at, rows)] = o
    return out[:rows]


def _run_own(s, case):
    import paper_2601_07396_amd as svdc
    if case["kind"] == "angles":
        svdc.svdcache_rotary_table(s["p"], s["positions"], s["table"])
        return s["table"]
    if case["kind"] == "heads":
        svdc.svdcache_norm_rotate(s["p"], s["Q"], s["K"], s["V"], s["gain_q"], s["gain_k"], s["table"], s["Qo"], s["Ko"], s["Vo"])
        return {"Q": s["Qo"], "K": s["Ko"], **({"V": s["Vo"]} if case["values"] else {})}
    svdc.svdcache_attention(s["p"], s["Q"], s["K"], s["V"], s["Out"], s["q_span"], s["k_span"], s["key_mask"], s["workspace"])
    return s["Out"]


def work(case):
    """Each input read once, each output written once; of the attention only what the mask leaves."""
    if case["kind"] == "angles":
        pairs = sum(_dims(case)) // 2
        return {"bytes": case["rows"] * (4 * len(_dims(case)) + 8 * pairs), "flops": 3 * case["rows"] * pairs}
    if case["kind"] == "heads":
        rows, d = case["batch"] * case["rows"], case["d"]
        turned = rows * (case["heads"] + case["kv_heads"]) * d
        moved = turned + (rows * case["kv_heads"] * d if case["values"] else 0)
        small = 8 * case["rows"] * case["pairs"] + (8 * d if case["norm"] else 0)
        return {"bytes": moved * (_SIZE[case["x"]] + _SIZE[case["out"]]) + small, "flops": turned * ((4 if case["norm"] else 0) + (3 if case["pairs"] else 0))}
    q_of = _lengths(case["q_lengths"]) if case["q_lengths"] else [case["q"]] * case["batch"]
    k_of = _lengths(case["k_lengths"]) if case["k_lengths"] else [case["k"] - case["masked"] + _kept(case, b) for b in range(case["batch"])]
    size, d = _SIZE[case["dtype"]], case["d"]
    moved = (2 * sum(q_of) * case["heads"] + 2 * sum(k_of) * case["kv_heads"]) * d * size + (case["batch"] * case["k"] if case["masked"] else 0)
    return {"bytes": moved, "flops": 4 * d * case["heads"] * sum(a * b for a, b in zip(q_of, k_of))}


# ---- 64 bits --------------------------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "angles":
        of_axis, pos = [], s["positions"].double()
        for a, n in enumerate(_dims(case)):
            step = torch.exp(torch.arange(0, n, 2, device="cuda", dtype=torch.float64) * (-math.log(case["theta"]) / n))
            of_axis.append(torch.outer(pos[:, a], step))
        return torch.view_as_real(torch.polar(torch.ones((), device="cuda", dtype=torch.float64), torch.cat(of_axis, 1)))
    if case["kind"] == "heads":
        out = {}
        for name in ("Q", "K"):
            x = s[name].double()
            if case["norm"]:
                x = x / torch.sqrt(x.square().sum(-1, keepdim=True) / case["d"] + EPS) * s["gain_" + name.lower()].double()
            n = case["pairs"]
            if n:
                one, other = (slice(0, n), slice(n, 2 * n)) if case["halves"] else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
                z = torch.complex(x[..., one], x[..., other]) * torch.view_as_complex(s["table"].double())[:, None]
                x = x.clone()
                x[..., one], x[..., other] = z.real, z.imag
            out[name] = x
        if case["values"]:
            out["V"] = s["V"].double()
        return out
    out = torch.zeros(s["Q"].shape, device="cuda", dtype=torch.float64)
    share = case["heads"] // case["kv_heads"]
    q_at, k_at = _spans(case["q_lengths"]).tolist() if case["q_lengths"] else None, _spans(case["k_lengths"]).tolist() if case["k_lengths"] else None
    for b in range(case["batch"]):
        def of(name, at, head):
            t = s[name]
            return (t[b, :, head] if at is None else t[at[b][0]:at[b][0] + at[b][1], head]).double()
        there = None if s["key_mask"] is None else s["key_mask"][b].bool()
        for h in range(case["heads"]):
            q, k, v = of("Q", q_at, h), of("K", k_at, h // share), of("V", k_at, h // share)
            if there is not None:
                k, v = k[there], v[there]
            if not len(q) or not len(k):
                continue
            o = torch.softmax(q @ k.t().contiguous() / math.sqrt(case["d"]), 1) @ v
            if q_at is None:
                out[b, :, h] = o
            else:
                out[q_at[b][0]:q_at[b][0] + q_at[b][1], h] = o
    return out
