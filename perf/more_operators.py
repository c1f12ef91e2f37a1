"""What is measured of the operators around the block-scaled product: the RMS norm that writes its operands, and products grouped by expert.

A model's layer in 8 bits begins with the norm of its input, to which the residual stream is added, and whose answer is the operand of
the next products: E4M3 with a scale for each block of 128, along the channels and, while training, along the tokens.  Where a layer has
experts, each row of its operand meets the weights of one of them: rows lie in the order of the experts, in segments of any length.

`own` False: the operators written out in elementary torch operations in 32 bits.  `own` True: the calls a user makes.
"""
import math

import torch

own = False

E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu
EPS = 1e-6


# ----------------------------------------------------------------------------------------------------------------------
# The cases.
# ----------------------------------------------------------------------------------------------------------------------
def listed():
    return [
        # the next token of one sequence, before a layer's projections: latency
        dict(name="norm_one_token", op="norm", rows=1, cols=4096, dtype="bf16", residual="bf16", weight="bf16", kind="rows"),
        # prompts packed to an odd length, a ragged width, a residual stream that is kept in 32 bits
        dict(name="norm_ragged", op="norm", rows=5003, cols=4100, dtype="bf16", residual="f32", weight="f32", kind="both"),
        # a training batch, wanted along the channels (forward) and along the tokens (weight gradient)
        dict(name="norm_training_both", op="norm", rows=16384, cols=4096, dtype="bf16", residual="bf16", weight="bf16", kind="both"),
        # its gradient, joined with the residual stream's
        dict(name="norm_gradient", op="norm_gradient", rows=16384, cols=4096, dtype="bf16", grad="bf16", weight="bf16", add=True),
        # a short batch of a wide model with a stream in 32 bits
        dict(name="norm_gradient_wide", op="norm_gradient", rows=733, cols=16384, dtype="f32", grad="bf16", weight="f32", add=True),
        # one token and its eight experts of 64: the weights of eight experts are read
        dict(name="experts_one_token", op="experts", way="forward", rows=8, experts=64, inputs=2048, outputs=4096, spread="once", out="bf16", add=False),
        # a serving batch of 61 tokens with four experts each
        dict(name="experts_decode", op="experts", way="forward", rows=244, experts=32, inputs=4096, outputs=2048, spread="uneven", out="bf16", add=False),
        # prompts, or the forward pass of a training batch
        dict(name="experts_forward", op="experts", way="forward", rows=16384, experts=16, inputs=4096, outputs=4096, spread="uneven", out="bf16", add=False),
        # gradient of the inputs of ragged layers
        dict(name="experts_input_gradient", op="experts", way="dgrad", rows=9001, experts=24, inputs=2056, outputs=4100, spread="uneven", out="bf16", add=False),
        # gradient of the weights, added to 32-bit gradient buffers over micro-batches
        dict(name="experts_weight_gradient", op="experts", way="wgrad", rows=16384, experts=16, inputs=2048, outputs=4096, spread="uneven", out="f32", add=True),
        # output gradients in the order of the experts, wanted along the channels and, expert by expert, along the tokens
        dict(name="experts_quantise", op="segments", rows=16384, cols=4096, experts=16, dtype="bf16", spread="uneven"),
        # a short batch of a ragged layer with 32-bit activations, many experts
        dict(name="experts_quantise_ragged", op="segments", rows=1003, cols=2055, experts=60, dtype="f32", spread="even"),
    ]


def _spread(rng, low, high):
    """A whole number whose logarithm is spread evenly."""
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high + 1)))))))


def draw(rng):
    op = rng.choice(["norm", "norm", "norm_gradient", "experts", "experts", "experts", "segments"])
    if op in ("norm", "norm_gradient"):
        rows = _spread(rng, 1, 16384)
        cols = _spread(rng, 100, min(16384, 16384 * 4096 // rows))
        dtype = rng.choice(["bf16", "f32"])
        case = dict(op=op, rows=rows, cols=cols, dtype=dtype, weight=rng.choice(["bf16", "f32"]))
        if op == "norm":
            return dict(case, residual=rng.choice(["none", "f32", dtype]), kind=rng.choice(["rows", "cols", "both"]))
        return dict(case, grad=rng.choice(["bf16", "f32"]), add=rng.random() < 0.6)
    experts = _spread(rng, 2, 64)
    spread = rng.choice(["uneven", "uneven", "even"])
    if op == "segments":
        rows = _spread(rng, 1, 16384)
        return dict(op=op, rows=rows, cols=_spread(rng, 100, 4096), experts=experts, dtype=rng.choice(["bf16", "f32"]), spread=spread)
    way = rng.choice(["forward", "forward", "dgrad", "wgrad"])
    rows = _spread(rng, 1, 16384)
    inputs = _spread(rng, 200, 4096)
    outputs = _spread(rng, 200, min(8192, 4096 * 4096 * 24 // (experts * inputs), 16384 * 4096 * 4096 // (rows * inputs)))
    out = rng.choice(["bf16", "f32"]) if way != "wgrad" else "f32"
    return dict(op=op, way=way, rows=rows, experts=experts, inputs=inputs, outputs=outputs, spread=spread, out=out, add=way == "wgrad" and rng.random() < 0.5)


# ----------------------------------------------------------------------------------------------------------------------
# Inputs.
# ----------------------------------------------------------------------------------------------------------------------
def _up(n, m):
    return -(-n // m) * m


def _dtype(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _activations(g, rows, cols, size):
    """Rows of unlike size and a few channels that stand out, as activations and their gradients have."""
    x = torch.randn(rows, cols, generator=g, device="cuda")
    x.mul_(torch.randn(rows, 1, generator=g, device="cuda").mul_(0.5).exp_().mul_(size))
    loud = torch.rand(1, cols, generator=g, device="cuda") < 0.01
    return x.mul_(torch.where(loud, 20.0, 1.0))


def _padded(codes):
    """Codes in rows of a multiple of 16 bytes."""
    out = torch.zeros(*codes.shape[:-1], _up(codes.shape[-1], 16), dtype=torch.uint8, device="cuda")
    out[..., :codes.shape[-1]] = codes.view(torch.uint8)
    return out


def _counts(case, g):
    """Rows of each expert: some popular, some without any; a few rows behind the last segment belong to nobody (a padded batch)."""
    rows, n = case["rows"], case["experts"]
    if case["spread"] == "once":   # one row for each of as many experts
        counts = torch.zeros(n, dtype=torch.int64)
        counts[torch.randperm(n, generator=g)[:rows]] = 1
        return counts
    used = rows - (rows // 40 if case["spread"] == "uneven" else 0)
    taste = torch.randn(n, generator=g).mul_(0.7 if case["spread"] == "uneven" else 0.02).exp_()
    if case["spread"] == "uneven" and n >= 8:
        taste[torch.randperm(n, generator=g)[:n // 8]] = 0.0
    at = (taste.double().cumsum(0) / taste.double().sum() * used).round().long()
    return torch.diff(at, prepend=torch.zeros(1, dtype=torch.int64))


def _blocks(rows, experts):
    """Blocks of 128 rows that segments may take where each begins a block of its own."""
    return (rows + 127 * min(experts, rows)) // 128


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    s = dict(case=case)
    op = case["op"]
    if op in ("norm", "norm_gradient"):
        rows, cols = case["rows"], case["cols"]
        s["w"] = torch.randn(cols, generator=g, device="cuda").mul_(0.2).add_(1.0).to(_dtype(case["weight"]))
        x = _activations(g, rows, cols, 1.0)
        if op == "norm":
            s["x"] = x.to(_dtype(case["dtype"]))
            s["residual"] = None if case["residual"] == "none" else _activations(g, rows, cols, 2.0).to(_dtype(case["residual"]))
            if own:  # the buffers that a program reuses from step to step
                from paper_2608_06812_b200 import lowbit
                s["total"] = None if s["residual"] is None else torch.empty_like(s["residual"])
                s["root"] = torch.empty(rows, device="cuda")
                s["by_rows"] = lowbit.Fp8Matrix.empty(rows, cols, lowbit.ROWS) if case["kind"] != "cols" else None
                s["by_cols"] = lowbit.Fp8Matrix.empty(rows, cols, lowbit.COLS) if case["kind"] != "rows" else None
        else:
            s["total"] = x.to(_dtype(case["dtype"]))
            s["root"] = _plain_root(s["total"].float())
            s["dy"] = _activations(g, rows, cols, 1e-3).to(_dtype(case["grad"]))
            s["dtotal"] = _activations(g, rows, cols, 1e-3).to(_dtype(case["dtype"])) if case["add"] else None
        return s
    counts = _counts(case, torch.Generator().manual_seed(int(seed)))
    s["most"] = int(counts.max())
    s["offsets"] = torch.cat([torch.zeros(1, dtype=torch.int64), counts.cumsum(0)]).to("cuda", torch.int32)
    if op == "segments":
        rows, cols = case["rows"], case["cols"]
        s["x"] = _activations(g, rows, cols, 1e-3).to(_dtype(case["dtype"]))
        if own:
            from paper_2608_06812_b200 import lowbit
            s["by_rows"] = lowbit.Fp8Matrix.empty(rows, cols, lowbit.ROWS)
            s["by_cols"] = lowbit.Fp8Segments.empty(rows, cols, case["experts"])
            for q in (s["by_rows"], s["by_cols"]):  # what no segment covers stays as it is
                q.codes.zero_()
                q.scales.fill_(127)
        return s
    t, i, o, n = case["rows"], case["inputs"], case["outputs"], case["experts"]
    if case["way"] == "wgrad":
        for name, width, size in (("a", o, 1e-3), ("b", i, 1.0)):
            codes, scales = _by_segments(_activations(g, t, width, size), s["offsets"])
            s[name], s[name + "_scales"] = _padded(codes), _pack(scales, True)
        s["out"] = torch.zeros(n, o, _up(i, 8), device="cuda")[:, :, :i]
        if case["add"]:
            s["out"].copy_(torch.randn(n, o, i, generator=g, device="cuda"))
        if own:
            from paper_2608_06812_b200 import lowbit
            s["left"] = lowbit.Fp8Segments(s["a"], s["a_scales"], t, o, n)
            s["right"] = lowbit.Fp8Segments(s["b"], s["b_scales"], t, i, n)
        return s
    width = i if case["way"] == "forward" else o
    codes, scales = _quantise(_activations(g, t, width, 1.0 if case["way"] == "forward" else 1e-3), "rows")
    s["a"], s["a_scales"] = _padded(codes), _pack(scales, False)
    w = torch.randn(n, o, i, generator=g, device="cuda").mul_(0.02)
    w *= torch.randn(n, 1, 1, generator=g, device="cuda").mul_(0.3).exp_()
    codes, s["b_scales"] = _quantise_experts(w)
    s["b"] = _padded(codes)
    del w, codes
    m = o if case["way"] == "forward" else i
    s["out"] = torch.zeros(t, _up(m, 8), dtype=_dtype(case["out"]), device="cuda")[:, :m]
    if own:
        from paper_2608_06812_b200 import lowbit
        s["left"] = lowbit.Fp8Matrix(s["a"], s["a_scales"], t, width, lowbit.ROWS)
        s["right"] = lowbit.Fp8Experts(s["b"], s["b_scales"], o, i)
    return s


# ----------------------------------------------------------------------------------------------------------------------
# The plain forms.
# ----------------------------------------------------------------------------------------------------------------------
def _scale_codes(amax):
    """Codes c of the scales 2^(c - 127): the least power of two, not under 2^-127, that brings amax to 448 or less; 1 for a block of zeros."""
    bits = amax.view(torch.int32)
    c = ((bits >> 23) - 8 + ((bits & 0x7FFFFF) > 0x600000).to(torch.int32)).clamp_(min=0)
    return torch.where(amax > 0, c, 127).to(torch.uint8)


def _power(c, negative=False):
    """2^(c - 127), or 2^(127 - c), from codes."""
    c = c.to(torch.int32)
    if negative:
        c = 254 - c
    return torch.where(c > 0, c << 23, 1 << 22).view(torch.float32)


def _quantise(x, kind):
    """(codes as torch's 8-bit type, scale codes [lines or tiles][blocks]) of `x` by rows, by columns or by tiles."""
    rows, cols = x.shape
    br, bc = {"rows": (1, 128), "cols": (128, 1), "tiles": (128, 128)}[kind]
    f = torch.nn.functional.pad(x.float(), (0, _up(cols, bc) - cols, 0, _up(rows, br) - rows))
    f = f.view(f.shape[0] // br, br, f.shape[1] // bc, bc)
    size = f.abs()
    c = _scale_codes(torch.where(torch.isfinite(size), size, 0.0).amax((1, 3)))
    q = (f * _power(c, True)[:, None, :, None]).to(E4M3)
    return q.view(f.shape[0] * br, f.shape[2] * bc)[:rows, :cols], c


def _quantise_experts(w):
    """The same of [experts, rows, cols] by tiles that begin with each expert."""
    n, rows, cols = w.shape
    f = torch.nn.functional.pad(w, (0, 0, 0, _up(rows, 128) - rows)).view(n * _up(rows, 128), cols)
    q, c = _quantise(f, "tiles")
    return q.reshape(n, -1, cols)[:, :rows], c.view(n, -1, c.shape[1])


def _pack(c, cols):
    """Scale codes [lines][blocks] ([blocks][lines] if `cols`) as the words of four blocks that the product reads: [groups][lines][4]."""
    c = c if cols else c.T
    blocks, lines = c.shape
    full = torch.full((_up(blocks, 4), lines), 127, dtype=torch.uint8, device=c.device)
    full[:blocks] = c
    return full.view(-1, 4, lines).permute(0, 2, 1).contiguous()


def _unpack(words, blocks):
    """The inverse of _pack: [blocks][lines]."""
    return words.permute(0, 2, 1).reshape(-1, words.shape[1])[:blocks]


def _values(codes, cols, scales, lines, blocks):
    """Codes times scales [.., line blocks][column blocks], each for `lines` x `blocks` of them, in 32 bits."""
    f = codes.view(E4M3)[..., :cols].float()
    full = scales.repeat_interleave(lines, -2)[..., :codes.shape[-2], :].repeat_interleave(blocks, -1)[..., :cols]
    return f * full


def _expert_of(at, starts, ends):
    """The expert whose range covers each of `at`, where in that range it is, and whether there is one."""
    e = torch.searchsorted(ends.contiguous(), at, right=True)
    inside = e < ends.numel()
    e = e.clamp(max=ends.numel() - 1)
    local = at - starts[e]
    return e, local, inside & (local >= 0)


def _segment_starts(offsets):
    """Rows at which segments begin and end once each begins a block of 128."""
    ends = ((torch.diff(offsets.long()) + 127) // 128).cumsum(0) * 128
    return torch.cat([ends.new_zeros(1), ends[:-1]]), ends


def _by_segments(x, offsets):
    """_quantise by columns, with blocks of 128 rows that begin with each segment: (codes [blocks * 128, cols], scale codes [blocks][cols])."""
    rows, cols = x.shape
    starts, ends = _segment_starts(offsets)
    at = torch.arange(_blocks(rows, offsets.numel() - 1) * 128, device=x.device)
    e, local, inside = _expert_of(at, starts, ends)
    source = offsets.long()[e] + local
    inside &= source < offsets.long()[e + 1]
    return _quantise(torch.where(inside[:, None], x.float()[source.clamp(0, rows - 1)], 0.0), "cols")


def _plain_root(h):
    return torch.rsqrt(h.square().mean(1) + EPS)


def _plain_norm(s):
    h = s["x"]
    if s["residual"] is not None:
        h = (s["x"].float() + s["residual"].float()).to(s["residual"].dtype)
    f = h.float()
    root = _plain_root(f)
    y = f * root[:, None] * s["w"].float()
    kind = s["case"]["kind"]
    return _norm_answer(s, h, root, [(*_quantise(y, k), k == "cols") for k in (("rows", "cols") if kind == "both" else (kind,))])


def _norm_answer(s, total, root, forms):
    forms = [dict(codes=q, scales=_pack(c, cols).view(E8M0)) for q, c, cols in forms]
    return dict(total=None if s["residual"] is None else total, root=root, forms=forms)


def _plain_norm_gradient(s):
    h, root, dy = s["total"].float(), s["root"][:, None], s["dy"].float()
    g = dy * s["w"].float()
    dx = root * g - h * (root * root * root) * (g * h).mean(1, keepdim=True)
    if s["dtotal"] is not None:
        dx += s["dtotal"].float()
    return dict(dx=dx.to(s["total"].dtype), dw=(dy * (h * root)).sum(0))


def _plain_experts(s):
    case, offsets = s["case"], s["offsets"].long()
    local = torch.arange(s["most"], device="cuda")
    inside = (local < torch.diff(offsets)[:, None])[..., None]
    if case["way"] == "wgrad":
        at = _segment_starts(offsets)[0][:, None] + local
        a, b = (_values(s[n], w, _power(_unpack(s[n + "_scales"], s[n].shape[0] // 128)), 128, 1) for n, w in (("a", case["outputs"]), ("b", case["inputs"])))
        at = at.clamp(max=a.shape[0] - 1)
        c = torch.bmm(torch.where(inside, a[at], 0.0).transpose(1, 2), torch.where(inside, b[at], 0.0))
        return s["out"].add_(c) if case["add"] else c.to(_dtype(case["out"]))
    width = case["inputs"] if case["way"] == "forward" else case["outputs"]
    a = _values(s["a"], width, _power(_unpack(s["a_scales"], _up(width, 128) // 128)).T, 1, 128)
    w = _values(s["b"], case["inputs"], _power(s["b_scales"]), 128, 128)
    a = torch.where(inside, a[(offsets[:-1, None] + local).clamp(max=case["rows"] - 1)], 0.0)
    c = torch.bmm(a, w.transpose(1, 2) if case["way"] == "forward" else w)
    e, place, covered = _expert_of(torch.arange(case["rows"], device="cuda"), offsets[:-1], offsets[1:])
    c = c[e, place.clamp(0, s["most"] - 1)].to(_dtype(case["out"]))
    return torch.where(covered[:, None], c, s["out"])


def _plain_segments(s):
    offsets, rows = s["offsets"], s["case"]["rows"]
    q, c = _quantise(s["x"], "rows")
    covered = (torch.arange(rows, device="cuda") < offsets[-1])[:, None]
    q = torch.where(covered, q.view(torch.uint8), 0).view(E4M3)
    by_rows = dict(codes=q, scales=_pack(torch.where(covered, c, 127), False).view(E8M0))
    q, c = _by_segments(s["x"], offsets)
    return [by_rows, dict(codes=q, scales=_pack(c, True).view(E8M0))]


# ----------------------------------------------------------------------------------------------------------------------
# One pass.
# ----------------------------------------------------------------------------------------------------------------------
def run(state):
    s = state
    case, op = s["case"], s["case"]["op"]
    if not own:
        return {"norm": _plain_norm, "norm_gradient": _plain_norm_gradient, "experts": _plain_experts, "segments": _plain_segments}[op](s)
    from paper_2608_06812_b200 import lowbit
    if op == "norm":
        lowbit.rms_norm(s["x"], s["w"], s["residual"], eps=EPS, rows=s["by_rows"], cols=s["by_cols"], total=s["total"], root=s["root"])
        return dict(total=s["total"], root=s["root"], forms=[dict(codes=q.values8(), scales=q.scales.view(E8M0)) for q in (s["by_rows"], s["by_cols"]) if q is not None])
    if op == "norm_gradient":
        dx, dw = lowbit.rms_norm_backward(s["dy"], s["total"], s["root"], s["w"], s["dtotal"])
        return dict(dx=dx, dw=dw)
    if op == "experts":
        return lowbit.grouped_matmul(s["left"], s["right"], s["offsets"], out=s["out"], over_rows=case["way"] == "dgrad", accumulate=case["add"])
    lowbit.quantize_segments(s["x"], s["offsets"], rows=s["by_rows"], cols=s["by_cols"])
    return [dict(codes=q.values8(), scales=q.scales.view(E8M0)) for q in (s["by_rows"], s["by_cols"])]


def work(case):
    size = lambda d: {"f32": 4, "bf16": 2, "none": 0}[d]  # noqa: E731
    if case["op"] in ("norm", "norm_gradient"):
        n = case["rows"] * case["cols"]
        if case["op"] == "norm":
            each = size(case["dtype"]) + 2 * size(case["residual"]) + (2 if case["kind"] == "both" else 1) * (1 + 1 / 128)
            return dict(bytes=n * each + case["cols"] * size(case["weight"]) + 4 * case["rows"], flops=8 * n)
        each = size(case["grad"]) + size(case["dtype"]) * (3 if case["add"] else 2)
        return dict(bytes=n * each + case["cols"] * (size(case["weight"]) + 4) + 4 * case["rows"], flops=12 * n)
    counts = _counts(case, torch.Generator().manual_seed(1))
    rows, active = int(counts.sum()), int((counts > 0).sum())
    if case["op"] == "segments":
        n = rows * case["cols"]
        return dict(bytes=n * (size(case["dtype"]) + 2 + 2 / 128), flops=3 * n)
    i, o = case["inputs"], case["outputs"]
    if case["way"] == "wgrad":
        sums = case["experts"] * o * i * size(case["out"]) * (2 if case["add"] else 1)
        return dict(bytes=rows * (i + o) * (1 + 1 / 128) + sums, flops=2 * rows * i * o)
    k, m = (i, o) if case["way"] == "forward" else (o, i)
    return dict(bytes=rows * k * (1 + 1 / 128) + active * i * o + rows * m * size(case["out"]), flops=2 * rows * i * o)


# ----------------------------------------------------------------------------------------------------------------------
# What the outputs are, in 64 bits, from the definitions.
# ----------------------------------------------------------------------------------------------------------------------
def _e4m3_values():
    """The values of the codes 0 .. 127: sign clear, four bits of exponent (bias 7), three of fraction, 127 not a number."""
    v = [(f / 8 * 2.0 ** -6) if e == 0 else (1 + f / 8) * 2.0 ** (e - 7) for e in range(16) for f in range(8)]
    v[127] = math.nan
    return torch.tensor(v, dtype=torch.float64, device="cuda")


def _nearest(x):
    """The nearest of those values, ties to the even code, in 64 bits."""
    v = _e4m3_values()[:127]
    size = x.abs()
    up = torch.searchsorted(v, size.clamp(max=448.0)).clamp_(1, 126)
    low, high = v[up - 1], v[up]
    take = (size - low > high - size) | ((size - low == high - size) & (up % 2 == 0))
    return torch.where(take, high, low) * torch.sign(x)


def _exact_scale(amax):
    """2^max(-127, ceil(log2(amax / 448))), 1 for zero."""
    e = torch.ceil(torch.log2(amax / 448.0))
    e = torch.where(torch.exp2(e - 1) * 448.0 >= amax, e - 1, e)  # the logarithm may have been rounded across a whole number
    e = torch.where(torch.exp2(e) * 448.0 < amax, e + 1, e)
    return torch.where(amax > 0, torch.exp2(e.clamp(min=-127.0)), 1.0)


def _exact_form(y, kind, segments=None):
    """Values of the codes and scales in words of four blocks; `segments`: (first row, rows) of ranges whose blocks are their own."""
    rows, cols = y.shape
    if kind == "rows":
        blocks = _up(cols, 128) // 128
        codes, scales = torch.empty_like(y), torch.ones(_up(blocks, 4), rows, dtype=torch.float64, device="cuda")
        for b in range(blocks):
            part = y[:, 128 * b:128 * b + 128]
            scales[b] = _exact_scale(part.abs().amax(1))
            codes[:, 128 * b:128 * b + 128] = _nearest(part / scales[b][:, None])
    else:
        blocks = _up(rows, 128) // 128 if segments is None else _blocks(rows, len(segments))
        codes = torch.zeros(rows if segments is None else 128 * blocks, cols, dtype=torch.float64, device="cuda")
        scales = torch.ones(_up(blocks, 4), cols, dtype=torch.float64, device="cuda")
        b = 0
        for first, count in segments or [(0, rows)]:
            for r in range(first, first + count, 128):
                part = y[r:min(r + 128, first + count)]
                scales[b] = _exact_scale(part.abs().amax(0))
                codes[128 * b:128 * b + part.shape[0]] = _nearest(part / scales[b])
                b += 1
    return dict(codes=codes, scales=scales.view(-1, 4, scales.shape[1]).permute(0, 2, 1).contiguous())


def _exact_codes(codes, cols):
    v = _e4m3_values()
    return torch.cat([v, -v])[codes[..., :cols].long()]


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        h = s["x"].double()
        total = None
        if s["residual"] is not None:
            total = h + s["residual"].double()
            h = total.to(s["residual"].dtype).double()  # the norm is of the stream as it is stored
        root = 1.0 / torch.sqrt((h * h).sum(1) / case["cols"] + EPS)
        y = s["w"].double() * (h * root[:, None])
        return dict(total=total, root=root, forms=[_exact_form(y, k) for k in ({"both": ("rows", "cols")}.get(case["kind"], (case["kind"],)))])
    if case["op"] == "norm_gradient":
        h, r, dy, w = s["total"].double(), s["root"].double()[:, None], s["dy"].double(), s["w"].double()
        n = h * r
        dn = dy * w
        dx = r * (dn - n * ((dn * n).sum(1, keepdim=True) / case["cols"]))
        if case["add"]:
            dx = dx + s["dtotal"].double()
        return dict(dx=dx, dw=(dy * n).sum(0))
    off = s["offsets"].tolist()
    segments = [(a, b - a) for a, b in zip(off, off[1:])]
    if case["op"] == "segments":
        x = s["x"].double()
        by_rows = _exact_form(x, "rows")
        by_rows["codes"][off[-1]:] = 0.0
        by_rows["scales"][:, off[-1]:] = 1.0
        return [by_rows, _exact_form(x, "cols", segments)]
    i, o = case["inputs"], case["outputs"]
    out = s["out"].double()
    if case["way"] == "wgrad":
        b0 = 0
        wide = lambda name, cols, b: _exact_codes(s[name][128 * b:128 * b + 128], cols) * torch.exp2(s[name + "_scales"][b // 4, :, b % 4].double() - 127.0)  # noqa: E731
        for e, (_, count) in enumerate(segments):
            blocks = (count + 127) // 128
            c = torch.zeros(o, i, dtype=torch.float64, device="cuda")
            for b in range(b0, b0 + blocks):
                c += wide("a", o, b).T @ wide("b", i, b)
            out[e] = out[e] + c if case["add"] else c
            b0 += blocks
        return out
    k = i if case["way"] == "forward" else o
    ki, ri = torch.arange(i, device="cuda"), torch.arange(o, device="cuda")
    kx = torch.arange(k, device="cuda")
    for e, (first, count) in enumerate(segments):
        if count == 0:
            continue
        t = torch.arange(first, first + count, device="cuda")
        a = _exact_codes(s["a"][first:first + count], k) * torch.exp2(s["a_scales"][kx // 512, :, (kx // 128) % 4].T[t].double() - 127.0)
        w = _exact_codes(s["b"][e], i) * torch.exp2(s["b_scales"][e].double() - 127.0)[ri // 128][:, ki // 128]
        out[first:first + count] = a @ (w.T if case["way"] == "forward" else w)
    return out
