"""What is measured of the 8-bit operators: quantisation by blocks of 128, the block-scaled matrix product, AdamW.

The three are one training step of a linear layer and its serving form: activations, weights and output gradients are
quantised to E4M3 with a scale for each block of 128, multiplied (forward, input gradient, weight gradient), and the
weights updated by an AdamW step over many tensors whose states are held in 8 or in 32 bits.

`own` False: the operators written out in elementary torch operations in 32 bits.  `own` True: the calls a user makes.
"""
import math

import torch

own = False

E4M3 = torch.float8_e4m3fn


# ----------------------------------------------------------------------------------------------------------------------
# The cases.
# ----------------------------------------------------------------------------------------------------------------------
def listed():
    return [
        # a few sequences' next tokens, before a projection while serving: latency
        dict(name="quantise_few_rows", op="quantise", rows=33, cols=4096, kind="rows", dtype="bf16"),
        # a training batch's activations, wanted along the channels (forward) and along the tokens (weight gradient)
        dict(name="quantise_batch_both", op="quantise", rows=16384, cols=8192, kind="both", dtype="bf16"),
        # 32-bit master weights of a ragged layer, after an optimiser step
        dict(name="quantise_master_weights", op="quantise", rows=8190, cols=4100, kind="tiles", dtype="f32"),
        # one token through a square projection
        dict(name="product_one_token", op="product", way="forward", tokens=1, inputs=4096, outputs=4096, scales="e8m0", out="bf16", add=False),
        # a serving batch through an up-projection whose checkpoint carries 32-bit scales
        dict(name="product_serving_batch", op="product", way="forward", tokens=61, inputs=4096, outputs=16384, scales="f32", out="bf16", add=False),
        # prompt processing with the same kind of checkpoint
        dict(name="product_prompt_f32_scales", op="product", way="forward", tokens=4096, inputs=4096, outputs=8192, scales="f32", out="bf16", add=False),
        # forward pass of a training batch
        dict(name="product_forward", op="product", way="forward", tokens=8192, inputs=8192, outputs=8192, scales="e8m0", out="bf16", add=False),
        # gradient of the inputs of a ragged layer, packed batch of odd length
        dict(name="product_input_gradient", op="product", way="dgrad", tokens=5003, inputs=4100, outputs=8190, scales="e8m0", out="bf16", add=False),
        # gradient of the weights, added to a 32-bit gradient buffer over micro-batches
        dict(name="product_weight_gradient", op="product", way="wgrad", tokens=16384, inputs=4096, outputs=4096, scales="e8m0", out="f32", add=True),
        # many small tensors (norm weights, biases, adapters), 32-bit states: latency and launches
        dict(name="adamw_many_small", op="adamw", tensors=150, mean=5000, param="f32", grad="f32", states=32, stochastic=False, copy=False, clip=True),
        # a model's 32-bit master weights with 8-bit states, and the 16-bit copy that the next forward pass reads
        dict(name="adamw_8bit_master", op="adamw", tensors=64, mean=4000000, param="f32", grad="bf16", states=8, stochastic=True, copy=True, clip=True),
        # 16-bit weights without masters, rounded stochastically, 8-bit states
        dict(name="adamw_8bit_16bit_weights", op="adamw", tensors=37, mean=700000, param="bf16", grad="bf16", states=8, stochastic=True, copy=False, clip=False),
    ]


def _spread(rng, low, high):
    """A whole number whose logarithm is spread evenly."""
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high + 1)))))))


def draw(rng):
    op = rng.choice(["quantise", "product", "product", "adamw"])
    if op == "quantise":
        rows = _spread(rng, 1, 16384)
        cols = _spread(rng, 100, min(16384, 16384 * 8192 // rows))
        return dict(op=op, rows=rows, cols=cols, kind=rng.choice(["rows", "cols", "both", "tiles"]), dtype=rng.choice(["bf16", "f32"]))
    if op == "product":
        way = rng.choice(["forward", "forward", "dgrad", "wgrad"])
        tokens = _spread(rng, 1, 16384)
        inputs = _spread(rng, 200, 8192)
        outputs = _spread(rng, 200, min(16384, 8192 ** 3 // (tokens * inputs)))
        out = "f32" if way == "wgrad" else rng.choice(["bf16", "bf16", "f32"])
        return dict(op=op, way=way, tokens=tokens, inputs=inputs, outputs=outputs, scales=rng.choice(["e8m0", "f32"]) if way == "forward" else "e8m0",
                    out=out, add=out == "f32" and rng.random() < 0.5)
    tensors = _spread(rng, 1, 300)
    param = rng.choice(["f32", "bf16"])
    return dict(op=op, tensors=tensors, mean=_spread(rng, 500, min(8000000, 140000000 // tensors)), param=param, grad=rng.choice(["f32", "bf16"]),
                states=rng.choice([8, 32]), stochastic=rng.random() < 0.5, copy=param == "f32" and rng.random() < 0.5, clip=rng.random() < 0.5)


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
    rows, cols = codes.shape
    out = torch.zeros(rows, _up(cols, 16), dtype=torch.uint8, device="cuda")
    out[:, :cols] = codes.view(torch.uint8)
    return out


def _tensor_sizes(case):
    """Sizes of a model's tensors: unlike, the odd ones among them, the mean about as asked."""
    n, state = [], 12345 + case["tensors"]
    for _ in range(case["tensors"]):
        state = (state * 1103515245 + 12345) % (1 << 31)
        n.append(max(1, int(case["mean"] * (0.25 + 1.5 * state / (1 << 31)))))
    return n


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    s = dict(case=case)
    if case["op"] == "quantise":
        rows, cols = case["rows"], case["cols"]
        s["x"] = _activations(g, rows, cols, 0.02 if case["kind"] == "tiles" else 1.0).to(_dtype(case["dtype"]))
        if own:  # the buffers that a program reuses from step to step
            from paper_2608_06812_b200 import lowbit
            kind = case["kind"]
            s["by_rows"] = lowbit.Fp8Matrix.empty(rows, cols, lowbit.ROWS) if kind in ("rows", "both") else None
            s["by_cols"] = lowbit.Fp8Matrix.empty(rows, cols, lowbit.COLS) if kind in ("cols", "both") else None
            s["tiles"] = lowbit.Fp8Matrix.empty(rows, cols, lowbit.TILES) if kind == "tiles" else None
    elif case["op"] == "product":
        t, i, o = case["tokens"], case["inputs"], case["outputs"]
        x = _activations(g, t, i, 1.0) if case["way"] != "dgrad" else None
        dy = _activations(g, t, o, 1e-3) if case["way"] != "forward" else None
        w = torch.randn(o, i, generator=g, device="cuda").mul_(0.02) if case["way"] != "wgrad" else None
        if case["scales"] == "f32":  # scales that are no powers of two: amax / 448 of each block
            a, b = _quantise_f32(x, 1), _quantise_f32(w, 128)
        else:
            a = _quantise(x, "rows") if case["way"] == "forward" else _quantise(dy, "rows" if case["way"] == "dgrad" else "cols")
            b = _quantise(x, "cols") if case["way"] == "wgrad" else _quantise(w, "tiles")
        s["a"], s["a_scales"] = _padded(a[0]), a[1]
        s["b"], s["b_scales"] = _padded(b[0]), b[1]
        if case["scales"] == "e8m0":
            s["a_scales"] = _pack(s["a_scales"], case["way"] == "wgrad")
            if case["way"] == "wgrad":
                s["b_scales"] = _pack(s["b_scales"], True)
        m, n = (o, i) if case["way"] == "wgrad" else (t, i if case["way"] == "dgrad" else o)
        s["out"] = torch.zeros(m, _up(n, 8), dtype=_dtype(case["out"]), device="cuda")[:, :n]
        if case["add"]:
            s["out"].copy_(torch.randn(m, n, generator=g, device="cuda"))
        s["a_shape"] = (t, i if case["way"] == "forward" else o)
        s["b_shape"] = (t, i) if case["way"] == "wgrad" else (o, i)
        if own:  # the same tensors, in the framework's handles
            from paper_2608_06812_b200 import lowbit
            s["left"] = lowbit.Fp8Matrix(s["a"], s["a_scales"], *s["a_shape"], lowbit.COLS if case["way"] == "wgrad" else lowbit.ROWS)
            s["right"] = lowbit.Fp8Matrix(s["b"], s["b_scales"], *s["b_shape"], lowbit.COLS if case["way"] == "wgrad" else lowbit.TILES)
    else:
        sizes = _tensor_sizes(case)
        at = [0]
        for n in sizes:
            at.append(at[-1] + _up(n, 128))
        total = at[-1]
        which = torch.repeat_interleave(torch.arange(len(sizes), device="cuda"), torch.tensor([_up(n, 128) for n in sizes], device="cuda"))
        index = torch.arange(total, device="cuda") - torch.tensor(at[:-1], device="cuda")[which]
        live = index < torch.tensor(sizes, device="cuda")[which]
        if case["stochastic"]:
            s["key"] = torch.bitwise_xor(index & 0xFFFFFFFF, _mix(which + 1))
        del index
        size = torch.randn(len(sizes), generator=g, device="cuda").mul_(0.7).exp_().mul_(1e-3)[which]
        del which
        draw_ = lambda scale: torch.randn(total, generator=g, device="cuda").mul_(scale).mul_(live)  # noqa: E731
        s["grad"] = draw_(size).to(_dtype(case["grad"]))
        m = draw_(size * 0.25)
        v = (draw_(size) + 0.5 * size).square_().mul_(live)
        del size
        s["param"] = draw_(0.02).to(_dtype(case["param"]))
        if case["states"] == 8:
            s["m"], s["m_scale"] = _quantise_flat(m)
            s["v"], s["v_scale"] = _quantise_flat(v.sqrt_())
        else:
            s["m"], s["v"], s["m_scale"], s["v_scale"] = m, v, None, None
        del m, v, live
        s["copy"] = s["param"].to(torch.bfloat16) if case["copy"] else None
        s["clip"] = torch.rand((), generator=g, device="cuda").mul_(0.5).add_(0.25) if case["clip"] else None
        s["options"] = dict(lr=3e-4, betas=(0.9, 0.95), eps=1e-8, weight_decay=0.1, step=1000 + int(seed) % 97)
        s["seed"] = int(seed) * 7919 % (1 << 32) if case["stochastic"] else None
        if own:  # the table of tensors that a program builds once
            from paper_2608_06812_b200 import lowbit
            parts = lambda x: None if x is None else [x[a:a + n] for a, n in zip(at, sizes)]  # noqa: E731
            scales = lambda x: None if x is None else [x[a // 128:(a + n + 127) // 128] for a, n in zip(at, sizes)]  # noqa: E731
            s["table"] = lowbit.AdamWTable(parts(s["param"]), parts(s["grad"]), parts(s["m"]), parts(s["v"]), scales(s["m_scale"]), scales(s["v_scale"]),
                                           parts(s["copy"]))
    return s


# ----------------------------------------------------------------------------------------------------------------------
# The plain forms.
# ----------------------------------------------------------------------------------------------------------------------
def _mix(x):
    """32 bits of `x` (int64) well mixed: xor-shifts and odd multiplications."""
    x = x & 0xFFFFFFFF
    x = ((x ^ (x >> 16)) * 0x7FEB352D) & 0xFFFFFFFF
    x = ((x ^ (x >> 15)) * 0x846CA68B) & 0xFFFFFFFF
    return x ^ (x >> 16)


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
    amax = torch.where(torch.isfinite(size), size, 0.0).amax((1, 3))
    c = _scale_codes(amax)
    q = (f * _power(c, True)[:, None, :, None]).to(E4M3)
    q = q.view(f.shape[0] * br, f.shape[2] * bc)[:rows, :cols]
    return q, c


def _quantise_f32(x, lines):
    """The same by 1 x 128 or 128 x 128 blocks with 32-bit scales amax / 448."""
    rows, cols = x.shape
    f = torch.nn.functional.pad(x, (0, _up(cols, 128) - cols, 0, _up(rows, lines) - rows))
    f = f.view(f.shape[0] // lines, lines, f.shape[1] // 128, 128)
    scale = f.abs().amax((1, 3)).clamp_(min=1e-30) * (1.0 / 448.0)
    q = (f / scale[:, None, :, None]).clamp_(-448.0, 448.0).to(E4M3)
    return q.view(f.shape[0] * lines, f.shape[2] * 128)[:rows, :cols], scale.contiguous()


def _quantise_flat(x):
    f = x.view(-1, 128)
    c = _scale_codes(f.abs().amax(1))
    return (f * _power(c, True)[:, None]).to(E4M3).view(torch.uint8).view(-1), c


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


def _values(codes, shape, scales, lines, blocks):
    """Codes times scales [line blocks][column blocks], each for `lines` x `blocks` of them, in 32 bits."""
    rows, cols = shape
    f = codes.view(E4M3)[:, :cols].float()
    full = scales.repeat_interleave(lines, 0)[:rows].repeat_interleave(blocks, 1)[:, :cols]
    return f * full


def _plain_product(s):
    case = s["case"]
    if case["scales"] == "f32":
        a = _values(s["a"], s["a_shape"], s["a_scales"], 1, 128)
        b = _values(s["b"], s["b_shape"], s["b_scales"], 128, 128)
        c = a @ b.T
    elif case["way"] == "wgrad":
        blocks = _up(case["tokens"], 128) // 128
        a = _values(s["a"], s["a_shape"], _power(_unpack(s["a_scales"], blocks)), 128, 1)
        b = _values(s["b"], s["b_shape"], _power(_unpack(s["b_scales"], blocks)), 128, 1)
        c = a.T @ b
    else:
        a = _values(s["a"], s["a_shape"], _power(_unpack(s["a_scales"], _up(s["a_shape"][1], 128) // 128)).T, 1, 128)
        b = _values(s["b"], s["b_shape"], _power(s["b_scales"]), 128, 128)
        c = a @ (b.T if case["way"] == "forward" else b)
    return s["out"].add_(c) if case["add"] else c.to(_dtype(case["out"]))


def _round_root(y, noise):
    """Non-negative y <= 448 to E4M3: to nearest, or up or down by 16 random bits; what is not zero stays so."""
    if noise is None:
        w = y.to(E4M3).float()
    else:
        low = y < 2.0 ** -6
        z = torch.where(low, y + 2.0 ** -6, y)
        z = ((z.view(torch.int32) + (noise << 4).to(torch.int32)) & -0x100000).view(torch.float32)
        w = torch.where(low, z - 2.0 ** -6, z)
    return torch.where(y > 0, w.clamp(min=2.0 ** -9), y).to(E4M3)


def _plain_adamw(s):
    case, o = s["case"], s["options"]
    beta1, beta2 = o["betas"]
    g = s["grad"].float()
    if s["clip"] is not None:
        g = g * s["clip"]
    if case["states"] == 8:
        m = (s["m"].view(E4M3).float().view(-1, 128) * _power(s["m_scale"])[:, None]).view(-1)
        r = (s["v"].view(E4M3).float().view(-1, 128) * _power(s["v_scale"])[:, None]).view(-1)
        v = r * r
    else:
        m, v = s["m"], s["v"]
    m = m * beta1 + g * (1.0 - beta1)
    v = v * beta2 + (g * (1.0 - beta2)) * g
    r = v.sqrt()
    step = m / (r * (1.0 / math.sqrt(1.0 - beta2 ** o["step"])) + o["eps"])
    p = s["param"].float() * (1.0 - o["lr"] * o["weight_decay"]) - step * (o["lr"] / (1.0 - beta1 ** o["step"]))
    noise = _mix(s["key"] ^ _mix(torch.tensor(s["seed"], device="cuda"))) if case["stochastic"] else None
    if case["param"] == "bf16" and noise is not None:
        p = ((p.view(torch.int32) + (noise & 0xFFFF).to(torch.int32)) & -0x10000).view(torch.float32)
    s["param"].copy_(p)
    if case["copy"]:
        s["copy"].copy_(p)
    if case["states"] == 8:
        m, r = m.view(-1, 128), r.view(-1, 128)
        cm, cr = _scale_codes(m.abs().amax(1)), _scale_codes(r.amax(1))
        s["m"].copy_((m * _power(cm, True)[:, None]).to(E4M3).view(torch.uint8).view(-1))
        y = (r * _power(cr, True)[:, None]).view(-1)
        s["v"].copy_(_round_root(y, None if noise is None else noise >> 16).view(torch.uint8))
        s["m_scale"].copy_(cm)
        s["v_scale"].copy_(cr)
    else:
        s["m"].copy_(m)
        s["v"].copy_(v)


def _quantise_answer(codes, scales):
    return dict(codes=codes, scales=scales)


def _adamw_answer(s):
    eight = s["case"]["states"] == 8
    return dict(param=s["param"], copy=s["copy"], m=s["m"].view(E4M3) if eight else s["m"], v=s["v"].view(E4M3) if eight else s["v"],
                m_scale=s["m_scale"], v_scale=s["v_scale"])


# ----------------------------------------------------------------------------------------------------------------------
# One pass.
# ----------------------------------------------------------------------------------------------------------------------
def run(state):
    s = state
    case = s["case"]
    if case["op"] == "quantise":
        kind = case["kind"]
        if own:
            from paper_2608_06812_b200 import lowbit
            if kind == "tiles":
                lowbit.quantize_tiles(s["x"], out=s["tiles"])
                return _quantise_answer(s["tiles"].values8(), s["tiles"].scale_codes())
            lowbit.quantize_lines(s["x"], s["by_rows"], s["by_cols"])
            return [_quantise_answer(q.values8(), q.scale_codes()) for q in (s["by_rows"], s["by_cols"]) if q is not None]
        if kind == "tiles":
            return _quantise_answer(*_quantise(s["x"], kind))
        return [_quantise_answer(*_quantise(s["x"], k)) for k in (("rows", "cols") if kind == "both" else (kind,))]
    if case["op"] == "product":
        if not own:
            return _plain_product(s)
        from paper_2608_06812_b200 import lowbit
        return lowbit.matmul(s["left"], s["right"], out=s["out"], over_rows=case["way"] != "forward", accumulate=case["add"])
    if own:
        s["table"].step(seed=s["seed"], grad_scale=s["clip"], **s["options"])
    else:
        _plain_adamw(s)
    return _adamw_answer(s)


def work(case):
    if case["op"] == "quantise":
        n, size = case["rows"] * case["cols"], 4 if case["dtype"] == "f32" else 2
        blocks = {"rows": n / 128, "cols": n / 128, "both": n / 64, "tiles": n / 16384}[case["kind"]]
        return dict(bytes=n * size + n * (2 if case["kind"] == "both" else 1) + blocks, flops=3 * n)
    if case["op"] == "product":
        t, i, o = case["tokens"], case["inputs"], case["outputs"]
        m, n, k = dict(forward=(t, o, i), dgrad=(t, i, o), wgrad=(o, i, t))[case["way"]]
        out = m * n * (4 if case["out"] == "f32" else 2) * (2 if case["add"] else 1)
        scale = 4 if case["scales"] == "f32" else 1
        blocks = (m * k / 128 + (n * k / 128 if case["way"] == "wgrad" else n * k / 16384)) * scale
        return dict(bytes=m * k + n * k + blocks + out, flops=2 * m * n * k)
    n = sum(_tensor_sizes(case))
    size = lambda d: 4 if d == "f32" else 2  # noqa: E731
    each = 2 * size(case["param"]) + size(case["grad"]) + (4 + 4 / 128 if case["states"] == 8 else 16) + (2 if case["copy"] else 0)
    return dict(bytes=n * each, flops=16 * n)


# ----------------------------------------------------------------------------------------------------------------------
# What the outputs are, in 64 bits, from the definitions.
# ----------------------------------------------------------------------------------------------------------------------
def _e4m3_values():
    """The values of the codes 0 .. 127: sign clear, four bits of exponent (bias 7), three of fraction, 127 not a number."""
    v = [(f / 8 * 2.0 ** -6) if e == 0 else (1 + f / 8) * 2.0 ** (e - 7) for e in range(16) for f in range(8)]
    v[127] = math.nan
    return torch.tensor(v, dtype=torch.float64, device="cuda")


def _nearest(x):
    """The nearest of those values, ties to the even code, in 64 bits; nan for what is not finite."""
    v = _e4m3_values()[:127]
    size = x.abs()
    up = torch.searchsorted(v, size.clamp(max=448.0)).clamp_(1, 126)
    low, high = v[up - 1], v[up]
    take = (size - low > high - size) | ((size - low == high - size) & (up % 2 == 0))
    return torch.where(torch.isfinite(x), torch.where(take, high, low) * torch.sign(x), math.nan)


def _exact_scale(amax):
    """2^max(-127, ceil(log2(amax / 448))), 1 for zero."""
    e = torch.ceil(torch.log2(amax / 448.0))
    e = torch.where(torch.exp2(e - 1) * 448.0 >= amax, e - 1, e)  # the logarithm may have been rounded across a whole number
    e = torch.where(torch.exp2(e) * 448.0 < amax, e + 1, e)
    return torch.where(amax > 0, torch.exp2(e.clamp(min=-127.0)), 1.0)


def _exact_codes(codes, shape):
    v = _e4m3_values()
    return torch.cat([v, -v])[codes[:, :shape[1]].long()]


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "quantise":
        found = []
        for kind in {"both": ("rows", "cols")}.get(case["kind"], (case["kind"],)):
            x = s["x"].double()
            rows, cols = x.shape
            out = torch.empty(rows, cols, dtype=torch.float64, device="cuda")
            strip = 128 * max(1, (1 << 24) // (128 * cols))
            for r in range(0, rows, strip):
                part = x[r:r + strip]
                if kind == "rows":
                    for c in range(0, cols, 128):
                        b = part[:, c:c + 128]
                        out[r:r + strip, c:c + 128] = _nearest(b / _exact_scale(b.abs().amax(1, keepdim=True)))
                else:
                    for k in range(0, part.shape[0], 128):
                        b = part[k:k + 128]
                        top = b.abs().amax(0, keepdim=True)
                        if kind == "tiles":
                            top = torch.cat([t.amax(1, keepdim=True).expand_as(t) for t in top.split(128, 1)], 1)
                        out[r + k:r + k + 128] = _nearest(b / _exact_scale(top))
            found.append(dict(codes=out, scales=None))
        return found[0] if case["kind"] == "tiles" else found
    if case["op"] == "product":
        a, b = _exact_codes(s["a"], s["a_shape"]), _exact_codes(s["b"], s["b_shape"])
        sa, sb = s["a_scales"].double(), s["b_scales"].double()
        at, bt = [torch.arange(n, device="cuda") for n in s["a_shape"]], [torch.arange(n, device="cuda") for n in s["b_shape"]]
        if case["scales"] == "f32":
            a *= sa[:, at[1] // 128]
            b *= sb[bt[0] // 128][:, bt[1] // 128]
        else:
            word = lambda w, line, k: torch.exp2(w[k // 512, line, (k // 128) % 4] - 127.0)  # noqa: E731
            if case["way"] == "wgrad":
                a *= word(sa, at[1][None, :], at[0][:, None])
                b *= word(sb, bt[1][None, :], bt[0][:, None])
            else:
                a *= word(sa, at[0][:, None], at[1][None, :])
                b *= torch.exp2(sb - 127.0)[bt[0] // 128][:, bt[1] // 128]
        c = a @ b.T if case["way"] == "forward" else a @ b if case["way"] == "dgrad" else a.T @ b
        return c + s["out"].double() if case["add"] else c
    o = s["options"]
    (b1, b2), t, n = o["betas"], o["step"], s["param"].numel()
    wide = lambda x: x.double()  # noqa: E731
    table = _e4m3_values()
    out = dict(param=[], copy=[], m=[], v=[])
    part = 1 << 24
    for i in range(0, n, part):
        j = min(n, i + part)
        g = wide(s["grad"][i:j]) * (wide(s["clip"]) if s["clip"] is not None else 1.0)
        if case["states"] == 8:
            load = lambda c, e: (torch.cat([table, -table])[c[i:j].long()].view(-1, 128) * torch.exp2(wide(e[i // 128:j // 128]) - 127.0)[:, None]).view(-1)  # noqa: E731
            m, v = load(s["m"], s["m_scale"]), load(s["v"], s["v_scale"]) ** 2
        else:
            m, v = wide(s["m"][i:j]), wide(s["v"][i:j])
        m, v = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
        p = wide(s["param"][i:j])
        p = p - o["lr"] * o["weight_decay"] * p - o["lr"] * (m / (1 - b1 ** t)) / ((v / (1 - b2 ** t)).sqrt() + o["eps"])
        noise = None
        if case["stochastic"]:
            noise = _mix(s["key"][i:j] ^ _mix(torch.tensor(s["seed"], device="cuda")))
        if case["param"] == "bf16" and noise is not None:  # down to a whole number of units in the last place after a fraction of one is added
            unit = torch.exp2(torch.floor(torch.log2(p.abs().clamp(min=2.0 ** -126))) - 7)
            p = torch.sign(p) * torch.floor(p.abs() / unit + (noise & 0xFFFF).double() / 65536.0) * unit
        out["param"].append(p)
        out["copy"].append(p)
        if case["states"] == 8:
            m, r = m.view(-1, 128), v.sqrt().view(-1, 128)
            out["m"].append(_nearest(m / _exact_scale(m.abs().amax(1, keepdim=True))).view(-1))
            y = (r / _exact_scale(r.amax(1, keepdim=True))).view(-1)
            if noise is None:
                w = _nearest(y)
            else:
                unit = torch.exp2(torch.floor(torch.log2(y.clamp(min=2.0 ** -6))) - 3)
                w = torch.floor(y / unit + (noise >> 16).double() / 65536.0) * unit
            out["v"].append(torch.where(y > 0, w.clamp(min=2.0 ** -9), y))
        else:
            out["m"].append(m)
            out["v"].append(v)
    found = {k: torch.cat(v) for k, v in out.items()}
    if not case["copy"]:
        found["copy"] = None
    return {**found, "m_scale": None, "v_scale": None}
