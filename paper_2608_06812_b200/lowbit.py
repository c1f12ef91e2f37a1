"""The 8-bit operators on torch tensors: quantisation by blocks of 128, the block-scaled product, AdamW.

A linear layer in 8 bits:

    x8, xt8 = quantize_lines(x, rows=True, cols=True)   # for the forward product and for the weight gradient
    w8 = quantize_tiles(w)                              # one set of codes serves forward and backward
    y = matmul(x8, w8)                                  # y  = x w^T
    dx = matmul(quantize_lines(dy)[0], w8, over_rows=True)                       # dx = dy w
    dw = matmul(quantize_lines(dy, rows=False, cols=True)[1], xt8, over_rows=True, dtype=torch.float32)   # dw = dy^T x

`linear` is the same as a differentiable function.  Everything runs on the current stream of the tensors' device
through libozk.so; arguments are checked here (ValueError) and in the library (OzkError), nothing falls back.
"""
from __future__ import annotations

import ctypes

import torch
from torch.autograd.function import once_differentiable

from . import binding as ozk

ROWS, COLS, TILES = "rows", "cols", "tiles"
_TYPES = {torch.float32: ozk.OZK_F32, torch.bfloat16: ozk.OZK_BF16}


def _up(n: int, m: int) -> int:
    return -(-n // m) * m


# The raw handle of the current stream of a device, and the current device (a torch without CUDA has neither).
_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_device = getattr(torch._C, "_cuda_getDevice", None)


def _code(index: int, name: str, *args) -> int:
    """Calls the library with the device current."""
    fn = getattr(ozk.lib(), name)
    if _device() == index:
        return fn(*args)
    with torch.cuda.device(index):
        return fn(*args)


def _call(index: int, name: str, *args) -> None:
    """The same, and raises the library's errors (written out: a call inside a call costs 0.2 us)."""
    fn = getattr(ozk.lib(), name)
    if _device() == index:
        status = fn(*args)
    else:
        with torch.cuda.device(index):
            status = fn(*args)
    if status != ozk.OZK_OK:
        raise ozk.OzkError(status, name)


def _type(t: torch.Tensor, what: str) -> int:
    try:
        return _TYPES[t.dtype]
    except KeyError:
        raise ValueError(f"{what} is float32 or bfloat16, not {t.dtype}") from None


def _need_cuda(t: torch.Tensor, what: str) -> None:
    if not t.is_cuda:
        raise ValueError(f"{what} is not on a GPU")


# Tells autograd that the library has written to tensors of the caller (a list): a backward pass that saved one of them raises.
_written = torch._C._increment_version


def _versioned(tensors) -> list[torch.Tensor]:
    """Those that have versions: tensors made in inference mode have none."""
    return [t for t in tensors if not t.is_inference()]


# The status word of the products' bounded waits, one for each device: (address, tensor).
_statuses: dict[int, tuple[int, torch.Tensor]] = {}


def _status(index: int) -> int:
    found = _statuses.get(index)
    if found is None:
        if torch.cuda.is_current_stream_capturing():
            raise RuntimeError("the first product on a GPU cannot be captured: make one before, for its status word")
        t = torch.zeros(1024, dtype=torch.uint8, device=torch.device("cuda", index))
        torch.cuda.current_stream(index).synchronize()   # other streams may use it next
        found = _statuses.setdefault(index, (t.data_ptr(), t))   # the first of two threads
    return found[0]


def check_async(device: torch.device | str | int | None = None) -> None:
    """Waits for the current stream and raises OzkError if a wait inside a product kernel on that GPU had run out."""
    index = device if isinstance(device, int) else None if device is None else torch.device(device).index
    index = torch.cuda.current_device() if index is None else index
    if index in _statuses:
        _call(index, "ozk_get_workspace_status", _statuses[index][0], _stream(index))


class Fp8Matrix:
    """A rows x cols matrix of E4M3 codes (uint8 [rows, ld], ld a multiple of 16) and its scales.

    kind ROWS: a scale per 1 x 128 block, for products that sum over the columns; COLS: per 128 x 1 block, for products
    that sum over the rows; TILES: per 128 x 128 tile, for either.  Scales are uint8 UE8M0 codes, [ceil(k/512), lines, 4]
    for ROWS and COLS, [ceil(rows/128), ceil(cols/128)] for TILES; or float32 [rows, ceil(cols/128)] for ROWS and
    [ceil(rows/128), ceil(cols/128)] for TILES."""

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor, rows: int, cols: int, kind: str):
        if kind not in (ROWS, COLS, TILES):
            raise ValueError(f"kind is {ROWS!r}, {COLS!r} or {TILES!r}, not {kind!r}")
        _need_cuda(codes, "codes")
        if codes.dtype == torch.float8_e4m3fn:
            codes = codes.view(torch.uint8)
        if codes.dtype != torch.uint8 or codes.dim() != 2 or codes.shape[0] != rows or codes.shape[1] < cols:
            raise ValueError(f"codes are uint8 or float8_e4m3fn [{rows}, at least {cols}], not {codes.dtype} {tuple(codes.shape)}")
        ld = codes.stride(0) if rows > 1 else _up(max(codes.shape[1], 1), 16)
        if rows and cols and (codes.stride(1) != 1 or ld % 16 or ld < cols or codes.data_ptr() % 16):
            raise ValueError("codes lie in rows of a multiple of 16 bytes, at a multiple of 16 bytes")
        floats = scales.dtype == torch.float32
        br, bc = -(-rows // 128), -(-cols // 128)
        if floats:
            want = {ROWS: (rows, bc), TILES: (br, bc)}.get(kind)
        else:
            want = {ROWS: (-(-cols // 512), rows, 4), COLS: (-(-rows // 512), cols, 4), TILES: (br, bc)}[kind]
        if (not floats and scales.dtype != torch.uint8) or scales.device != codes.device or not scales.is_contiguous() or want is None or tuple(scales.shape) != want:
            raise ValueError(f"scales of {rows} x {cols} by {kind}: {scales.dtype} {tuple(scales.shape)}, wanted {want} on {codes.device}")
        self.codes, self.scales, self.rows, self.cols, self.kind = codes, scales, rows, cols, kind
        self.index = codes.device.index
        # views that are asked for at every step
        self._values8 = codes.view(torch.float8_e4m3fn)[:, :cols]
        self._words = None if floats or kind == TILES else scales.transpose(1, 2)
        self._seen = None   # what autograd is told of when the library writes, once it does
        # what the quantisers are given, and what a matrix to be written is compared with
        self._target = (codes.data_ptr(), ld, scales.data_ptr())
        self._form = (rows, cols, kind, floats, self.index)
        if floats:
            code = ozk.OZK_SCALE_LINES_F32 if kind == ROWS else ozk.OZK_SCALE_TILES_F32
        else:
            code = ozk.OZK_SCALE_TILES if kind == TILES else ozk.OZK_SCALE_LINES
        self.ld = ld
        # the operand summed over its columns, and over its rows
        self._operand = [ozk.ozk_fp8_operand(codes.data_ptr(), ld, scales.data_ptr(), code, over) for over in (0, 1)]
        self._at = [ctypes.addressof(o) for o in self._operand]

    @classmethod
    def empty(cls, rows: int, cols: int, kind: str, device: torch.device | str = "cuda") -> "Fp8Matrix":
        codes = torch.empty(rows, max(_up(cols, 16), 16), dtype=torch.uint8, device=device)
        shape = {ROWS: (-(-cols // 512), rows, 4), COLS: (-(-rows // 512), cols, 4), TILES: (-(-rows // 128), -(-cols // 128))}[kind]
        return cls(codes, torch.empty(shape, dtype=torch.uint8, device=device), rows, cols, kind)

    def values8(self) -> torch.Tensor:
        """The codes as torch's 8-bit type, [rows, cols], without the scales."""
        return self._values8

    def scale_codes(self) -> torch.Tensor:
        """Scales by stored block: [rows, blocks] (ROWS), [blocks, cols] (COLS), [row tiles, column tiles] (TILES)."""
        if self._words is None:
            return self.scales
        k, lines = (self.cols, self.rows) if self.kind == ROWS else (self.rows, self.cols)
        blocks, s = -(-k // 128), self._words.contiguous()   # [groups][four blocks][lines]
        return s.as_strided((lines, blocks), (1, lines)) if self.kind == ROWS else s.as_strided((blocks, lines), (lines, 1))

    def dequantize(self) -> torch.Tensor:
        """Codes times scales in float32."""
        s = self.scale_codes()
        if s.dtype != torch.float32:
            s = torch.where(s > 0, s.int() << 23, 1 << 22).view(torch.float32)
        lines, blocks = {ROWS: (1, 128), COLS: (128, 1), TILES: (128, 128)}[self.kind]
        full = s.repeat_interleave(lines, 0)[:self.rows].repeat_interleave(blocks, 1)[:, :self.cols]
        return self.values8().float() * full


_NONE = (None, 0, None)


def _input(x: torch.Tensor) -> tuple[int, int, int, int]:
    kind = _TYPES.get(x.dtype)
    if kind is None:
        _type(x, "x")
    if not x.is_cuda or x.dim() != 2:
        _need_cuda(x, "x")
        raise ValueError(f"x has two dimensions, not {x.dim()}")
    rows, cols = x.shape
    ld, step = x.stride()
    if cols > 1 and step != 1 and rows:
        raise ValueError("the rows of x are contiguous")
    return rows, cols, kind, ld if rows > 1 else max(cols, 1)


def _rewritten(q: Fp8Matrix) -> None:
    if q._seen is None:
        q._seen = _versioned((q.codes, q.scales))
    _written(q._seen)


def _output(q: Fp8Matrix, rows: int, cols: int, kind: str, index: int) -> tuple:
    if q._form != (rows, cols, kind, False, index):
        raise ValueError(f"out is a {rows} x {cols} Fp8Matrix by {kind} with UE8M0 scales on GPU {index}")
    return q._target


def quantize_lines(x: torch.Tensor, rows: "bool | Fp8Matrix | None" = True, cols: "bool | Fp8Matrix | None" = False):
    """x [rows, cols] (float32 or bfloat16) by 1 x 128 blocks, by 128 x 1 blocks, or both in one pass over x.
    `rows`, `cols`: whether that form is wanted, or an Fp8Matrix to write it to.  Returns the pair (None where not wanted)."""
    r, c, kind, ld = _input(x)
    index = x.get_device()
    by_rows = Fp8Matrix.empty(r, c, ROWS, x.device) if rows is True else rows or None
    by_cols = Fp8Matrix.empty(r, c, COLS, x.device) if cols is True else cols or None
    if by_rows is None and by_cols is None:
        raise ValueError("neither rows nor columns are wanted")
    to_rows = _NONE if by_rows is None else _output(by_rows, r, c, ROWS, index)
    to_cols = _NONE if by_cols is None else _output(by_cols, r, c, COLS, index)
    _call(index, "ozk_fp8_quantize_lines", r, c, x.data_ptr(), kind, ld, *to_rows, *to_cols, _stream(index))
    if by_rows is rows and rows:
        _rewritten(rows)
    if by_cols is cols and cols:
        _rewritten(cols)
    return by_rows, by_cols


def quantize_tiles(x: torch.Tensor, out: Fp8Matrix | None = None) -> Fp8Matrix:
    """x [rows, cols] (float32 or bfloat16) by 128 x 128 tiles."""
    r, c, kind, ld = _input(x)
    index = x.get_device()
    q = Fp8Matrix.empty(r, c, TILES, x.device) if out is None else out
    _call(index, "ozk_fp8_quantize_tiles", r, c, x.data_ptr(), kind, ld, *_output(q, r, c, TILES, index), _stream(index))
    if out is not None:
        _rewritten(out)
    return q


def matmul(a: Fp8Matrix, b: Fp8Matrix, out: torch.Tensor | None = None, over_rows: bool = False, dtype: torch.dtype = torch.bfloat16,
           accumulate: bool = False) -> torch.Tensor:
    """The product of two 8-bit matrices, each summed over the axis its scales run along: columns for ROWS, rows for COLS.
    TILES serve either: `over_rows` says that b, if it is by tiles, is summed over its rows (and a by tiles over its rows if b is COLS).
      matmul(x by ROWS, w by TILES)                   x w^T
      matmul(dy by ROWS, w by TILES, over_rows=True)  dy w
      matmul(dy by COLS, x by COLS)                   dy^T x
    Returns a [lines of a, lines of b] tensor, `out` if given (float32 or bfloat16; float32 with accumulate, which adds)."""
    if over_rows and b.kind == ROWS:
        raise ValueError("a matrix by rows cannot be summed over its rows")
    a_over = a.kind == COLS or (a.kind == TILES and b.kind == COLS)
    b_over = b.kind == COLS or (b.kind == TILES and over_rows)
    m, k = (a.cols, a.rows) if a_over else (a.rows, a.cols)
    n, kb = (b.cols, b.rows) if b_over else (b.rows, b.cols)
    if k != kb:
        raise ValueError(f"the operands are summed over {k} and {kb} elements")
    index = a.index
    if b.index != index:
        raise ValueError("the operands are on two devices")
    given = out
    if out is None:
        if accumulate:
            raise ValueError("accumulate needs out")
        if dtype not in _TYPES:
            raise ValueError(f"the result is float32 or bfloat16, not {dtype}")
        out = torch.empty(m, _up(n, 8), dtype=dtype, device=a.codes.device)[:, :n]   # rows at 16-byte boundaries
    elif out.shape != (m, n) or out.get_device() != index or (n > 1 and out.stride(1) != 1):
        raise ValueError(f"out is [{m}, {n}] on GPU {index} with contiguous rows")
    kind, ldc, add, status_at, stream = _type(out, "out"), out.stride(0) if m > 1 else max(n, 1), 1 if accumulate else 0, _status(index), _stream(index)
    at_a, at_b = a._at[a_over], b._at[b_over]
    status = _code(index, "ozk_fp8_gemm_scratch", m, n, k, at_a, at_b, out.data_ptr(), kind, ldc, add, status_at, None, 0, stream)
    if status == ozk.OZK_ERR_WORKSPACE:
        # K is split and nothing has been enqueued.  The sums' memory is this call's until both launches are, then the allocator's to
        # order on the stream: no two threads or streams hold the same, and what a graph captures is the graph's own.
        plan = ozk.ozk_fp8_plan()
        _call(index, "ozk_fp8_gemm_plan", m, n, k, at_a, at_b, kind, 0, ctypes.byref(plan))
        scratch = torch.empty(plan.scratch_bytes, dtype=torch.uint8, device=a.codes.device)
        status = _code(index, "ozk_fp8_gemm_scratch", m, n, k, at_a, at_b, out.data_ptr(), kind, ldc, add, status_at, scratch.data_ptr(), plan.scratch_bytes, stream)
    if status != ozk.OZK_OK:
        raise ozk.OzkError(status, "ozk_fp8_gemm")
    if given is not None and not given.is_inference():
        _written((given,))
    return out


def _rows(x: torch.Tensor) -> torch.Tensor:
    flat = x.reshape(x.shape[:-1].numel(), x.shape[-1])
    return flat if flat.stride(1) == 1 and flat.stride(0) >= flat.shape[1] else flat.contiguous()   # an expanded gradient has strides of 0


class _Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, w8, for_dx, for_dw):
        flat = _rows(x)
        by_rows, by_cols = quantize_lines(flat, True, for_dw)
        ctx.x8, ctx.w8, ctx.shape, ctx.types = by_cols, w8, x.shape, (x.dtype, w.dtype)
        ctx.versions = [(t, t._version) for t in _versioned((w8.codes, w8.scales))] if for_dx else []
        return matmul(by_rows, w8, dtype=x.dtype).reshape(*x.shape[:-1], w8.rows)

    @staticmethod
    @once_differentiable   # the products below are not seen by autograd: a second derivative raises
    def backward(ctx, dy):
        need_x, need_w = ctx.needs_input_grad[:2]
        if need_x and any(t._version != v for t, v in ctx.versions):
            raise RuntimeError("the 8-bit weights needed for the gradient of x have been modified by an inplace operation")
        by_rows, by_cols = quantize_lines(_rows(dy), need_x, need_w)
        dx = matmul(by_rows, ctx.w8, over_rows=True, dtype=ctx.types[0]).reshape(ctx.shape) if need_x else None
        dw = matmul(by_cols, ctx.x8, dtype=torch.float32).to(ctx.types[1]) if need_w else None
        return dx, dw, None, None, None


def linear(x: torch.Tensor, w: torch.Tensor, w8: Fp8Matrix | None = None) -> torch.Tensor:
    """x w^T in 8 bits, with gradients of x and w (formed from the same 8-bit weights and from the gradient's own 8-bit forms; gradients of these
    gradients raise RuntimeError).
    x: [..., inputs]; w: [outputs, inputs]; w8: quantize_tiles(w), where a program keeps it between steps (and leaves it as it is until
    the backward pass, which reads it for the gradient of x and raises RuntimeError if it has been written again)."""
    grads = torch.is_grad_enabled()   # a Function's needs_input_grad is set under no_grad too
    for_dx, for_dw = grads and x.requires_grad, grads and w.requires_grad
    if w8 is None:
        w8 = quantize_tiles(_rows(w.detach()))
    elif w.shape != (w8.rows, w8.cols) or w8.scales.dtype != torch.uint8 or not (w8.kind == TILES or (w8.kind == ROWS and not for_dx)):
        raise ValueError(f"w8 is a {tuple(w.shape)} Fp8Matrix by {TILES} with UE8M0 scales (or by {ROWS}, where x needs no gradient), not {w8.rows} x {w8.cols} by {w8.kind}")
    return _Linear.apply(x, w, w8, for_dx, for_dw)


class AdamWTable:
    """The tensors of an AdamW step: lists of equal length, entries of equal size, each contiguous.

    params float32 or bfloat16, grads float32 or bfloat16; m, v float32, or uint8 E4M3 codes with m_scale, v_scale (uint8,
    one for each 128 elements; v then holds the ROOT of the second moment); copies: optional bfloat16 copies of float32
    params, written at every step.  The table holds the tensors' addresses (and keeps the tensors alive): build it once.
    Where a gradient is a param's own `.grad`, a step raises RuntimeError once that has been replaced: zero_grad(set_to_none=False) keeps it.
    Autograd is told of writes to the copies and to params that require gradients; a program that hands in their detached aliases sees to
    it by itself that no step comes between a forward pass and its backward pass."""

    def __init__(self, params, grads, m, v, m_scale=None, v_scale=None, copies=None):
        lists = dict(params=list(params), grads=list(grads), m=list(m), v=list(v))
        count = len(lists["params"])
        for name, given in (("m_scale", m_scale), ("v_scale", v_scale), ("copies", copies)):
            lists[name] = None if given is None else list(given)
        for name, tensors in lists.items():
            if tensors is None:
                continue
            if len(tensors) != count:
                raise ValueError(f"{len(tensors)} {name} for {count} params")
            for t, p in zip(tensors, lists["params"]):
                _need_cuda(t, name)
                want = -(-p.numel() // 128) if name.endswith("scale") else p.numel()
                if t.numel() != want or not t.is_contiguous() or t.device != p.device or t.dtype != tensors[0].dtype or p.device != lists["params"][0].device:
                    raise ValueError(f"{name}: contiguous tensors of one type, {want} elements here, on the device of the params")
        first = {name: t[0].dtype if t else None for name, t in lists.items()}
        if count:
            if first["params"] not in _TYPES or first["grads"] not in _TYPES:
                raise ValueError("params and grads are float32 or bfloat16")
            eight = first["m"] == torch.uint8
            if first["m"] != first["v"] or first["m"] not in (torch.uint8, torch.float32):
                raise ValueError("m and v are both float32 or both uint8")
            if eight != (lists["m_scale"] is not None) or eight != (lists["v_scale"] is not None) or (eight and (first["m_scale"], first["v_scale"]) != (torch.uint8,) * 2):
                raise ValueError("m_scale and v_scale (uint8) go with 8-bit m and v")
            if copies is not None and (first["params"] != torch.float32 or first["copies"] != torch.bfloat16):
                raise ValueError("copies are bfloat16, of float32 params")
        self.tensors, self.count = lists, count
        # what autograd may have saved when a step writes to it; 0.05 us a tensor and step
        self._seen = _versioned([p for p in lists["params"] if p.requires_grad] + (lists["copies"] or []))
        # gradients that autograd owns: it may put others in their place
        self._owned = [(p, g, g.data_ptr()) for p, g in zip(lists["params"], lists["grads"]) if p.numel() and p.is_leaf and p.grad is not None and p.grad.data_ptr() == g.data_ptr()]
        self._table = (ozk.ozk_adamw_tensor * max(count, 1))()
        self._options = ozk.ozk_adamw_options()
        self._table_at, self._options_at = ctypes.addressof(self._table), ctypes.addressof(self._options)
        if count:
            self.device = lists["params"][0].device
            at = lambda name, i: None if lists[name] is None else lists[name][i].data_ptr()  # noqa: E731
            for i in range(count):
                self._table[i] = ozk.ozk_adamw_tensor(*(at(name, i) for name in ("params", "grads", "m", "v", "m_scale", "v_scale", "copies")), lists["params"][i].numel())
            self._options.param_type, self._options.grad_type = _TYPES[first["params"]], _TYPES[first["grads"]]
            self._options.state_bits = 8 if eight else 32

    @classmethod
    def zeros(cls, params, grads, bits: int = 8, copies=None) -> "AdamWTable":
        """With states of zero, in 8 or 32 bits."""
        params = list(params)
        if bits not in (8, 32):
            raise ValueError("states have 8 or 32 bits")
        make = lambda: [torch.zeros(p.numel(), dtype=torch.uint8 if bits == 8 else torch.float32, device=p.device) for p in params]  # noqa: E731
        scale = lambda: [torch.full((-(-p.numel() // 128),), 127, dtype=torch.uint8, device=p.device) for p in params] if bits == 8 else None  # noqa: E731
        return cls(params, grads, make(), make(), scale(), scale(), copies)

    def step(self, lr: float, step: int, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay: float = 0.01, seed: int | None = None,
             grad_scale: torch.Tensor | None = None, skip: torch.Tensor | None = None) -> None:
        """Step number `step` (1 is the first), in place.  seed: round 8-bit roots and bfloat16 params stochastically, with
        another seed at each step; None: to nearest.  grad_scale: float32 scalar on the GPU that multiplies the gradients.
        skip: int32 scalar on the GPU; if it is not zero, nothing changes."""
        if self.count == 0:
            return
        for t, dtype, name in ((grad_scale, torch.float32, "grad_scale"), (skip, torch.int32, "skip")):
            if t is not None and (t.dtype != dtype or t.numel() != 1 or t.device != self.device):
                raise ValueError(f"{name} is one {dtype} on {self.device}")
        for p, g, at in self._owned:
            now = p.grad
            if now is not g and (now is None or now.data_ptr() != at):
                raise RuntimeError("the gradient of a param is no longer the tensor that the table was built with: zero gradients in place (set_to_none=False), or build the table again")
        o = self._options
        o.stochastic, o.seed = (0, 0) if seed is None else (1, seed & 0xFFFFFFFF)
        o.lr, (o.beta1, o.beta2), o.eps, o.weight_decay, o.step = lr, betas, eps, weight_decay, step
        o.grad_scale = None if grad_scale is None else grad_scale.data_ptr()
        o.skip = None if skip is None else skip.data_ptr()
        _call(self.device.index, "ozk_adamw_step", self._table_at, self.count, self._options_at, _stream(self.device.index))
        if self._seen:
            _written(self._seen)
