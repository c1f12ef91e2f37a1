"""The RMS norm that writes 8-bit operands, and its gradients, against the formulas in 64 bits.

FP32 bounds (u = 2^-24).  A sum of n products in a fixed tree is off by at most d u of the sum of sizes, d the longest chain: 64 additions in a thread, five
steps over a warp, 16 warps, and the products' own rounding: d = 86.  The inverse root of a mean of squares is then off by at most (d + 2) / 2 + 2 = 46 u of its
value, and y = (h s) w by 48 u.  A code is that of some number so near to y; its scale that of some maximum so near.
"""
import numpy as np
import pytest
import torch

from oracle import lowbit as ref
from paper_2608_06812_b200 import binding as ozk
from paper_2608_06812_b200 import lowbit

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
F32, BF16 = torch.float32, torch.bfloat16
TYPES = [(BF16, None), (BF16, BF16), (BF16, F32), (F32, None), (F32, F32)]
SIZES = [(1, 1), (3, 5), (1, 128), (2, 130), (130, 512), (7, 516), (129, 1023), (5, 2048), (300, 1100), (9, 4096), (33, 4100), (2, 8192), (131, 8196), (3, 16385), (2, 20004), (2, 32768)]


def make(rows, cols, dtype, seed, size=1.0, pad=0, offset=0):
    """Values of unlike size, in a wider buffer at an odd place where asked for."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g) * torch.randn(rows, 1, generator=g).mul(1.5).exp() * size
    whole = torch.full((rows, cols + pad + offset), 3.0e4, dtype=dtype, device="cuda")
    part = whole[:, offset:offset + cols]
    part.copy_(x)
    return part


def exponents(top):
    """Scale exponents of maxima (arrays)."""
    return np.vectorize(lambda t: ref.scale_exponent(np.array([t])))(top)


def blocks_max(a, kind):
    rows, cols = a.shape
    if kind == "rows":
        return np.stack([np.fmax.reduce(a[:, c:c + 128], 1) for c in range(0, cols, 128)], 1)
    return np.stack([np.fmax.reduce(a[r:r + 128], 0) for r in range(0, rows, 128)], 0)


def check_form(q, y, kind):
    """Codes and scales of an Fp8Matrix against 64-bit y."""
    e = q.scale_codes().cpu().numpy().astype(np.int64) - 127
    size = np.where(np.isfinite(y), np.abs(y), 0.0)
    low, high = exponents(blocks_max(size * (1 - 48 * U), kind)), exponents(blocks_max(size * (1 + 48 * U), kind))
    assert ((e >= low) & (e <= high)).all(), kind
    s = 2.0 ** -ref.spread(e, y.shape, kind).astype(np.float64)
    got = ref.decode(q.codes.cpu().numpy()[:, :y.shape[1]])
    z = np.clip(y * s, -448 * (1 + 48 * U), 448 * (1 + 48 * U))
    a, b = (ref.nearest(np.clip(z * f, -448.0, 448.0)) for f in (1 - 48 * U, 1 + 48 * U))
    bad = ~((got >= np.fmin(a, b)) & (got <= np.fmax(a, b))) & ~(np.isnan(y) & np.isnan(got))
    assert not bad.any(), (kind, int(bad.sum()), np.argwhere(bad)[:4])


def check_forward(x, w, r, n, eps):
    h = x.double() if r is None else (x.float() + r.float()).to(r.dtype).double()
    if r is not None:
        assert torch.equal(n.total.double(), h)
    h, w = h.cpu().numpy(), w.double().cpu().numpy()
    s = 1.0 / np.sqrt((h * h).mean(1) + float(np.float32(eps)))
    if n.root is not None:
        got = n.root.double().cpu().numpy()
        assert (np.abs(got - s) <= 46 * U * s).all()
    y = h * s[:, None] * w
    if n.y is not None:
        half = torch.finfo(n.y.dtype).eps / 2
        assert (np.abs(n.y.double().cpu().numpy() - y) <= np.abs(y) * (48 * U + half * (1 + 48 * U)) + 1e-38).all()
    if n.rows is not None:
        check_form(n.rows, y, "rows")
    if n.cols is not None:
        check_form(n.cols, y, "cols")


@pytest.mark.parametrize("types", TYPES, ids=lambda t: "_".join("none" if x is None else str(x)[6:] for x in t))
@pytest.mark.parametrize("rows,cols", SIZES)
def test_forms(rows, cols, types):
    x = make(rows, cols, types[0], rows + cols)
    r = None if types[1] is None else make(rows, cols, types[1], rows + cols + 1, 2.0)
    w = make(1, cols, F32 if cols % 2 else BF16, 3)[0]
    check_forward(x, w, r, lowbit.rms_norm(x, w, r, rows=True, cols=True, y=True, root=True), 1e-6)


@pytest.mark.parametrize("rows,cols", [(1, 4096), (5, 700), (200, 1030)])
@pytest.mark.parametrize("want", ["rows", "cols", "y", "root", "nothing"])
def test_each_form_alone(rows, cols, want):
    x, r, w = make(rows, cols, BF16, 1), make(rows, cols, BF16, 2), make(1, cols, F32, 3)[0]
    n = lowbit.rms_norm(x, w, r, eps=1e-3, rows=want == "rows", cols=want == "cols", y=want == "y", root=want == "root")
    check_forward(x, w, r, n, 1e-3)
    assert [f is not None for f in (n.rows, n.cols, n.y)] == [want == "rows", want == "cols", want == "y"]


@pytest.mark.parametrize("pad,offset", [(1, 0), (4, 0), (2, 2), (8, 4), (3, 1)])
@pytest.mark.parametrize("types", TYPES, ids=lambda t: "_".join("none" if x is None else str(x)[6:] for x in t))
def test_strides_and_alignments(types, pad, offset):
    for rows, cols in ((5, 640), (130, 1021)):
        x = make(rows, cols, types[0], 1, pad=pad, offset=offset)
        r = None if types[1] is None else make(rows, cols, types[1], 2, pad=pad, offset=offset)
        total = None if r is None else make(rows, cols, types[1], 4, pad=pad, offset=offset)
        y = make(rows, cols, types[0], 5, pad=pad, offset=offset)
        w = make(1, cols, BF16, 3, pad=pad, offset=offset)[0]
        n = lowbit.rms_norm(x, w, r, rows=True, cols=True, y=y, total=total, root=True)
        check_forward(x, w, r, n, 1e-6)
        for part in (y, total):   # what lies beside the results stays
            if part is not None:
                part.fill_(3.0e4)
                assert (part._base == 3.0e4).all()


def test_the_stream_is_updated_in_place():
    for which in ("residual", "x"):
        x, r, w = make(70, 900, BF16, 1), make(70, 900, BF16, 2), make(1, 900, F32, 3)[0]
        kept = [x.clone(), r.clone()]
        n = lowbit.rms_norm(x, w, r, rows=True, cols=True, root=True, total=r if which == "residual" else x)
        assert n.total.data_ptr() == (r if which == "residual" else x).data_ptr()
        check_forward(kept[0], w, kept[1], n, 1e-6)


def test_the_answer_does_not_take_the_place_of_what_is_normed():
    """The columns' codes are formed from it after the answer has been written; the place of x is free once the stream has it."""
    x, r, w = make(140, 300, BF16, 1), make(140, 300, BF16, 2), make(1, 300, F32, 3)[0]
    for arguments in (dict(y=x), dict(residual=r, total=r, y=r), dict(residual=r, total=x, y=x)):
        with pytest.raises(ValueError, match="place"):
            lowbit.rms_norm(x, w, **arguments)
    kept = x.clone()
    check_forward(kept, w, r, lowbit.rms_norm(x, w, r, rows=True, cols=True, y=x, root=True), 1e-6)


@pytest.mark.parametrize("cols", [4096, 4097, 4100, 515])
def test_a_single_row_at_any_place(cols):
    for offset in (0, 1, 4):
        x, r = make(1, cols, BF16, 1, pad=3, offset=offset), make(1, cols, F32, 2, pad=1, offset=offset)
        w = make(1, cols, BF16, 3)[0]
        n = lowbit.rms_norm(x, w, r, cols=True, y=True, root=True)
        check_forward(x, w, r, n, 1e-6)
        check_backward(n.y, n.total, n.root, w, r, lowbit.rms_norm_backward(n.y, n.total, n.root, w, r))


@pytest.mark.parametrize("types", [(BF16, BF16), (BF16, F32), (F32, F32)], ids=["bf16", "bf16_f32", "f32"])
def test_the_stream_of_any_bits(types):
    """Every kind of number: subnormal, both zeros, infinities, NaN; sums as torch's, rounded once."""
    g = torch.Generator().manual_seed(0)
    bits = lambda d: torch.randint(-2 ** 15, 2 ** 15, (64, 2048), generator=g, dtype=torch.int16).view(BF16).to(d).cuda()  # noqa: E731
    x, r = bits(types[0]), bits(types[1])
    r[::2] = torch.where(torch.rand(32, 2048, generator=g).cuda() < 0.5, -x[::2].to(types[1]), x[::2].to(types[1]))   # what cancels
    x[:4] *= 1e-36
    r[:4] *= 1e-36
    for shift in (0, 1):   # rows at even and odd places
        a, b = x[:, shift:], r[:, shift:]
        total = lowbit.rms_norm(a, torch.ones(2048 - shift, device="cuda"), b, rows=False).total
        want = (a.float() + b.float()).to(types[1])
        assert torch.equal(total.isnan(), want.isnan())
        same = total.view(torch.int16 if types[1] is BF16 else torch.int32) == want.view(torch.int16 if types[1] is BF16 else torch.int32)
        assert (same | want.isnan()).all()


def test_zeros_infinities_and_nan():
    rows, cols = 9, 700
    x = make(rows, cols, F32, 1)
    x[1] = 0.0
    x[2, 5] = float("nan")
    x[3, 600] = float("inf")
    x[4] = 3.0e38          # squares beyond FP32
    x[5] = 1e-30           # squares below it: eps alone
    x[6] = -0.0
    w = make(1, cols, F32, 3)[0]
    for kind in ("rows", "cols"):
        n = lowbit.rms_norm(x, w, rows=kind == "rows", cols=kind == "cols", y=True, root=True)
        y, q = n.y.cpu(), (n.rows if kind == "rows" else n.cols)
        d = q.dequantize().cpu()
        assert (y[1] == 0).all() and (d[1] == 0).all() and n.root[1] == 1000.0
        assert y[2].isnan().all() and d[2].isnan().all()
        assert n.root[3] == 0 and y[3, 600].isnan() and (y[3, torch.arange(cols) != 600] == 0).all() and d[3, 600].isnan() and (d[3, torch.arange(cols) != 600] == 0).all()
        assert n.root[4] == 0 and (y[4] == 0).all()
        assert torch.allclose(y[5], (x[5] * 1000.0 * w).cpu(), rtol=1e-5)
        assert (y[6] == 0).all()
        if kind == "rows":   # finite rows do not mind the others
            keep = [0, 5, 7, 8]
            check_form(lowbit.rms_norm(x[keep], w).rows, (x[keep].double() * n.root[keep].double()[:, None] * w.double()).cpu().numpy(), "rows")
        else:
            assert not d[[0, 5, 7, 8]].isnan().any()


def test_empty():
    w = torch.ones(40, device="cuda")
    for rows, cols in ((0, 40), (3, 0), (0, 0)):
        x = torch.zeros(rows, cols, device="cuda")
        n = lowbit.rms_norm(x, w[:cols], x.clone(), rows=True, cols=True, y=True, root=True)
        assert n.rows.codes.shape[0] == rows and n.y.shape == x.shape
        dx, dw = lowbit.rms_norm_backward(x, x, torch.zeros(rows, device="cuda"), w[:cols], x)
        assert dx.shape == x.shape and (dw == 0).all()


# ---- gradients ----------------------------------------------------------------------------
# dx: the mean of g h s is a sum of products of three roundings each: (86 + 5) u of the mean of sizes; the rest six roundings of the terms' sizes, and the result's own.
# dw: `rows` products of two roundings in chains of at most `rows` + 40.
def check_backward(dy, h, root, w, dh, got):
    dy, h, w, s = dy.double().cpu().numpy(), h.double().cpu().numpy(), w.double().cpu().numpy(), root.double().cpu().numpy()[:, None]
    e = np.zeros_like(h) if dh is None else dh.double().cpu().numpy()
    g, n = dy * w, h * s
    mean, size = (g * n).mean(1, keepdims=True), np.abs(g * n).mean(1, keepdims=True)
    want = e + s * (g - n * mean)
    tol = np.abs(s * n) * 91 * U * size + 6 * U * (np.abs(e) + s * (np.abs(g) + np.abs(n) * size))
    dx, dw = got
    half = torch.finfo(dx.dtype).eps / 2
    off = np.abs(dx.double().cpu().numpy() - want)
    assert (off <= tol * (1 + half) + half * np.abs(want) + 1e-38).all(), (off - tol - half * np.abs(want)).max()
    if dw is not None:
        assert (np.abs(dw.double().cpu().numpy() - (dy * n).sum(0)) <= (h.shape[0] + 42) * U * np.abs(dy * n).sum(0) + 1e-38).all()


@pytest.mark.parametrize("types", [(BF16, BF16), (BF16, F32), (F32, BF16), (F32, F32)], ids=lambda t: "_".join(str(x)[6:] for x in t))
@pytest.mark.parametrize("rows,cols", SIZES + [(1000, 300), (2000, 1500)])
@pytest.mark.parametrize("add", [False, True])
def test_backward(rows, cols, types, add):
    h, dy, w = make(rows, cols, types[1], 1), make(rows, cols, types[0], 2, 1e-3), make(1, cols, BF16 if cols % 2 else F32, 3)[0]
    dh = make(rows, cols, types[1], 4, 1e-3) if add else None
    root = lowbit.rms_norm(h, w, rows=False, root=True).root
    check_backward(dy, h, root, w, dh, lowbit.rms_norm_backward(dy, h, root, w, dh))


@pytest.mark.parametrize("pad,offset", [(1, 0), (4, 4), (3, 1)])
def test_backward_strides(pad, offset):
    for rows, cols in ((5, 640), (130, 1021)):
        h, dy, dh = (make(rows, cols, BF16, i, 0.1, pad, offset) for i in (1, 2, 3))
        w = make(1, cols, BF16, 3, pad=pad, offset=offset)[0]
        root = lowbit.rms_norm(h, w, rows=False, root=True).root
        check_backward(dy, h, root, w, dh, lowbit.rms_norm_backward(dy, h, root, w, dh))
        check_backward(dy, h, root, w, None, lowbit.rms_norm_backward(dy, h, root, w, need_weight=False))


def test_backward_against_differences():
    """Along random directions, in 64 bits: the formula's gradient is that of the formula (the kernel is held to it above)."""
    g = torch.Generator().manual_seed(0)
    h, w, dy = (torch.randn(s, generator=g, dtype=torch.float64) for s in ((4, 60), (60,), (4, 60)))
    loss = lambda h, w: (h / (h.square().mean(1, keepdim=True) + 1e-6).sqrt() * w * dy).sum()  # noqa: E731
    root = 1 / (h.square().mean(1) + 1e-6).sqrt()
    dx, dw = lowbit.rms_norm_backward(dy.float().cuda(), h.float().cuda(), root.float().cuda(), w.float().cuda())
    a, b = torch.randn(4, 60, generator=g, dtype=torch.float64), torch.randn(60, generator=g, dtype=torch.float64)
    t = 1e-5
    want = (loss(h + t * a, w + t * b) - loss(h - t * a, w - t * b)) / (2 * t)
    got = (dx.double().cpu() * a).sum() + (dw.double().cpu() * b).sum()
    assert abs(got - want) < 1e-5 * (dx.double().cpu().abs() * a.abs()).sum()


def test_results_do_not_depend_on_timing_and_may_be_captured():
    x, r, dy, w = make(3000, 1100, BF16, 1), make(3000, 1100, F32, 2), make(3000, 1100, BF16, 3), make(1, 1100, F32, 4)[0]

    def run():
        n = lowbit.rms_norm(x, w, r, rows=True, cols=True, root=True)
        return [n.total, n.root, n.rows.codes[:, :1100], n.cols.codes[:, :1100], n.rows.scales, n.cols.scales, *lowbit.rms_norm_backward(dy, n.total, n.root, w, n.total)]

    want = run()
    assert all(torch.equal(a, b) for a, b in zip(want, run()))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run()
    for _ in range(2):
        for t in got:
            t.zero_()
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_streams():
    """A norm, its gradients and their temporary memory on a stream of their own."""
    x, w, dy = make(2000, 4096, BF16, 1), make(1, 4096, F32, 2)[0], make(2000, 4096, BF16, 3)
    n = lowbit.rms_norm(x, w, root=True)
    want = lowbit.rms_norm_backward(dy, x, n.root, w)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for _ in range(20):
            m = lowbit.rms_norm(x, w, root=True)
            got = lowbit.rms_norm_backward(dy, x, m.root, w)
    for _ in range(20):
        again = lowbit.rms_norm_backward(dy, x, n.root, w)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) and torch.equal(a, c) for a, b, c in zip(want, got, again))
    assert torch.equal(m.rows.codes, n.rows.codes)


def test_refusals():
    x, w = make(4, 256, BF16, 1), make(1, 256, F32, 2)[0]
    bad = [dict(residual=make(4, 255, BF16, 1)), dict(residual=make(5, 256, BF16, 1)), dict(residual=make(4, 256, BF16, 1).half()), dict(total=x.clone()), dict(root=torch.zeros(3, device="cuda")),
           dict(residual=x.clone(), total=x.float()), dict(y=x.float()), dict(residual=x.cpu()), dict(root=torch.zeros(4, device="cuda", dtype=BF16)),
           dict(rows=lowbit.Fp8Matrix.empty(4, 256, lowbit.COLS)), dict(cols=lowbit.Fp8Matrix.empty(4, 255, lowbit.COLS))]
    for arguments in bad:
        with pytest.raises(ValueError):
            lowbit.rms_norm(x, w, **arguments)
    for a, b in ((x.T, w[:4]), (x, w[:255]), (x.half(), w), (x, w.half()), (x.cpu(), w), (x[0], w), (x.float(), w.cpu())):
        with pytest.raises(ValueError):
            lowbit.rms_norm(a, b)
    with pytest.raises(ValueError):
        lowbit.rms_norm(x.float(), w, x)       # a stream in fewer bits than x
    root = torch.ones(4, device="cuda")
    for arguments in ((x[:3], x, root, w), (x, x, root[:3], w), (x, x, root, w[:200]), (x.half(), x, root, w), (x, x, root, w, x.float()), (x, x, root.bfloat16(), w)):
        with pytest.raises(ValueError):
            lowbit.rms_norm_backward(*arguments)
    with pytest.raises(ozk.OzkError):
        lowbit.rms_norm(torch.zeros(1, 32769, device="cuda"), torch.zeros(32769, device="cuda"))
