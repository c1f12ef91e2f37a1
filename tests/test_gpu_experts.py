"""Products grouped by expert against 64-bit sums of the same scaled values, with the bound of an FP32 sum on the tensor cores that the tests
of the product with one matrix derive: (K / 32 + 33) units of 2^-23 of the sum of sizes.
"""
import numpy as np
import pytest
import torch

from oracle import lowbit as ref
from paper_2608_06812_b200 import binding as ozk
from paper_2608_06812_b200 import lowbit
from tests.test_gpu_fp8_gemm import random_matrix, values

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def experts_of(n, rows, cols, seed):
    """Random codes (no NaN), scales over 12 binades, in a buffer with NaN codes between what belongs to the experts."""
    g = torch.Generator().manual_seed(seed)
    ld = -(-max(cols, 1) // 16) * 16 + 16 * (seed % 2)
    codes = torch.randint(0, 256, (n, rows + seed % 3, ld), generator=g, dtype=torch.uint8)
    codes[(codes & 0x7F) == 0x7F] = 0x3A
    codes[:, rows:] = 0x7F
    codes[:, :, cols:] = 0x7F
    scales = torch.randint(115, 128, (n, -(-rows // 128), -(-cols // 128)), generator=g, dtype=torch.uint8)
    return lowbit.Fp8Experts(codes.cuda()[:, :rows], scales.cuda(), rows, cols)


def expert_values(w):
    codes, s = ref.decode(w.codes.cpu().numpy()[:, :, :w.cols]), w.scales.cpu().numpy().astype(np.float64) - 127.0
    return np.stack([c * 2.0 ** ref.spread(e, c.shape, "tiles") for c, e in zip(codes, s)]) if w.experts else codes.astype(np.float64)


def offsets_of(counts, first=0):
    return torch.tensor(np.cumsum([first, *counts]), dtype=torch.int32, device="cuda")


def within(got, want, size, k):
    tol = (k / 32 + 33) * 2.0 ** -23 * size
    low, high = want - tol, want + tol
    if got.dtype == BF16:
        low, high = (torch.from_numpy(x).bfloat16().double().numpy() for x in (low, high))
    got = got.double().cpu().numpy()
    bad = ~((got >= low) & (got <= high))
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4], np.abs(got - want).max())


def check_rows(c, a, w, offsets, over, rest=None):
    A, W, off = values(a), expert_values(w), offsets.tolist()
    covered = np.zeros(a.rows, bool)
    for e, (b, f) in enumerate(zip(off, off[1:])):
        B = W[e] if over else W[e].T
        if f > b:
            within(c[b:f], A[b:f] @ B, np.abs(A[b:f]) @ np.abs(B), a.cols)
        covered[b:f] = True
    if rest is not None:
        assert (c[torch.from_numpy(~covered).cuda()] == rest).all()


# counts of rows, first row, rows behind the last segment
COUNTS = [([1], 0, 0), ([0, 1, 0], 0, 0), ([5, 0, 3], 2, 4), ([32, 33, 31], 0, 0), ([64, 65, 1, 0, 127, 128, 129], 1, 1), ([224, 225, 223], 0, 0), ([0, 0], 3, 2), ([300, 7, 449, 0, 2], 5, 100),
          ([1] * 40, 0, 0), ([3, 0] * 33, 0, 7), ([1000], 0, 0), ([4000, 10], 0, 0)]


@pytest.mark.parametrize("over", [False, True], ids=["forward", "dgrad"])
@pytest.mark.parametrize("counts,first,behind", COUNTS, ids=[str(i) for i in range(len(COUNTS))])
@pytest.mark.parametrize("n,k", [(1, 1), (16, 128), (130, 300), (300, 520), (520, 1100), (255, 640)])
def test_rows(counts, first, behind, n, k, over):
    rows = first + sum(counts) + behind
    a = random_matrix(rows, k, "rows", rows + n)
    w = experts_of(len(counts), *((k, n) if over else (n, k)), seed=n + k)
    offsets = offsets_of(counts, first)
    for dtype in (BF16, F32):
        check_rows(lowbit.grouped_matmul(a, w, offsets, over_rows=over, dtype=dtype), a, w, offsets, over, 0.0)
        out = torch.full((rows, n), -7.0, dtype=dtype, device="cuda")
        got = lowbit.grouped_matmul(a, w, offsets, out=out, over_rows=over)
        assert got.data_ptr() == out.data_ptr()
        check_rows(out, a, w, offsets, over, -7.0)
    lowbit.check_async()


@pytest.mark.parametrize("dtype,pad", [(BF16, 1), (BF16, 2), (BF16, 3), (BF16, 8), (F32, 1), (F32, 4)])
def test_strided_results_leave_their_surroundings(dtype, pad):
    for counts, n, k in (([3, 40, 0, 9], 200, 256), ([300, 100], 333, 512), ([1], 77, 2000)):
        rows = sum(counts)
        a, w, offsets = random_matrix(rows, k, "rows", 5), experts_of(len(counts), n, k, 6), offsets_of(counts)
        whole = torch.full((rows + 2, n + 2 * pad), -7.0, dtype=dtype, device="cuda")
        out = whole[1:1 + rows, pad:pad + n]
        lowbit.grouped_matmul(a, w, offsets, out=out)
        check_rows(out, a, w, offsets, False)
        out.fill_(-7.0)
        assert (whole == -7.0).all()
    lowbit.check_async()


@pytest.mark.parametrize("over", [False, True])
@pytest.mark.parametrize("counts,n,k", [([700, 0, 20, 1300], 1000, 4096), ([4] * 16, 2048, 2048), ([100, 30, 60, 7], 700, 20000), ([3000, 2500, 1], 2100, 700), ([90] * 12, 500, 9000)])
def test_larger(counts, n, k, over):
    rows = sum(counts)
    a, w, offsets = random_matrix(rows, k, "rows", 3), experts_of(len(counts), *((k, n) if over else (n, k)), seed=4), offsets_of(counts)
    for dtype in (BF16, F32):
        check_rows(lowbit.grouped_matmul(a, w, offsets, over_rows=over, dtype=dtype), a, w, offsets, over)
    lowbit.check_async()


def test_one_expert_is_the_product_with_one_matrix():
    """Both lie within the bound of one sum; their bits may differ, because the other product joins ranges of K in its own order."""
    a, w, offsets = random_matrix(500, 1000, "rows", 1), experts_of(1, 700, 1000, 2), offsets_of([500])
    one = lowbit.Fp8Matrix(w.codes[0], w.scales[0].contiguous(), 700, 1000, lowbit.TILES)
    for c in (lowbit.grouped_matmul(a, w, offsets, dtype=F32), lowbit.matmul(a, one, dtype=F32)):
        check_rows(c, a, w, offsets, False)


def test_offsets_that_fall_or_leave_the_rows():
    """Read as the nearest that do not; nothing outside the operands is touched."""
    a, w = random_matrix(300, 256, "rows", 1), experts_of(4, 200, 256, 2)
    for bad, good in (([0, 100, 50, 400, 10], [0, 100, 100, 300, 300]), ([-5, 20, 20, 10 ** 9, -3], [0, 20, 20, 300, 300]), ([250, 0, 0, 260, 270], [250, 250, 250, 260, 270])):
        bad, good = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (bad, good))
        assert torch.equal(lowbit.grouped_matmul(a, w, bad), lowbit.grouped_matmul(a, w, good))
        check_rows(lowbit.grouped_matmul(a, w, good), a, w, good, False, 0.0)
        x = torch.randn(300, 70, generator=torch.Generator().manual_seed(1)).cuda()
        (p, q), (r, s) = lowbit.quantize_segments(x, good), lowbit.quantize_segments(x, bad)
        assert torch.equal(lowbit.grouped_matmul(q, q, good), lowbit.grouped_matmul(s, s, bad))
    lowbit.check_async()


# ---- quantisation -------------------------------------------------------------------------
def make(rows, cols, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g) * torch.randn(rows, 1, generator=g).exp()
    if rows > 2 and cols > 3:
        x[1, 2], x[2, 3], x[0] = float("nan"), float("inf"), 0.0
    return x.to(dtype).cuda()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("counts,first,behind", COUNTS, ids=[str(i) for i in range(len(COUNTS))])
@pytest.mark.parametrize("cols", [1, 100, 128, 520])
def test_quantize_segments(counts, first, behind, cols, dtype):
    rows, n = first + sum(counts) + behind, len(counts)
    x, offsets = make(rows, cols, dtype, rows + cols), offsets_of(counts, first)
    by_rows, by_cols = lowbit.Fp8Matrix.empty(rows, cols, lowbit.ROWS), lowbit.Fp8Segments.empty(rows, cols, n)
    for q in (by_rows, by_cols):
        q.codes.fill_(0x55)
        q.scales.fill_(9)
    got = lowbit.quantize_segments(x, offsets, by_rows, by_cols)
    assert got[0] is by_rows and got[1] is by_cols
    want = lowbit.quantize_lines(x)[0]
    inside = torch.zeros(rows, dtype=torch.bool, device="cuda")
    inside[first:first + sum(counts)] = True
    assert torch.equal(by_rows.codes[inside][:, :cols], want.codes[inside][:, :cols]) and torch.equal(by_rows.scales[:, inside], want.scales[:, inside])
    assert (by_rows.codes[~inside] == 0x55).all() and (by_rows.scales[:, ~inside] == 9).all()
    block = 0
    flat = by_cols.scales.transpose(1, 2).reshape(-1, cols)
    for b, f in zip(offsets.tolist(), offsets.tolist()[1:]):
        if f == b:
            continue
        q, blocks = lowbit.quantize_lines(x[b:f], False, True)[1], -(-(f - b) // 128)
        part = by_cols.codes[block * 128:(block + blocks) * 128]
        assert torch.equal(part[:f - b, :cols], q.codes[:, :cols]) and (part[f - b:, :cols] == 0).all()
        assert torch.equal(flat[block:block + blocks], q.scale_codes())
        block += blocks
    assert (by_cols.codes[block * 128:] == 0x55).all() and (flat[block:] == 9).all()
    assert (by_cols.codes[:, cols:] == 0x55).all()
    alone = lowbit.quantize_segments(x, offsets, False)
    assert alone[0] is None and torch.equal(alone[1].codes[:block * 128, :cols], by_cols.codes[:block * 128, :cols])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,rows,cols", [(1, 1, 1), (3, 100, 200), (5, 128, 128), (2, 300, 517), (7, 129, 64)])
def test_quantize_experts(n, rows, cols, dtype):
    whole = make(n * (rows + 1), cols + 3, dtype, 1).view(n, rows + 1, cols + 3)
    for w in (whole[:, :rows, :cols], whole[:, :rows, :cols].contiguous()):
        q = lowbit.quantize_experts(w)
        for e in range(n):
            one = lowbit.quantize_tiles(w[e])
            assert torch.equal(q.codes[e, :, :cols], one.codes[:, :cols]) and torch.equal(q.scales[e], one.scales)
            assert torch.equal(q.dequantize()[e].isnan(), one.dequantize().isnan()) and torch.equal(q.dequantize()[e].nan_to_num(), one.dequantize().nan_to_num())
        out = lowbit.Fp8Experts.empty(n, rows, cols)
        assert lowbit.quantize_experts(w, out) is out and torch.equal(out.scales, q.scales)


# ---- weight gradients -------------------------------------------------------------------
def segments_of(counts, first, behind, cols, seed):
    """Random codes and scales by segments, NaN codes in the blocks that nobody takes; and the values of each segment."""
    rows, n = first + sum(counts) + behind, len(counts)
    g = torch.Generator().manual_seed(seed)
    blocks = lowbit.segment_blocks(rows, n)
    codes = torch.full((blocks * 128, -(-cols // 16) * 16), 0x7F, dtype=torch.uint8)
    scales = torch.randint(115, 128, (-(-blocks // 4), cols, 4), generator=g, dtype=torch.uint8)
    found, b = [], 0
    for c in counts:
        part = torch.randint(0, 256, (c, cols), generator=g, dtype=torch.uint8)
        part[(part & 0x7F) == 0x7F] = 0x3A
        nb = -(-c // 128)
        codes[b * 128:(b + nb) * 128] = 0
        codes[b * 128:b * 128 + c, :cols] = part
        e = scales.transpose(1, 2).reshape(-1, cols)[b:b + nb].numpy().astype(np.float64) - 127.0
        found.append(ref.decode(part.numpy()) * 2.0 ** ref.spread(e, (c, cols), "cols"))
        b += nb
    return lowbit.Fp8Segments(codes.cuda(), scales.cuda(), rows, cols, n), found


def check_segments(c, A, B, before=None):
    for e, (a, b) in enumerate(zip(A, B)):
        want, size = a.T @ b, np.abs(a).T @ np.abs(b)
        if before is not None:
            want, size = want + before[e], size + np.abs(before[e])
        within(c[e], want, size, a.shape[0])


@pytest.mark.parametrize("counts,first,behind", COUNTS + [([128 * 5, 128 * 3, 1, 128 * 70, 300], 0, 0), ([9000, 0, 8300], 7, 9)], ids=[str(i) for i in range(len(COUNTS) + 2)])
@pytest.mark.parametrize("m,n", [(1, 1), (16, 130), (257, 300), (300, 64)])
def test_segments(counts, first, behind, m, n):
    a, A = segments_of(counts, first, behind, m, 1)
    b, B = segments_of(counts, first, behind, n, 2)
    offsets = offsets_of(counts, first)
    for dtype in (BF16, F32):
        check_segments(lowbit.grouped_matmul(a, b, offsets, dtype=dtype), A, B)
    for pad in (0, 1, 4):
        whole = torch.randn(len(counts), m + pad, n + 2 * pad, generator=torch.Generator().manual_seed(3)).mul(100).cuda()
        out, kept = whole[:, :m, pad:pad + n], whole.clone()
        before = out.double().cpu().numpy()
        lowbit.grouped_matmul(a, b, offsets, out=out, accumulate=True)
        check_segments(out, A, B, before)
        out.copy_(kept[:, :m, pad:pad + n])
        assert torch.equal(whole, kept)
    lowbit.check_async()


@pytest.mark.parametrize("counts,m,n", [([2000, 0, 900, 40], 1500, 700), ([600] * 8, 512, 1024)])
def test_larger_segments(counts, m, n):
    (a, A), (b, B), offsets = segments_of(counts, 0, 0, m, 1), segments_of(counts, 0, 0, n, 2), offsets_of(counts)
    check_segments(lowbit.grouped_matmul(a, b, offsets, dtype=F32), A, B)
    check_segments(lowbit.grouped_matmul(a, b, offsets), A, B)
    lowbit.check_async()


def test_nothing():
    offsets = torch.zeros(4, dtype=torch.int32, device="cuda")
    assert lowbit.grouped_matmul(random_matrix(0, 64, "rows", 1), experts_of(3, 32, 64, 1), offsets).shape == (0, 32)
    c = lowbit.grouped_matmul(lowbit.Fp8Matrix.empty(9, 0, lowbit.ROWS), lowbit.Fp8Experts.empty(3, 32, 0), torch.tensor([1, 4, 4, 7], dtype=torch.int32, device="cuda"))
    assert c.shape == (9, 32) and (c == 0).all()
    out = torch.ones(9, 32, device="cuda")
    lowbit.grouped_matmul(lowbit.Fp8Matrix.empty(9, 0, lowbit.ROWS), lowbit.Fp8Experts.empty(3, 32, 0), torch.tensor([1, 4, 4, 7], dtype=torch.int32, device="cuda"), out=out)
    assert (out[1:7] == 0).all() and (out[0] == 1).all() and (out[7:] == 1).all()
    none = torch.zeros(1, dtype=torch.int32, device="cuda")
    assert (lowbit.grouped_matmul(random_matrix(5, 64, "rows", 1), lowbit.Fp8Experts.empty(0, 32, 64), none) == 0).all()
    empty = lowbit.Fp8Segments.empty(0, 24, 3)
    assert (lowbit.grouped_matmul(empty, empty, offsets, dtype=F32) == 0).all()
    assert lowbit.quantize_segments(torch.zeros(0, 24, device="cuda"), offsets)[1].codes.shape[0] == 0


def test_many_experts():
    counts = [(7 * e) % 5 for e in range(1024)]
    a, w, offsets = random_matrix(sum(counts), 130, "rows", 1), experts_of(1024, 40, 130, 2), offsets_of(counts)
    check_rows(lowbit.grouped_matmul(a, w, offsets, dtype=F32), a, w, offsets, False)
    (a, A), (b, B) = segments_of(counts, 0, 0, 24, 1), segments_of(counts, 0, 0, 40, 2)
    check_segments(lowbit.grouped_matmul(a, b, offsets, dtype=F32), A, B)
    with pytest.raises(ozk.OzkError):
        lowbit.grouped_matmul(random_matrix(9, 64, "rows", 1), experts_of(1025, 16, 64, 1), torch.zeros(1026, dtype=torch.int32, device="cuda"))


def test_graphs_take_the_offsets_of_each_replay():
    a, w, out = random_matrix(600, 700, "rows", 1), experts_of(3, 300, 700, 2), torch.zeros(600, 300, device="cuda")
    (p, P), (q, Q) = segments_of([200, 300, 100], 0, 0, 64, 1), segments_of([200, 300, 100], 0, 0, 90, 2)
    dw = torch.zeros(3, 64, 90, device="cuda")
    offsets = offsets_of([200, 300, 100])
    lowbit.grouped_matmul(a, w, offsets, out=out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lowbit.grouped_matmul(a, w, offsets, out=out)
        lowbit.grouped_matmul(p, q, offsets, out=dw)
    graph.replay()
    check_segments(dw, P, Q)
    for counts in ([200, 300, 100], [0, 0, 600], [599, 1, 0], [10, 20, 30]):
        offsets.copy_(offsets_of(counts))
        out.fill_(-7.0)
        graph.replay()
        check_rows(out, a, w, offsets, False, -7.0)
    lowbit.check_async()


def test_refusals():
    a, w, offsets = random_matrix(9, 64, "rows", 1), experts_of(3, 32, 64, 2), offsets_of([3, 3, 3])
    s = lowbit.Fp8Segments.empty(9, 64, 3)
    bad = [(a, w, offsets[:3]), (a, w, offsets.long()), (a, w, offsets.cpu()), (random_matrix(9, 65, "rows", 1), w, offsets), (random_matrix(9, 64, "cols", 1), w, offsets), (a, a, offsets), (s, w, offsets), (a, s, offsets),
           (s, lowbit.Fp8Segments.empty(8, 64, 3), offsets), (s, lowbit.Fp8Segments.empty(9, 64, 4), offsets), (random_matrix(9, 64, "rows", 1, True), w, offsets)]
    for arguments in bad:
        with pytest.raises(ValueError):
            lowbit.grouped_matmul(*arguments)
    for more in (dict(accumulate=True), dict(out=torch.zeros(9, 31, device="cuda")), dict(out=torch.zeros(9, 32)), dict(over_rows=True), dict(dtype=torch.float16), dict(out=torch.zeros(32, 9, device="cuda").T)):
        with pytest.raises(ValueError):
            lowbit.grouped_matmul(a, w, offsets, **more)
    for more in (dict(accumulate=True), dict(over_rows=True), dict(out=torch.zeros(3, 64, 63, device="cuda"))):
        with pytest.raises(ValueError):
            lowbit.grouped_matmul(s, s, offsets, **more)
    with pytest.raises(ozk.OzkError):
        lowbit.grouped_matmul(s, s, offsets, out=torch.zeros(3, 64, 64, device="cuda", dtype=BF16), accumulate=True)
    x = torch.zeros(9, 64, device="cuda")
    for arguments in ((x.T, offsets), (x, offsets.long()), (x, offsets, lowbit.Fp8Matrix.empty(9, 64, lowbit.COLS)), (x, offsets, True, lowbit.Fp8Segments.empty(9, 64, 2)), (x, offsets[0])):
        with pytest.raises(ValueError):
            lowbit.quantize_segments(*arguments)
    for arguments in ((x,), (torch.zeros(2, 3, 4, device="cuda").half(),), (torch.zeros(2, 3, 4),), (torch.zeros(2, 3, 4, device="cuda").transpose(1, 2),), (torch.zeros(2, 3, 4, device="cuda"), lowbit.Fp8Experts.empty(2, 3, 5))):
        with pytest.raises(ValueError):
            lowbit.quantize_experts(*arguments)
    with pytest.raises(ValueError):
        lowbit.Fp8Experts(torch.zeros(2, 3, 24, dtype=torch.uint8, device="cuda")[:, :, 8:], torch.zeros(2, 1, 1, dtype=torch.uint8, device="cuda"), 3, 16)
    with pytest.raises(ValueError):
        lowbit.Fp8Segments(torch.zeros(128, 16, dtype=torch.uint8, device="cuda"), torch.zeros(1, 16, 4, dtype=torch.uint8, device="cuda"), 200, 16, 2)
