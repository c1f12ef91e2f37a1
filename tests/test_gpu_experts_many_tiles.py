"""Products by expert where pairs of CTAs take several tiles each and FP32 sums several ranges of K, with more experts than a warp has lanes; answers of few rows beside those of many."""
import numpy as np
import pytest
import torch

from paper_2608_06812_b200 import lowbit
from tests.test_gpu_experts import BF16, F32, check_rows, check_segments, experts_of, offsets_of, segments_of
from tests.test_gpu_fp8_gemm import random_matrix

pytestmark = pytest.mark.gpu


# 74 pairs: 9 tiles of lines times 12, 10 and 14 tiles of rows
@pytest.mark.parametrize("over", [False, True], ids=["forward", "dgrad"])
@pytest.mark.parametrize("counts,n,k", [([300] * 6, 2100, 8400), ([250, 1, 449, 0, 300, 250], 2100, 17000), ([230] * 7, 2050, 16384)])
def test_several_ranges_and_rounds(counts, n, k, over):
    rows = sum(counts) + 5
    a, w, offsets = random_matrix(rows, k, "rows", 3), experts_of(len(counts), *((k, n) if over else (n, k)), seed=4), offsets_of(counts, 2)
    out = torch.full((rows, n + 3), -7.0, device="cuda")[:, 1:n + 1]
    check_rows(lowbit.grouped_matmul(a, w, offsets, out=out, over_rows=over), a, w, offsets, over, -7.0)
    check_rows(lowbit.grouped_matmul(a, w, offsets, over_rows=over), a, w, offsets, over, 0.0)
    lowbit.check_async()


@pytest.mark.parametrize("counts,m,n", [([9000, 100, 8300], 1300, 1290), ([8192, 8193, 40, 0], 1290, 1100)])
def test_several_ranges_and_rounds_of_segments(counts, m, n):
    (a, A), (b, B), offsets = segments_of(counts, 3, 1, m, 1), segments_of(counts, 3, 1, n, 2), offsets_of(counts, 3)
    check_segments(lowbit.grouped_matmul(a, b, offsets, dtype=F32), A, B)
    out = torch.randn(len(counts), m, n, generator=torch.Generator().manual_seed(3)).mul(100).cuda()
    before = out.double().cpu().numpy()
    check_segments(lowbit.grouped_matmul(a, b, offsets, out=out, accumulate=True), A, B, before)
    lowbit.check_async()


@pytest.mark.parametrize("experts", [33, 100, 256])
def test_more_experts_than_lanes_in_tiles_of_many_rows(experts):
    g = np.random.default_rng(experts)
    counts = [int(c) for c in g.integers(0, 150, experts)]
    counts[3] = counts[experts // 2] = 0
    counts[-1] += max(0, 65 * experts - sum(counts))   # above 64 rows an expert: pairs of CTAs
    a, w, offsets = random_matrix(sum(counts) + 40, 200, "rows", 1), experts_of(experts, 300, 200, 2), offsets_of(counts, 20)
    for dtype in (BF16, F32):
        check_rows(lowbit.grouped_matmul(a, w, offsets, dtype=dtype), a, w, offsets, False, 0.0)
    (p, P), (q, Q) = segments_of(counts, 20, 20, 64, 1), segments_of(counts, 20, 20, 90, 2)
    check_segments(lowbit.grouped_matmul(p, q, offsets), P, Q)
    lowbit.check_async()


@pytest.mark.parametrize("experts,n,k", [(8, 512, 256), (8, 256, 512), (3, 300, 2000)])
def test_rows_answered_alone_and_together(experts, n, k):
    """Each row with all the others and by itself, whose kernels and divisions of K differ: the same operands, both within the bound of one sum."""
    rows = 70 * experts
    a, w, offsets = random_matrix(rows, k, "rows", 1), experts_of(experts, n, k, 2), offsets_of([70] * experts)
    for dtype in (BF16, F32):
        check_rows(lowbit.grouped_matmul(a, w, offsets, dtype=dtype), a, w, offsets, False)
        for row in (0, 69, 70, rows // 2, rows - 1):
            e = row // 70
            one = lowbit.Fp8Matrix(a.codes[row:row + 1].clone(), a.scales[:, row:row + 1].contiguous(), 1, k, lowbit.ROWS)
            alone = torch.tensor([0] * (e + 1) + [1] * (experts - e), dtype=torch.int32, device="cuda")
            check_rows(lowbit.grouped_matmul(one, w, alone, dtype=dtype), one, w, alone, False)
    lowbit.check_async()
