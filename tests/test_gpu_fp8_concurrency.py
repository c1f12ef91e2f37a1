"""Products whose sums pass through device memory (K split over pairs of CTAs, joined by a second launch) beside each other: from two host
threads on one stream, from graphs captured on one stream and replayed on two, from graphs beside eager calls."""
import threading

import pytest
import torch

from paper_2608_06812_b200 import binding as ozk
from paper_2608_06812_b200 import lowbit
from tests.test_gpu_fp8_gemm import check, operands

pytestmark = pytest.mark.gpu

# (way, m, n, k, FP32 scales)
SPLIT = [("forward", 512, 2048, 8192, True), ("wgrad", 256, 256, 40000, False)]


def job(i, seed):
    way, m, n, k, floats = SPLIT[i]
    a, b, over = operands(way, m, n, k, seed, floats)
    x = (a.cols, a.rows) if a.kind == "cols" else (a.rows, a.cols)
    plan = ozk.ozk_fp8_gemm_plan(x[0], n, x[1], a._operand[a.kind == "cols"], b._operand[b.kind == "cols"], ozk.OZK_F32)
    assert plan.pairs and plan.splits > 1 and plan.scratch_bytes > 0
    return a, b, over


def product(j, out=None):
    return lowbit.matmul(j[0], j[1], out=out, over_rows=j[2], dtype=torch.float32)


@pytest.mark.parametrize("i", [0, 1])
def test_two_threads_on_one_stream(i):
    jobs = [job(i, 10), job(i, 20)]
    want = [product(j) for j in jobs]
    check(want[0], *jobs[0])
    torch.cuda.synchronize()
    wrong, errors, start = [0, 0], [], threading.Barrier(2)

    def work(t):
        try:
            start.wait(60)
            for _ in range(8):
                got = [product(jobs[t]) for _ in range(25)]
                wrong[t] += sum(not torch.equal(c, want[t]) for c in got)
        except Exception as e:  # noqa: BLE001  (shown by the main thread)
            errors.append(e)

    threads = [threading.Thread(target=work, args=(t,)) for t in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors and wrong == [0, 0]
    lowbit.check_async()


def test_graphs_of_one_stream_on_two_and_eager_calls_beside_them():
    jobs = [job(0, 30), job(0, 40), job(1, 50)]
    want = [product(j) for j in jobs]
    s, outs, graphs = torch.cuda.Stream(), [torch.zeros_like(w) for w in want[:2]], []
    s.wait_stream(torch.cuda.current_stream())
    for j, c in zip(jobs, outs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            product(j, c)
        graphs.append(g)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(20):
        for c in outs:
            c.zero_()
        torch.cuda.synchronize()
        for _ in range(3):
            for g, r in zip(graphs, streams):
                with torch.cuda.stream(r):
                    g.replay()
            with torch.cuda.stream(s):
                eager = product(jobs[2])
        torch.cuda.synchronize()
        assert all(torch.equal(w, c) for w, c in zip(want, [*outs, eager]))


def test_a_first_product_on_a_stream_may_be_captured():
    a, b, over = operands("forward", 20, 300, 700, 9)
    want = lowbit.matmul(a, b)
    out = torch.zeros_like(want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        lowbit.matmul(a, b, out=out)
    g.replay()
    assert torch.equal(out, want)


def test_check_async_names_a_device_in_every_way():
    a, b, over = operands("forward", 20, 300, 700, 9)
    lowbit.matmul(a, b)
    for device in (None, 0, "cuda", "cuda:0", torch.device("cuda"), torch.device("cuda", 0)):
        lowbit.check_async(device)
