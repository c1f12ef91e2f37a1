"""The differentiable layers (norm and projection, experts) against the formulas, and the operators together as a model uses them.

The gradients are compared with those of the same network on the values that the 8-bit forms stand for: what each product gets is known exactly, so that the only differences
are FP32 sums (bounded as in the products' own tests by (K / 32 + 33) 2^-23 of the sums of sizes, here taken over the whole 2-norm) and the roundings of the results.
"""
import os
import sys

import pytest
import torch

from paper_2608_06812_b200 import lowbit

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

F32, BF16 = torch.float32, torch.bfloat16


def rand(*shape, seed=0, dtype=F32, scale=1.0):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).mul(scale).to(dtype).cuda()


def near(got, want, dtype, extra=0.0):
    """2-norm: half a step of the type, and the sums' 2^-17 (K / 32 + 33 <= 64 at the sizes here)."""
    half = torch.finfo(dtype).eps / 2
    assert torch.linalg.norm(got.double() - want.double()) <= (half + 2.0 ** -17 + extra) * torch.linalg.norm(want.double())


def by_rows(x):
    return lowbit.quantize_lines(x)[0].dequantize().double()


def by_cols(x):
    return lowbit.quantize_lines(x, False, True)[1].dequantize().double()


@pytest.mark.parametrize("dtype,stream", [(F32, None), (F32, F32), (BF16, BF16), (BF16, F32), (BF16, None)])
@pytest.mark.parametrize("tokens,inputs,outputs", [(5, 130, 70), (300, 512, 200)])
def test_norm_linear(tokens, inputs, outputs, dtype, stream):
    x, nw, w = rand(tokens, inputs, seed=1, dtype=dtype).requires_grad_(), (1 + rand(inputs, seed=2, scale=0.1)).requires_grad_(), rand(outputs, inputs, seed=3, scale=0.05).requires_grad_()
    r = None if stream is None else rand(tokens, inputs, seed=4, dtype=stream).requires_grad_()
    y, total = lowbit.norm_linear(x, nw, w, r)
    dy, dt = rand(tokens, outputs, seed=5, dtype=dtype), rand(tokens, inputs, seed=6, dtype=total.dtype)
    leaves = [x, nw, w] + ([] if r is None else [r])
    grads = torch.autograd.grad([y, total] if r is not None else [y], leaves, [dy, dt] if r is not None else [dy])
    # the formula, on the values of the 8-bit forms
    h = total.detach()
    n = lowbit.rms_norm(h, nw.detach(), rows=True, cols=True, root=True)
    w8 = lowbit.quantize_tiles(w.detach()).dequantize().double()
    near(y, n.rows.dequantize().double() @ w8.T, dtype)
    dn = (by_rows(dy) @ w8)
    s, hd, nwd = n.root.double()[:, None], h.double(), nw.detach().double()
    g = dn * nwd
    dx = s * (g - hd * s * (g * hd * s).mean(1, keepdim=True)) + (dt.double() if r is not None else 0.0)
    half = torch.finfo(dtype).eps / 2    # dn is rounded to the type of x on its way
    near(grads[0], dx, dtype, half + (torch.finfo(h.dtype).eps / 2))
    near(grads[1], (dn * hd * s).sum(0), F32, half)
    near(grads[2], by_cols(dy).T @ n.cols.dequantize().double(), F32)
    if r is not None:
        near(grads[3], dx, h.dtype, half)
        assert total.dtype == stream and torch.equal(total, (x.float() + r.float()).to(stream))
    else:
        assert total is x
    lowbit.check_async()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("counts,behind", [([3, 0, 40, 1], 2), ([200, 130, 0, 70], 0), ([0, 0, 5, 0], 300)])
def test_expert_linear(counts, behind, dtype):
    rows, inputs, outputs = sum(counts) + behind, 260, 130
    offsets = torch.tensor([0, *torch.tensor(counts).cumsum(0).tolist()], dtype=torch.int32, device="cuda")
    x, w = rand(rows, inputs, seed=1, dtype=dtype).requires_grad_(), rand(len(counts), outputs, inputs, seed=2, scale=0.05).requires_grad_()
    y = lowbit.expert_linear(x, w, offsets)
    dy = rand(rows, outputs, seed=3, dtype=dtype)
    dx, dw = torch.autograd.grad(y, (x, w), dy)
    w8 = lowbit.quantize_experts(w.detach()).dequantize().double()
    x8, dy8 = by_rows(x.detach()), by_rows(dy)
    for e, (b, f) in enumerate(zip(offsets.tolist(), offsets.tolist()[1:])):
        if b == f:
            assert (dw[e] == 0).all()
            continue
        near(y[b:f], x8[b:f] @ w8[e].T, dtype)
        near(dx[b:f], dy8[b:f] @ w8[e], dtype)
        near(dw[e], by_cols(dy[b:f]).T @ by_cols(x.detach()[b:f]), F32)
    for t in (y, dx):
        assert (t[sum(counts):] == 0).all()   # rows of nobody
    lowbit.check_async()


def test_only_what_is_wanted():
    x, nw, w, r = rand(40, 128, seed=1), rand(128, seed=2).abs(), rand(64, 128, seed=3), rand(40, 128, seed=4)
    for wanted in ([0], [1], [2], [3], [0, 3], [1, 2]):
        leaves = [t.clone().requires_grad_(i in wanted) for i, t in enumerate((x, nw, w, r))]
        y, total = lowbit.norm_linear(*leaves)
        (y.square().sum() + total.sum()).backward()
        assert [i for i, t in enumerate(leaves) if t.grad is not None] == wanted
    leaves = [t.clone().requires_grad_() for t in (x, nw, w, r)]
    _, total = lowbit.norm_linear(*leaves)
    total.square().sum().backward()          # the stream alone
    assert torch.equal(leaves[0].grad, 2 * (x + r)) and torch.equal(leaves[3].grad, leaves[0].grad) and leaves[2].grad is None
    with torch.no_grad():
        kept = lowbit.quantize_tiles(w)
        y, total = lowbit.norm_linear(x, nw, w, r, w8=kept)
    assert torch.equal(y, lowbit.norm_linear(x, nw, w, r)[0]) and not y.requires_grad
    offsets = torch.tensor([0, 10, 40], dtype=torch.int32, device="cuda")
    we = rand(2, 64, 128, seed=5)
    for wanted in ([0], [1], []):
        leaves = [t.clone().requires_grad_(i in wanted) for i, t in enumerate((x, we))]
        y = lowbit.expert_linear(*leaves, offsets)
        assert y.requires_grad == bool(wanted)
        if wanted:
            y.sum().backward()
        assert [i for i, t in enumerate(leaves) if t.grad is not None] == wanted


def test_gradients_of_leaves_that_are_used_twice():
    """The same weights and stream twice in one graph: gradients add up and do not write into each other."""
    x, nw, w = rand(70, 128, seed=1).requires_grad_(), (1 + rand(128, seed=2, scale=0.1)).requires_grad_(), rand(128, 128, seed=3, scale=0.05).requires_grad_()
    y, total = lowbit.norm_linear(x, nw, w, x)
    z, total = lowbit.norm_linear(y, nw, w, total)
    grads = torch.autograd.grad(z.square().sum() + total.sum(), (x, nw, w))
    again = [t.detach().clone().requires_grad_() for t in (x, nw, w)]
    y, total = lowbit.norm_linear(again[0], again[1], again[2], again[0])
    z, total = lowbit.norm_linear(y, again[1], again[2], total)
    (z.square().sum() + total.sum()).backward()
    assert all(torch.equal(a, b.grad) for a, b in zip(grads, again))


def test_writes_between_the_passes_are_noticed():
    x, nw, w, r = (rand(*s, seed=i) for i, s in enumerate(((9, 128), (128,), (64, 128), (9, 128))))
    w.requires_grad_()
    offsets, we = torch.tensor([0, 3, 9], dtype=torch.int32, device="cuda"), rand(2, 64, 128, seed=5).requires_grad_()
    kept, kept_experts = lowbit.quantize_tiles(w.detach()), lowbit.quantize_experts(we.detach())
    leaf = x.clone().requires_grad_()
    y, total = lowbit.norm_linear(leaf, nw, w, r, w8=kept)
    lowbit.rms_norm(x, nw, total.detach(), rows=False, total=total.detach())   # the saved stream written over
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()
    y, _ = lowbit.norm_linear(leaf, nw, w, r, w8=kept)
    lowbit.quantize_tiles(w.detach() * 2, out=kept)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()
    y = lowbit.expert_linear(leaf, we, offsets, kept_experts)
    lowbit.quantize_experts(we.detach() * 2, out=kept_experts)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()
    y = lowbit.expert_linear(leaf, we, offsets)
    offsets.copy_(torch.tensor([0, 4, 9], dtype=torch.int32))
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


def test_a_captured_step():
    """Forward and backward pass of both layers in one graph, with new inputs and new offsets at each replay."""
    x, r, nw, w, we = rand(96, 128, seed=1), rand(96, 128, seed=2), 1 + rand(128, seed=3, scale=0.1), rand(128, 128, seed=4, scale=0.1), rand(3, 64, 128, seed=5, scale=0.1)
    offsets = torch.tensor([0, 30, 30, 96], dtype=torch.int32, device="cuda")

    def step():
        leaves = [t.detach().requires_grad_() for t in (x, nw, w, we, r)]
        h, total = lowbit.norm_linear(leaves[0], leaves[1], leaves[2], leaves[4])
        y = lowbit.expert_linear(h, leaves[3], offsets)
        return [y, total, *torch.autograd.grad(y.square().sum() + total.sum(), leaves)]

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for seed, cuts in ((7, [0, 30, 30, 96]), (8, [0, 1, 95, 96]), (9, [0, 0, 0, 96])):
        x.copy_(rand(96, 128, seed=seed))
        offsets.copy_(torch.tensor(cuts, dtype=torch.int32))
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(got, step()))
    lowbit.check_async()


def test_the_example_runs():
    import train_experts_8bit as example
    plain, eight, off = example.main(4)
    assert len(plain) == len(eight) == 4 and all(torch.isfinite(torch.tensor(eight)))
    assert off == off


def test_the_example_in_eight_bits_has_the_gradients_of_the_one_in_32():
    """Codes of three fraction bits: each operand of a product is off by at most 2^-4 of its value, so that after four products in a row, their gradients included, directions agree
    far beyond chance and sizes to a quarter.  Routes must agree for that: one expert for all rows here."""
    import train_experts_8bit as example
    p = {k: v.requires_grad_() for k, v in example.parameters(3).items() if k != "router"}
    x, stream = rand(128, example.WIDTH, seed=1), rand(128, example.WIDTH, seed=2)
    offsets = torch.tensor([0] + [128] * example.EXPERTS, dtype=torch.int32, device="cuda")

    def grads(norm_linear, expert_linear):
        h, total = norm_linear(x, p["norm"], p["project"], stream)
        y = total + expert_linear(torch.relu(expert_linear(h, p["up"], offsets)), p["down"], offsets)
        return torch.autograd.grad(y.square().mean(), list(p.values()))

    plain, eight = grads(example.plain_norm_linear, example.plain_expert_linear), grads(lowbit.norm_linear, lowbit.expert_linear)
    for a, b in zip(plain, eight):
        assert torch.nn.functional.cosine_similarity(a.reshape(-1), b.reshape(-1), 0) > 0.97 and 0.75 < float(b.norm() / a.norm()) < 1.25


@pytest.mark.parametrize("operator", ["norm", "experts", "segments"])
def test_threads_and_streams(operator):
    """Two host threads, each on a stream of its own and first with CUDA there, at the same time."""
    import threading
    x, nw = rand(500, 512, seed=1, dtype=BF16), rand(512, seed=2).abs()
    offsets, w = torch.tensor([0, 100, 500], dtype=torch.int32, device="cuda"), lowbit.quantize_experts(rand(2, 300, 512, seed=3))

    def once():
        if operator == "norm":
            n = lowbit.rms_norm(x, nw, rows=True, cols=True, root=True)
            dx, dw = lowbit.rms_norm_backward(x, x, n.root, nw, x)
            return [n.rows.codes, n.cols.codes, dx, dw]
        if operator == "experts":
            return [lowbit.grouped_matmul(lowbit.quantize_lines(x)[0], w, offsets), lowbit.grouped_matmul(lowbit.quantize_lines(x[:8])[0], w, offsets.clamp(max=8))]
        s = lowbit.quantize_segments(x, offsets)[1]
        return [lowbit.grouped_matmul(s, s, offsets, dtype=F32)]

    want = once()
    torch.cuda.synchronize()
    found, errors, start = [None, None], [], threading.Barrier(2)

    def work(i):
        try:
            start.wait(60)
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(30):
                    found[i] = once()
                torch.cuda.current_stream().synchronize()
        except Exception as e:  # noqa: BLE001  (shown by the main thread)
            errors.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors
    assert all(torch.equal(a, b) for f in found for a, b in zip(want, f))
    lowbit.check_async()
