"""The AdamW step against the formula in 64 bits.

FP32 bounds, from the roundings in the formula (u = 2^-24): the moments take two products and a sum, at most 3 u of the sum
of their terms' sizes; the update's quotient takes the moment, the root (half the moment's error and one rounding), a
product, a sum and a division, at most 10 u; the parameter two products and a difference: 3 u of its size plus 12 u of
the step's.  States in 8 bits may fall on the neighbouring code where those errors cross the middle of two.
"""
import numpy as np
import pytest
import torch

from oracle import lowbit as ref
from paper_2608_06812_b200 import binding as ozk
from paper_2608_06812_b200 import lowbit

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
OPTIONS = dict(lr=1e-2, betas=(0.9, 0.95), eps=1e-8, weight_decay=0.1)


def decode8(codes, scales, n):
    return ref.decode(codes.cpu().numpy()) * 2.0 ** (np.repeat(scales.cpu().numpy().astype(np.float64), 128)[:n] - 127.0)


def make(sizes, ptype, gtype, bits, copies, seed, offset=0):
    g = torch.Generator().manual_seed(seed)

    def cut(x):   # at an odd place of a larger buffer when offset is given
        whole = torch.zeros(x.numel() + 64, dtype=x.dtype, device="cuda")
        part = whole[offset:offset + x.numel()]
        part.copy_(x)
        return part

    params = [cut(torch.randn(n, generator=g).mul(0.3).to(ptype)) for n in sizes]
    grads = [cut(torch.randn(n, generator=g).mul(10.0 ** float(torch.randn((), generator=g))).to(gtype)) for n in sizes]
    ms, vs, es, fs = [], [], [], []
    for n in sizes:
        m, r = torch.randn(n, generator=g).mul(0.1).double().numpy(), torch.randn(n, generator=g).mul(0.3).abs().double().numpy()
        if bits == 32:
            ms.append(cut(torch.from_numpy(m).float()))
            vs.append(cut(torch.from_numpy(r * r).float()))
            continue
        for x, codes, scales in ((m, ms, es), (r, vs, fs)):
            e = ref.flat_exponents(x.astype(np.float32).astype(np.float64))
            q = torch.from_numpy(ref.nearest(x.astype(np.float32) * 2.0 ** -np.repeat(e, 128)[:n].astype(np.float64))).to(torch.float8_e4m3fn)
            codes.append(cut(q.view(torch.uint8)))
            scales.append(cut(torch.from_numpy((e + 127).astype(np.uint8))))
    cs = [cut(torch.zeros(n, dtype=torch.bfloat16)) for n in sizes] if copies else None
    return lowbit.AdamWTable(params, grads, ms, vs, es if bits == 8 else None, fs if bits == 8 else None, cs)


def states(t, i, bits):
    x = t.tensors
    n = x["params"][i].numel()
    if bits == 32:
        return x["m"][i].double().cpu().numpy(), x["v"][i].double().cpu().numpy()
    return decode8(x["m"][i], x["m_scale"][i], n), decode8(x["v"][i], x["v_scale"][i], n) ** 2


def run_and_check(t, bits, step, seed=None, scale=None):
    x = t.tensors
    before = [(x["params"][i].double().cpu().numpy(), x["grads"][i].double().cpu().numpy(), *states(t, i, bits)) for i in range(t.count)]
    clip = None if scale is None else torch.tensor(scale, device="cuda")
    t.step(step=step, seed=seed, grad_scale=clip, **OPTIONS)
    torch.cuda.synchronize()
    b1, b2 = OPTIONS["betas"]
    f32 = lambda v: float(np.float32(v))  # noqa: E731
    for i, (p, g, m, v) in enumerate(before):
        n = len(p)
        if n == 0:
            continue
        g = g * (1.0 if scale is None else f32(scale))
        p1, m1, v1 = ref.adamw(p, g, m, v, lr=OPTIONS["lr"], beta1=b1, beta2=b2, eps=OPTIONS["eps"], weight_decay=OPTIONS["weight_decay"], step=step)
        size_m = np.abs(b1 * m) + np.abs((1 - b1) * g)
        tol_m, tol_v = 5 * U * size_m, 6 * U * v1     # one unit more for each rounded constant
        got = x["params"][i].double().cpu().numpy()
        move = np.abs(p1 - p * (1 - OPTIONS["lr"] * OPTIONS["weight_decay"]))
        reach = OPTIONS["lr"] / (1 - b1 ** step) * size_m / (np.sqrt(v1 / (1 - b2 ** step)) + OPTIONS["eps"])   # the moment's terms may cancel
        tol_p = 4 * U * np.abs(p) + 16 * U * np.maximum(move, reach)
        bits32 = ref.noise(n, i, seed) if seed is not None else None
        if x["params"][i].dtype == torch.float32:
            assert (np.abs(got - p1) <= tol_p).all()
            if x["copies"] is not None:
                assert torch.equal(x["copies"][i], x["params"][i].bfloat16())
        else:
            unit = 2.0 ** (np.floor(np.log2(np.maximum(np.abs(p1), 2.0 ** -126))) - 7)
            if seed is None:
                assert (np.abs(got - p1) <= tol_p + unit * 0.5 * (1 + 1e-6)).all()
            else:
                down = np.floor((np.abs(p1) - tol_p) / unit + (bits32 & np.uint64(0xFFFF)).astype(np.float64) / 65536) * unit
                up = np.floor((np.abs(p1) + tol_p) / unit + (bits32 & np.uint64(0xFFFF)).astype(np.float64) / 65536) * unit
                assert ((np.abs(got) >= down - 1e-30) & (np.abs(got) <= up + 1e-30)).all()
        m2, v2 = states(t, i, bits)
        if bits == 32:
            assert (np.abs(m2 - m1) <= tol_m).all() and (np.abs(v2 - v1) <= tol_v).all()
            continue
        for got8, scales, exact, tol, root in ((x["m"][i], x["m_scale"][i], m1, tol_m, False), (x["v"][i], x["v_scale"][i], np.sqrt(v1), 5 * U * np.sqrt(v1), True)):
            e = scales.cpu().numpy().astype(np.int64) - 127
            want_e = ref.flat_exponents(exact.astype(np.float32).astype(np.float64))
            assert (np.abs(e - want_e) <= 1).all() and (e != want_e).mean() <= 0.05
            q = ref.decode(got8.cpu().numpy())
            s = 2.0 ** -np.repeat(e, 128)[:n].astype(np.float64)
            noise = (bits32 >> np.uint64(16)).astype(np.float64) if root and seed is not None else None
            if root:
                low, high = ref.root_values(np.maximum(exact - tol, 0) , e, noise), ref.root_values(exact + tol, e, noise)
            else:
                low, high = ref.nearest((exact - tol) * s), ref.nearest((exact + tol) * s)
            assert ((q >= np.minimum(low, high)) & (q <= np.maximum(low, high))).all()


SIZES = [1, 2, 127, 128, 129, 1000, 4096, 4097, 20000]


@pytest.mark.parametrize("ptype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("gtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("seed", [None, 77])
def test_step(ptype, gtype, bits, seed):
    t = make(SIZES, ptype, gtype, bits, ptype == torch.float32, 1)
    run_and_check(t, bits, step=1, seed=seed)
    run_and_check(t, bits, step=2, seed=None if seed is None else seed + 1, scale=0.37)
    run_and_check(t, bits, step=5000, seed=None if seed is None else (1 << 32) - 1)


@pytest.mark.parametrize("offset", [1, 2, 3, 8])
@pytest.mark.parametrize("bits", [8, 32])
def test_unaligned_tensors(offset, bits):
    run_and_check(make([5, 700, 4100], torch.float32, torch.bfloat16, bits, True, 2, offset), bits, step=3, seed=5)
    run_and_check(make([5, 700, 4100], torch.bfloat16, torch.float32, bits, False, 3, offset), bits, step=3)


def test_more_tensors_than_one_launch_holds_and_empty_ones():
    sizes = [(i * 37) % 300 for i in range(1000)]
    t = make(sizes, torch.float32, torch.float32, 8, False, 4)
    run_and_check(t, 8, step=2, seed=9)
    lowbit.AdamWTable([], [], [], []).step(lr=1.0, step=1)


def test_nothing_outside_the_tensors_is_written():
    n = 1003
    for bits in (8, 32):
        t = make([n], torch.float32, torch.bfloat16, bits, True, 5, offset=16)
        before = {}
        for name, x in t.tensors.items():
            if x is not None:
                whole = x[0]._base
                whole[:16], whole[16 + x[0].numel():] = 93, 93
        t.step(step=1, seed=3, **OPTIONS)
        for name, x in t.tensors.items():
            if x is not None:
                whole = x[0]._base
                assert (whole[:16] == 93).all() and (whole[16 + x[0].numel():] == 93).all(), name


def test_skip_flag_leaves_everything():
    t = make([300, 5000], torch.float32, torch.float32, 8, True, 6)
    before = {k: [y.clone() for y in x] for k, x in t.tensors.items() if x is not None}
    t.step(step=1, skip=torch.tensor(1, dtype=torch.int32, device="cuda"), **OPTIONS)
    assert all(torch.equal(a, b) for k, x in before.items() for a, b in zip(x, t.tensors[k]))
    t.step(step=1, skip=torch.tensor(0, dtype=torch.int32, device="cuda"), **OPTIONS)
    assert not torch.equal(before["params"][1], t.tensors["params"][1])


@pytest.mark.parametrize("bits", [8, 32])
def test_non_finite_gradients_stay_in_their_element(bits):
    t = make([1000], torch.float32, torch.float32, bits, False, 7)
    u = make([1000], torch.float32, torch.float32, bits, False, 7)
    for i, v in ((3, float("nan")), (200, float("inf")), (999, float("-inf"))):
        t.tensors["grads"][0][i] = v
        u.tensors["grads"][0][i] = 0.0
    t.step(step=1, **OPTIONS)
    u.step(step=1, **OPTIONS)
    p, q = t.tensors["params"][0], u.tensors["params"][0]
    bad = torch.isnan(p)
    assert bad[[3, 200, 999]].all() and bad.sum() == 3
    keep = torch.ones(1000, dtype=torch.bool, device="cuda")
    keep[[3, 200, 999]] = False
    assert torch.equal(p[keep], q[keep])
    m, v = states(t, 0, bits)
    for i in (3, 200, 999):
        assert not np.isfinite(m[i]) and not np.isfinite(v[i])
    assert np.isfinite(m[keep.cpu().numpy()]).all() and np.isfinite(v[keep.cpu().numpy()]).all()


def test_eight_bit_roots_follow_a_falling_second_moment():
    """With the gradients gone, v falls by beta2 a step: 0.1 % of a unit that 8 bits cannot show.  Rounded to nearest the
    roots stand still; rounded stochastically they fall as they should on average."""
    n, steps = 1 << 16, 400
    for seed, follows in ((None, False), (1, True)):
        p, g = torch.zeros(n, device="cuda"), torch.randn(n, generator=torch.Generator().manual_seed(0)).cuda()
        t = lowbit.AdamWTable.zeros([p], [g], bits=8)
        t.step(lr=0.0, step=1, betas=(0.9, 0.999), seed=seed)
        first = decode8(t.tensors["v"][0], t.tensors["v_scale"][0], n).mean()
        g.zero_()
        for i in range(steps):
            t.step(lr=0.0, step=2 + i, betas=(0.9, 0.999), seed=None if seed is None else seed + 1 + i)
        fall = decode8(t.tensors["v"][0], t.tensors["v_scale"][0], n).mean() / first
        # 65536 entries, each a sum of 400 roundings of at most a unit in 8..15: the mean is known to far better than 1 %
        assert (abs(fall - 0.999 ** (steps / 2)) < 0.02) == follows


def test_zero_gradients_from_zero_states_change_nothing_but_the_decay():
    p = torch.randn(500, generator=torch.Generator().manual_seed(0)).cuda()
    q = p.clone()
    for bits in (8, 32):
        lowbit.AdamWTable.zeros([p], [torch.zeros(500, device="cuda")], bits=bits).step(lr=0.1, step=1, weight_decay=0.0)
        assert torch.equal(p, q)


def test_refusals():
    z = lambda n, d=torch.float32: torch.zeros(n, dtype=d, device="cuda")  # noqa: E731
    for args in (([z(5)], [z(4)], [z(5)], [z(5)]), ([z(5)], [], [z(5)], [z(5)]), ([z(5)], [z(5)], [z(5)], [z(5, torch.uint8)]), ([z(5).half()], [z(5)], [z(5)], [z(5)]),
                 ([z(5)], [z(5)], [z(5, torch.uint8)], [z(5, torch.uint8)]), ([z(5)], [z(5)], [z(5)], [z(5)], [z(1, torch.uint8)], [z(1, torch.uint8)]),
                 ([z(10)[::2]], [z(5)], [z(5)], [z(5)]), ([z(5).cpu()], [z(5)], [z(5)], [z(5)]), ([z(5)], [z(5)], [z(5)], [z(5)], None, None, [z(5)])):
        with pytest.raises(ValueError):
            lowbit.AdamWTable(*args)
    t = lowbit.AdamWTable.zeros([z(5)], [z(5)])
    with pytest.raises(ozk.OzkError):
        t.step(lr=1e-3, step=0)
    with pytest.raises(ValueError):
        t.step(lr=1e-3, step=1, grad_scale=torch.ones(()))
