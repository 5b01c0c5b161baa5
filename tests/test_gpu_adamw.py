"""AdamW over many tensors, its 8-bit states and the gradients' global norm, against the formulas in 64 bits.

u = 2^-24.  m is the sum of two rounded products (3 u of their magnitudes; the gradient's factor one more, and one for 1 - beta), v
of two (6 u of itself: all its terms are positive).  The update has 4 u for m, half of v's error, a square root and a division of
2 u each and four products: below 24 u of |m|'s terms / denominator; the parameter two more roundings of itself."""
import math

import pytest
import torch

from paper_2407_12075_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
F, H = torch.float32, torch.bfloat16
INF, NAN = float("inf"), float("nan")


def rand(seed, n, dtype=F, scale=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (torch.randn(n, generator=g, device=DEV) * scale).to(dtype)


def cut(flat, n, offset):
    """n elements of a larger buffer from `offset` on, so that the pointer has only its type's alignment."""
    return flat[offset:offset + n]


def make(sizes, p_dtype, g_dtype, bits, seed=0, offset=0, copy=False):
    t = {k: [] for k in ("params", "grads", "m", "v", "m_scale", "v_scale", "copies")}
    for i, n in enumerate(sizes):
        s = seed + 10 * i
        at = lambda x: cut(x, n, offset)  # noqa: E731
        t["params"].append(at(rand(s, n + offset, p_dtype, 0.05)))
        t["grads"].append(at(rand(s + 1, n + offset, g_dtype, 1e-2)))
        if bits == 32:
            t["m"].append(at(rand(s + 2, n + offset, F, 5e-3)))
            t["v"].append(at(rand(s + 3, n + offset, F, 1e-2).square()))
            t["m_scale"].append(None), t["v_scale"].append(None)
        else:
            blocks = -(-n // 256)
            t["m"].append(at((rand(s + 2, n + offset) * 50).clamp(-127, 127).to(torch.int8)))
            t["v"].append(at((rand(s + 3, n + offset) * 60 + 120).clamp(1, 254).to(torch.uint8)))
            t["m_scale"].append((rand(s + 4, blocks).abs() + 0.2) * 1e-6)
            t["v_scale"].append((rand(s + 5, blocks).abs() + 0.2) * 1e-13)
        t["copies"].append(at(torch.zeros(n + offset, dtype=H, device=DEV)) if copy else None)
    return t


def clone(t):
    return {k: [None if x is None else x.clone() for x in v] for k, v in t.items()}


def values(t, i):
    """m and v of tensor i in 64 bits."""
    m, v = t["m"][i].double(), t["v"][i].double()
    if t["m_scale"][i] is None:
        return m, v
    block = torch.arange(m.numel(), device=DEV) // 256
    return m * m.abs() * t["m_scale"][i].double()[block], v ** 4 * t["v_scale"][i].double()[block]


def expected(t, i, step, lr, b1, b2, eps, wd, gs=1.0):
    """New parameter, m and v before any rounding to 8 bits, and the magnitudes that their errors go by."""
    g = t["grads"][i].double() * gs
    m0, v0 = values(t, i)
    m, v = b1 * m0 + (1 - b1) * g, b2 * v0 + (1 - b2) * g * g
    size = (b1 * m0).abs() + ((1 - b1) * g).abs()
    denom = torch.sqrt(v / (1 - b2 ** step)) + eps
    p = t["params"][i].double()
    new = p * (1 - lr * wd) - lr / (1 - b1 ** step) * m / denom
    return new, m, v, size, 3 * U * p.abs() + 24 * U * lr / (1 - b1 ** step) * size / denom


def near(got, want, bound, what):
    err = (got.double() - want).abs()
    assert (err <= bound).all(), f"{what}: {err.max().item()}, {(err - bound).max().item()} over its bound"


def check_step(t, after, i, args, gs=1.0):
    step, lr, b1, b2, eps, wd = args
    new, m, v, size, p_err = expected(t, i, step, lr, b1, b2, eps, wd, gs)
    got = after["params"][i]
    near(got, new, p_err + (torch.finfo(H).eps / 2 * new.abs() * 1.01 if got.dtype == H else U * new.abs()) + 1e-45, "param")
    if after["copies"][i] is not None:
        near(after["copies"][i], new, p_err + torch.finfo(H).eps / 2 * new.abs() * 1.01 + 1e-45, "copy")
    if t["m_scale"][i] is None:
        near(after["m"][i], m, 5 * U * size + 1e-44, "m")
        near(after["v"][i], v, 6 * U * v + 1e-44, "v")
        return
    n = m.numel()
    block = torch.arange(n, device=DEV) // 256
    for name, x, power, top, least, err in (("m", m.abs(), 2, 127, 2.0 ** -100, 8 * U * size), ("v", v, 4, 254, 2.0 ** -94, 10 * U * v)):
        largest = torch.zeros(-(-n // 256), dtype=torch.float64, device=DEV).scatter_reduce_(0, block, x, "amax").clamp_(min=least)
        scale = after[name + "_scale"][i]
        off = torch.zeros_like(largest).scatter_reduce_(0, block, err, "amax")
        near(scale, largest / top ** power, off / top ** power + 3 * U * scale.double(), name + "_scale")
        # the code is one of the two around the value, whose place among the codes is known to `slack`
        y = x / scale.double()[block]
        slack = (err / scale.double()[block] + 6 * U * y)
        code = after[name][i].double().abs()
        low = torch.minimum((y - slack).clamp(min=0) ** (1 / power), torch.tensor(float(top), device=DEV)).sub(1e-9).floor().clamp(min=0)
        high = torch.minimum((y + slack) ** (1 / power), torch.tensor(float(top), device=DEV)).add(1e-9).floor() + 1
        assert (code >= low).all() and (code <= high.clamp(max=top)).all(), name
        if name == "v":
            assert (code[v > 1e-44] >= 1).all()
        else:
            assert (after["m"][i].double() * m >= -1e-30).all()


SIZES = [[1], [7, 0, 256], [255, 257, 1, 4096], [2049, 31, 100000], [300] * 30, [5] * 600]


@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: f"{len(s)}x{s[0]}")
@pytest.mark.parametrize("p_dtype,g_dtype,copy", [(F, F, False), (F, H, True), (H, H, False), (H, F, False)])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("offset", [0, 1])
def test_step(sizes, p_dtype, g_dtype, copy, bits, offset):
    t = make(sizes, p_dtype, g_dtype, bits, seed=100, offset=offset, copy=copy)
    before = clone(t)
    decay = [0.1 if i % 2 else 0.0 for i in range(len(sizes))]
    h = B.tbn_adamw_tensors(**t, weight_decay=decay)
    args = (7, 1e-2, 0.9, 0.95, 1e-8)
    B.tbn_adamw_step(h, *args, seed=3)
    for i in range(0, len(sizes), max(1, len(sizes) // 8)):
        check_step(before, t, i, (*args, decay[i]))
    if bits == 8:
        m, v = B.tbn_adamw_unpack(h)
        for i in range(0, len(sizes), max(1, len(sizes) // 8)):
            want = values(t, i)
            near(m[i], want[0], 2 * U * want[0].abs(), "unpacked m")
            near(v[i], want[1], 4 * U * want[1], "unpacked v")
    again = clone(before)
    B.tbn_adamw_step(B.tbn_adamw_tensors(**again, weight_decay=decay), *args, seed=3)
    for k in t:
        assert all(a is None or torch.equal(a, b) for a, b in zip(t[k], again[k])), k


@pytest.mark.parametrize("bits", [32, 8])
def test_first_steps_from_zero_states(bits):
    """From zero states the first update is lr * sign(g) (m / bc1 = g, v / bc2 = g^2), whatever the gradient's size."""
    n, lr = 3000, 1e-2
    g = rand(1, n, F) * torch.logspace(-4, 6, n, device=DEV)
    p = torch.zeros(n, device=DEV)
    m, v, ms, vs = B.tbn_adamw_state([p], bits)
    B.tbn_adamw_step(B.tbn_adamw_tensors([p], [g], m, v, ms, vs), 1, lr, 0.9, 0.999, 1e-12)
    near(p, -lr * torch.sign(g).double(), lr * (40 * U + 1e-12 / g.double().abs()), "param")


def test_kinds_of_tensors_in_one_call():
    kinds = [(F, F, 32), (H, H, 8), (F, H, 8), (H, F, 32)]
    parts = [make([513, 70], p, g, b, seed=20 * i) for i, (p, g, b) in enumerate(kinds)]
    t = {k: sum((q[k] for q in parts), []) for k in parts[0]}
    before = clone(t)
    B.tbn_adamw_step(B.tbn_adamw_tensors(**t, weight_decay=0.01), 3, 1e-3, seed=9)
    for i in range(8):
        check_step(before, t, i, (3, 1e-3, 0.9, 0.999, 1e-8, 0.01))


def test_codes_are_unbiased():
    """One value repeated under many seeds: the mean of its 8-bit form is the value.  4096 draws of a variable that is off by at most
    the gap between two codes: six standard deviations of the mean are 6 * gap / 2 / 64 at most."""
    n, draws = 256, 4096
    g = torch.cat([torch.ones(1, device=DEV), rand(1, n - 1).abs() * 0.3]) * 0.1
    total_m, total_v = torch.zeros(n, dtype=torch.float64, device=DEV), torch.zeros(n, dtype=torch.float64, device=DEV)
    p = torch.zeros(n, device=DEV)
    for seed in range(draws // 64):
        params, grads = [p.clone() for _ in range(64)], [g] * 64
        m, v, ms, vs = B.tbn_adamw_state(params, 8)
        h = B.tbn_adamw_tensors(params, grads, m, v, ms, vs)
        B.tbn_adamw_step(h, 1, 1e-3, 0.9, 0.999, seed=seed + (seed << 33))
        for a, b in zip(*B.tbn_adamw_unpack(h)):
            total_m += a.double()
            total_v += b.double()
    for total, want, power, scale in ((total_m, 0.1 * g.double(), 2, ms[0]), (total_v, 1e-3 * g.double() ** 2, 4, vs[0])):
        y = want / scale.double()
        low = y.pow(1 / power).floor()
        gap = ((low + 1) ** power - low ** power) * scale.double()
        above = y >= 1 if power == 4 else y >= 0                        # a v below the first code is raised to it
        assert ((total / draws - want).abs() <= 6 * gap / 2 / 64 + 1e-5 * want)[above].all()


def test_a_small_second_moment_moves():
    """With beta2 = 0.999 and a constant gradient v goes from 0.25 g^2 towards g^2 by a thousandth of the way at a time, each step below a
    code's distance.  After 1000 steps the mean over 255 elements is 1 - 0.75 exp(-1) of it, to a few hundredths."""
    n = 256
    g = torch.full((n,), 0.5, device=DEV)
    g[0] = 1.0                                                          # holds the block's scale
    p = torch.zeros(n, device=DEV)
    m, v, ms, vs = B.tbn_adamw_state([p], 8)
    v[0].fill_(round(254 * (0.25 * 0.25) ** 0.25))
    v[0][0] = 254
    vs[0].fill_(1.0 / 254 ** 4)
    h = B.tbn_adamw_tensors([p], [g], m, v, ms, vs)
    for t in range(1, 1001):
        B.tbn_adamw_step(h, t, 1e-6, 0.9, 0.999, seed=1)
    got = B.tbn_adamw_unpack(h)[1][0][1:].double().mean().item()
    start = (round(254 * 0.0625 ** 0.25) / 254) ** 4
    want = 0.25 + (start - 0.25) * 0.999 ** 1000
    # a step adds the variance of a draw, at most (gap / 2)^2 with gap = 4 / 127 of v, and 0.999 keeps it: below 0.25 * 0.016 * sqrt(500) = 0.09
    # for an element, a 16th of it for the mean over 255; four of those
    assert abs(got - want) < 4 * 0.09 / 16
    assert want - start > 0.1


def test_bad_values_stay_to_themselves():
    for bits in (32, 8):
        t = make([1000], F, F, bits, seed=5)
        t["grads"][0][3], t["grads"][0][300], t["grads"][0][700], t["grads"][0][999] = NAN, INF, 1e30, -INF
        before = clone(t)
        h = B.tbn_adamw_tensors(**t)
        B.tbn_adamw_step(h, 5, 1e-3, 0.9, 0.999)
        p = t["params"][0]
        assert torch.isnan(p[[3, 300, 999]]).all() and int(torch.isnan(p).sum()) == 3
        good = torch.ones(1000, dtype=torch.bool, device=DEV)
        good[[3, 300, 700, 999]] = False
        new, _, _, _, err = expected(before, 0, 5, 1e-3, 0.9, 0.999, 1e-8, 0.0)
        assert ((p.double() - new).abs() <= err + U * new.abs())[good].all()
        # 1e30: its square is infinite, its update nothing
        assert p[700] == before["params"][0][700]
        m, v = (x.float() for x in ((t["m"][0], t["v"][0]) if bits == 32 else (x[0] for x in B.tbn_adamw_unpack(h))))
        assert torch.isnan(v[3]) or bits == 8 and torch.isinf(v[3])
        assert not torch.isfinite(m[[3, 300, 999]]).any() and not torch.isfinite(v[[300, 700, 999]]).any()
        assert torch.isfinite(m[good]).all() and torch.isfinite(v[good]).all()
        B.tbn_adamw_step(h, 6, 1e-3, 0.9, 0.999)
        assert torch.isnan(p[[3, 300, 999]]).all() and int(torch.isnan(p).sum()) == 3


def test_tiny_and_huge_blocks():
    for scale in (1e-44, 1e-38, 1e-30, 1e-20, 1e-10, 1e10, 1e18):
        for bits in (32, 8):
            n = 700
            t = make([n], F, F, bits, seed=6)
            t["grads"][0].copy_(rand(8, n) * scale)
            m, v, ms, vs = B.tbn_adamw_state(t["params"], bits)
            t.update(m=m, v=v, m_scale=ms or [None], v_scale=vs or [None])
            before = clone(t)
            h = B.tbn_adamw_tensors(**t)
            B.tbn_adamw_step(h, 1, 1e-3, 0.9, 0.999, 1e-8)
            assert torch.isfinite(t["params"][0]).all()
            if scale >= 1e-15 or bits == 32:
                new, _, _, _, err = expected(before, 0, 1, 1e-3, 0.9, 0.999, 1e-8, 0.0)
                # the second moments of the smallest gradients are below the smallest float: eps stands for them either way
                near(t["params"][0], new, err + 2 * U * new.abs() + (1e-3 * 1e-12 if scale < 1e-18 else 0.0), "param")
            if bits == 8:
                for a in B.tbn_adamw_unpack(h):
                    assert torch.isfinite(a[0]).all()


@pytest.mark.parametrize("bits", [32, 8])
def test_norm_and_clipping(bits):
    sizes = [1, 1000, 0, 255, 70001] + [33] * 300
    t = make(sizes, F, H, bits, seed=7, offset=1)
    before = clone(t)
    h = B.tbn_adamw_tensors(**t, weight_decay=0.1)
    want = math.sqrt(sum(g.double().square().sum().item() for g in t["grads"]))
    for limit in (want / 3, want * 3):
        norm, scale = B.tbn_grad_norm(h, limit)
        assert norm.item() == torch.tensor(want, dtype=F).item()        # 64-bit sums agree to far below a float's step
        assert scale.item() == torch.tensor(min(1.0, limit / want), dtype=F).item()
    norm, scale = B.tbn_grad_norm(h, want / 3)
    B.tbn_adamw_step(h, 2, 1e-3, 0.9, 0.999, grad_scale=scale)
    for i in (0, 1, 3, 4, 200):
        check_step(before, t, i, (2, 1e-3, 0.9, 0.999, 1e-8, 0.1), gs=scale.double().item())


def test_a_norm_that_is_not_finite_skips_the_step():
    for bad in (NAN, INF):
        for bits in (32, 8):
            t = make([300, 5000], F, F, bits, seed=8, copy=True)
            t["grads"][1][4321] = bad
            before = clone(t)
            h = B.tbn_adamw_tensors(**t, weight_decay=0.1)
            norm, scale = B.tbn_grad_norm(h, 1.0)
            assert not torch.isfinite(norm).item() and torch.isnan(scale).item()
            B.tbn_adamw_step(h, 2, 1e-3, grad_scale=scale)
            for k in ("params", "m", "v", "m_scale", "v_scale", "copies"):
                assert all(a is None or torch.equal(a, b) for a, b in zip(t[k], before[k]))


def test_norm_of_large_values_does_not_overflow():
    g = [torch.full((1000,), 1e25, device=DEV), torch.full((100,), -3e38, device=DEV)]
    p = [torch.zeros_like(x) for x in g]
    h = B.tbn_adamw_tensors(p, g, *B.tbn_adamw_state(p, 32))
    norm, scale = B.tbn_grad_norm(h, 1.0)
    want = math.sqrt(sum((x.double() ** 2).sum().item() for x in g))
    assert math.isinf(norm.item()) == (want > 3.4028235e38) and scale.item() == torch.tensor(1.0 / want, dtype=F).item()
    empty = B.tbn_adamw_tensors([], [], [], [])
    norm, scale = B.tbn_grad_norm(empty, 1.0)
    assert norm.item() == 0 and scale.item() == 1
    B.tbn_adamw_step(empty, 1, 1e-3)


@pytest.mark.parametrize("bits", [32, 8])
def test_step_and_rate_from_the_device_and_replayed(bits):
    """A captured step with its number, rate and clipping factor on the device equals eager steps with numbers, bit for bit."""
    sizes = [1000, 33, 4096]
    a = make(sizes, F, H, bits, seed=9, copy=True)
    b = clone(a)
    ha, hb = (B.tbn_adamw_tensors(**t, weight_decay=0.05) for t in (a, b))
    step, lr = torch.zeros(1, dtype=torch.int64, device=DEV), torch.zeros(1, device=DEV)
    ws = torch.empty(1 << 16, dtype=torch.uint8, device=DEV)

    def captured():
        _, scale = B.tbn_grad_norm(hb, 0.3, workspace=ws)
        B.tbn_adamw_step(hb, step, lr, 0.9, 0.95, 1e-8, grad_scale=scale, seed=11)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured()
    for t in range(1, 6):
        rate = torch.tensor(1e-3 * t, dtype=F).item()
        for ga, gb, s in zip(a["grads"], b["grads"], range(3)):
            ga.copy_(rand(50 * t + s, ga.numel(), H, 1e-2))
            gb.copy_(ga)
        _, scale = B.tbn_grad_norm(ha, 0.3)
        B.tbn_adamw_step(ha, t, rate, 0.9, 0.95, 1e-8, grad_scale=scale, seed=11)
        step.fill_(t), lr.fill_(rate)
        graph.replay()
        torch.cuda.synchronize()
        for k in a:
            assert all(x is None or torch.equal(x, y) for x, y in zip(a[k], b[k])), (t, k)


def test_elements_beyond_32_bit_indexes():
    n = 2 ** 32 + 777
    p, g = torch.zeros(n, dtype=H, device=DEV), torch.zeros(n, dtype=H, device=DEV)
    g[-777:] = 0.5
    g[:777] = 0.5
    m, v, ms, vs = B.tbn_adamw_state([p], 8)
    h = B.tbn_adamw_tensors([p], [g], m, v, ms, vs)
    norm, scale = B.tbn_grad_norm(h, 1.0)
    assert norm.item() == torch.tensor(math.sqrt(0.25 * 2 * 777), dtype=F).item()
    B.tbn_adamw_step(h, 1, 1e-2, 0.9, 0.999, 1e-8)
    want = torch.tensor(-1e-2, dtype=H).item()
    assert (p[-777:] == want).all() and (p[:777] == want).all() and not p[777:10 ** 6].any() and not p[2 ** 31 - 5:2 ** 31 + 10 ** 6].any()
    assert (m[0][-777:] >= 126).all() and (v[0][-777:] >= 253).all() and not v[0][-10 ** 6:-777].any()


def test_wrapper_refuses_what_does_not_fit():
    p, g = torch.zeros(10, device=DEV), torch.zeros(10, device=DEV)
    m, v, ms, vs = B.tbn_adamw_state([p], 8)
    with pytest.raises(B.TbnError):
        B.tbn_adamw_tensors([p], [g], m, v)                             # 8-bit states without scales
    with pytest.raises(TypeError):
        B.tbn_adamw_tensors([p], [g], m, m, ms, vs)
    with pytest.raises(TypeError):
        B.tbn_adamw_tensors([p.half()], [g], m, v, ms, vs)
    with pytest.raises(B.TbnError):
        B.tbn_adamw_tensors([p], [g[:9]], m, v, ms, vs)
    h = B.tbn_adamw_tensors([p], [g], m, v, ms, vs)
    with pytest.raises(B.TbnError):
        B.tbn_adamw_step(h, 0, 1e-3)
    with pytest.raises(TypeError):
        B.tbn_adamw_step(h, 1, 1e-3, grad_scale=torch.ones(1, dtype=torch.float64, device=DEV))
    with pytest.raises(B.TbnError):
        B.tbn_grad_norm(h, 1.0, workspace=torch.empty(8, dtype=torch.uint8, device=DEV))
    h32 = B.tbn_adamw_tensors([p], [g], *B.tbn_adamw_state([p], 32))
    with pytest.raises(B.TbnError):
        B.tbn_adamw_unpack(h32)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("n", [256 * 9 + 5, 3_000_003])
def test_alignment_does_not_change_the_result(bits, n):
    """The same tensor where accesses of eight elements may begin, and one element further on: the same bits."""
    a = make([n], F, H, bits, seed=60, copy=True)
    shift = lambda x: None if x is None else cut(torch.cat([x[:1], x]), n, 1)  # noqa: E731
    b = {k: [x.clone() if k.endswith("scale") and x is not None else shift(x) for x in v] for k, v in a.items()}
    for t in (a, b):
        h = B.tbn_adamw_tensors(**t, weight_decay=0.1)
        for step in (4, 5):
            B.tbn_adamw_step(h, step, 1e-3, seed=77)
    for k in a:
        assert all(x is None or torch.equal(x, y) for x, y in zip(a[k], b[k])), k


def test_two_streams_at_once():
    """Two optimizers stepped on two streams give what each gives alone."""
    tensors = [make([200_000, 33, 4096], F, H, bits, seed=70 + bits) for bits in (8, 32)]
    alone = [clone(t) for t in tensors]
    for t in alone:
        h = B.tbn_adamw_tensors(**t)
        for step in range(1, 6):
            _, scale = B.tbn_grad_norm(h, 0.1)
            B.tbn_adamw_step(h, step, 1e-3, grad_scale=scale, seed=2)
    torch.cuda.synchronize()
    streams, handles = [torch.cuda.Stream() for _ in tensors], [B.tbn_adamw_tensors(**t) for t in tensors]
    for step in range(1, 6):
        for h, s in zip(handles, streams):
            with torch.cuda.stream(s):
                _, scale = B.tbn_grad_norm(h, 0.1)
                B.tbn_adamw_step(h, step, 1e-3, grad_scale=scale, seed=2)
    torch.cuda.synchronize()
    for t, w in zip(tensors, alone):
        for k in t:
            assert all(x is None or torch.equal(x, y) for x, y in zip(t[k], w[k])), k
