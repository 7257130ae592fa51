"""Gradient norm and AdamW on the GPU against the fp64 oracle: types, odd sizes and places, 8-bit moments, clipping, skipped steps, streams,
graphs.  Tolerances come from the arithmetic: u = 2^-24 is half a step of fp32 relative to the value; the hardware's root and reciprocal
are off by at most 2^-22 each; a 16-bit result by half a step of its type."""
import math

import numpy as np
import pytest
import torch

import paper_1707_00424_b200 as pb
from oracle import optimizer_oracle as oo

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
TYPES = (torch.float32, torch.bfloat16, torch.float16)
SIZES = (1, 7, 8, 255, 256, 257, 1000, 4096, 4103, 20011)
HYPER = dict(lr=1e-2, betas=(0.9, 0.99), eps=1e-6, weight_decay=0.05)


def f64(t):
    return t.detach().double().cpu().numpy()


def half_step(dtype, value):
    if dtype == torch.float32:
        return U * np.abs(value)
    return np.maximum(torch.finfo(dtype).eps / 2 * np.abs(value), torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps / 2)


def place(x, shift):
    """x inside a larger buffer, `shift` elements behind a 512-byte boundary, with NaN around it."""
    buf = torch.full((x.numel() + 64,), math.nan, dtype=torch.float32, device=DEV).to(x.dtype)
    view = buf[shift:shift + x.numel()]
    view.copy_(x)
    return view, buf


def untouched(buf, shift, n):
    rest = torch.cat([buf[:shift], buf[shift + n:]]).float()
    return bool(torch.isnan(rest).all())


# ---- norm --------------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shift", [0, 1, 3])
def test_norm(dtype, shift):
    g = torch.Generator().manual_seed(3)
    for sizes in ((1,), (8,), SIZES, (300000, 1, 70001), (0, 5, 0)):
        grads = [place(torch.randn(n, generator=g).to(dtype).to(DEV), shift)[0] for n in sizes]
        want = oo.grad_norm([f64(x) for x in grads])
        got = pb.grad_norm(grads)
        assert got.shape == () and got.dtype == torch.float32
        assert abs(float(got) - want) <= want * (U + 8 * U / 2 + 1e-14), sizes      # eight squares in fp32 under a root; the last rounding
        assert torch.equal(pb.grad_norm(grads), got)


@pytest.mark.parametrize("count", [96, 97, 400, 401, 1600, 1601, 4000])
def test_norm_of_lists_of_any_length(count):
    """Around the lengths of one launch's list, and several launches."""
    g = torch.Generator().manual_seed(4)
    flat = torch.randn(10 * count, generator=g).to(DEV)
    grads = list(flat.view(count, 10).unbind())
    want = oo.grad_norm([f64(flat)])
    assert abs(float(pb.grad_norm(grads)) - want) <= want * 6 * U


@pytest.mark.parametrize("values, norm", [
    ([3e38, -3e38], math.inf), ([1e30] * 3, math.sqrt(3) * 1e30), ([1e-30] * 9, 3e-30), ([2.0 ** -149], 2.0 ** -149),
    ([1e-25, 1e-30], 1e-25), ([0.0] * 20, 0.0), ([math.inf, 1.0], math.inf), ([math.nan, 1.0], math.nan), ([math.inf, math.nan], math.nan),
])
def test_norm_over_the_whole_range(values, norm):
    got = float(pb.grad_norm([torch.tensor(values, device=DEV)]))
    assert got == norm or (math.isnan(got) and math.isnan(norm)) or abs(got - norm) <= 6 * U * norm


def test_norm_into_given_tensors():
    g = [torch.ones(100000, device=DEV)]
    out = torch.zeros(1, device=DEV)
    ws = torch.empty(8 * (1 + 100000 // 16384 + 1) + 128, dtype=torch.uint8, device=DEV)
    version = out._version
    assert pb.grad_norm(g, out=out, workspace=ws) is out and out._version == version + 1
    assert abs(float(out) - math.sqrt(100000)) < 1e-3
    with pytest.raises(pb.ParleError) as e:
        pb.grad_norm(g, workspace=ws[:8])
    assert e.value.code == -6


# ---- AdamW -------------------------------------------------------------------------------------------------------------------

class Case:
    """Tensors of these sizes with moments of earlier steps, on the GPU and in fp64."""

    def __init__(self, sizes, param, grad, bits, shift=0, copy=None, seed=0, spread=1.0):
        g = torch.Generator().manual_seed(seed)
        self.bits, self.shift, self.sizes, self.param_type, self.copy_type = bits, shift, sizes, param, copy
        normal = lambda n: torch.randn(n, generator=g)      # noqa: E731
        self.params, self.grads, self.m, self.v, self.ms, self.vs, self.copies, self.buffers = [], [], [], [], [], [], [], []
        for n in sizes:
            wide = torch.exp(spread * normal(n))
            self.add(self.params, normal(n).to(param))
            self.add(self.grads, (normal(n) * wide).to(grad))
            m, r = 0.3 * normal(n) * wide, (0.2 + torch.rand(n, generator=g)) * wide
            if bits == 32:
                self.add(self.m, m)
                self.add(self.v, r * r)
            else:
                for codes, scales, x, root in ((self.m, self.ms, m, False), (self.v, self.vs, r, True)):
                    c, s, _ = oo.quantise(x.double().numpy(), 5, root)
                    codes.append(torch.from_numpy(c).float().to(torch.float8_e4m3fn).to(DEV))
                    scales.append(torch.from_numpy(s).float().to(DEV))
            if copy:
                self.add(self.copies, torch.zeros(n).to(copy))

    def add(self, to, x):
        view, buf = place(x.to(DEV), self.shift)
        to.append(view)
        self.buffers.append((buf, x.numel()))

    def state(self, i):
        """Moments of tensor i in fp64."""
        if self.bits == 32:
            return f64(self.m[i]), f64(self.v[i])
        wide = lambda s, n: np.repeat(f64(s), 256)[:n]      # noqa: E731
        n = self.sizes[i]
        return f64(self.m[i]) * wide(self.ms[i], n), (f64(self.v[i]) * wide(self.vs[i], n)) ** 2

    def step(self, step, **kw):
        pb.adamw(self.params, self.grads, self.m, self.v, step=step, **{**HYPER, **kw}, exp_avg_scales=self.ms or None, exp_avg_sq_scales=self.vs or None,
                 copies=self.copies or None)

    def check(self, step, c=1.0, **kw):
        """One step against the oracle."""
        h = {**HYPER, **kw}
        (b1, b2), lr, eps, wd = h["betas"], h["lr"], h["eps"], h["weight_decay"]
        f32 = lambda x: float(np.float32(x))                # noqa: E731
        before = [(f64(p), f64(g), *self.state(i)) for i, (p, g) in enumerate(zip(self.params, self.grads))]
        self.step(step, **kw)
        torch.cuda.synchronize()
        for i, (p0, g, m0, v0) in enumerate(before):
            g = c * g
            m, v = oo.moments(g, m0, v0, f32(b1), f32(b2))
            m = m + (f32(1 - b1) - (1 - f32(b1))) * g       # (the complements are rounded from 1 - b)
            v = v + (f32(1 - b2) - (1 - f32(b2))) * g * g
            # roundings: of the coefficient 4 u, of its product with 1 - b or its root and of that with g, doubled by the square; of the old 8-bit
            # values: of sqrt(b2), of its product with the scale, of that with the code, doubled, and of the square; then of the sum
            m_off = (b1 * np.abs(m0) * 2 + (1 - b1) * np.abs(g) * 8) * U + np.abs(m) * U
            v_off = (b2 * v0 * (4 if self.bits == 32 else 8) + (1 - b2) * g * g * 15) * U + v * U
            den = np.sqrt(v / (1 - b2 ** step)) + eps
            rate = lr / (1 - b1 ** step)
            want = oo.param(p0, m, v, step, lr, b1, b2, eps, wd)
            # the new parameter: of m and v, root and reciprocal 2^-22 each, 8 roundings of factors; decay and the sum
            off = rate * (m_off / den + np.abs(m) / den * (v_off / (2 * np.maximum(v, 1e-300)) + 2 * 2.0 ** -22 + 8 * U)) + 2 * U * np.abs(p0) + U * np.abs(want)
            last = half_step(self.param_type, want) if self.param_type != torch.float32 else 0
            got = f64(self.params[i])
            assert (np.abs(got - want) <= off + last * (1 + 2.0 ** -7) + 1e-45).all(), (i, np.abs(got - want).max())
            if self.copy_type:
                assert torch.equal(self.copies[i], self.params[i].to(self.copy_type))
            if self.bits == 32:
                assert (np.abs(f64(self.m[i]) - m) <= m_off + 1e-45).all() and (np.abs(f64(self.v[i]) - v) <= v_off + 1e-45).all()
            else:
                self.codes(self.m[i], self.ms[i], m, m_off, step, False)
                r = np.sqrt(v)
                self.codes(self.v[i], self.vs[i], r, v_off / (2 * np.maximum(r, 1e-300)) + r * 2.0 ** -22, step, True)
        for buf, n in self.buffers:
            assert untouched(buf, self.shift, n)

    @staticmethod
    def codes(codes, scales, x, off, step, root):
        """The code of each value, but where it is as near to the border between two codes as it may be off."""
        want, s, border = oo.quantise(x, step, root)
        n = len(x)
        wide = np.repeat(s, 256)[:n]
        worst = np.array([o.max() for o in oo.blocks(off)])
        assert (np.abs(f64(scales) - s) <= worst / 448 + 2 * U * s).all()
        got = f64(codes)
        with np.errstate(divide="ignore", invalid="ignore"):
            y = np.where(wide > 0, np.abs(x) / wide, 0)
            slack = np.where(wide > 0, off / wide + y * (np.repeat(worst / np.maximum(s * 448, 1e-300), 256)[:n] + 4 * U), 0) / np.maximum(y / 16, 2.0 ** -9) + 2.0 ** -23
        near = (border <= slack) | (y >= 447.9)
        assert np.array_equal(got[~near], want[~near]), np.argwhere(got != want)[:5]
        assert (np.abs(np.abs(got) - y) <= np.maximum(y / 8, 2.0 ** -9) * 1.01).all()
        assert n < 3000 or near.mean() < 0.01


@pytest.mark.parametrize("param, grad, copy", [
    (torch.float32, torch.float32, None), (torch.float32, torch.bfloat16, torch.bfloat16), (torch.float32, torch.float16, torch.float16),
    (torch.float32, torch.bfloat16, None), (torch.bfloat16, torch.bfloat16, None), (torch.float16, torch.float16, None),
    (torch.bfloat16, torch.float32, None), (torch.float16, torch.bfloat16, None), (torch.float32, torch.float32, torch.float16),
])
@pytest.mark.parametrize("bits", [32, 8])
def test_one_step(param, grad, copy, bits):
    for shift in (0, 3, 8):
        Case(SIZES, param, grad, bits, shift, copy, seed=shift).check(4)
    Case((5000, 0, 3), param, grad, bits, copy=copy, seed=9).check(1000)


@pytest.mark.parametrize("bits", [32, 8])
def test_first_step_from_zeros_and_a_run_of_steps(bits):
    g = torch.Generator().manual_seed(5)
    params = [torch.randn(n, generator=g).to(DEV) for n in (700, 33)]
    want = [f64(p) for p in params]
    state = pb.adamw_state(params, bits)
    assert (state[2] is None) == (bits == 32) and all(float(x.float().abs().sum()) == 0 for x in (*state[0], *state[1]))
    exact = [(np.zeros(n), np.zeros(n)) for n in (700, 33)]
    for t in range(1, 30):
        grads = [torch.randn(p.shape, generator=g).to(DEV) for p in params]
        pb.adamw(params, grads, state[0], state[1], step=t, lr=0.01, exp_avg_scales=state[2], exp_avg_sq_scales=state[3])
        for i, gr in enumerate(grads):
            exact[i] = oo.moments(f64(gr), *exact[i], 0.9, 0.999)
            want[i] = oo.param(want[i], *exact[i], t, 0.01, 0.9, 0.999, 1e-8, 0.01)
        if t == 1:
            for p, w in zip(params, want):
                assert np.abs(f64(p) - w).max() < 1e-6
    # 32 bits: 29 steps of 0.01 (ratio below 3.2, off by 2^-20 a step) on parameters below 4; 8 bits: a code's distance (12.5 % of a
    # moment below the block's largest) in each of 29 steps that weigh 0.9^k, on a ratio of order 1
    tolerance = 29 * (0.01 * 3.2 * 2.0 ** -20 + 4 * 2 * U) if bits == 32 else 29 * 0.01 * 0.5
    for p, w in zip(params, want):
        assert np.abs(f64(p) - w).max() < tolerance


def test_a_second_moment_in_8_bits_that_moves_slowly_arrives():
    """As the oracle's: rounded to nearest it would stay at 0.25."""
    p, g = [torch.zeros(512, device=DEV)], [torch.ones(512, device=DEV)]
    g[0][::256] = 2.0
    m, v, ms, vs = pb.adamw_state(p, 8)
    v[0].copy_(torch.full((512,), 112.0).to(torch.float8_e4m3fn))
    v[0][::256] = 448.0
    vs[0].fill_(2.0 / 448)
    for t in range(1, 3001):
        pb.adamw(p, g, m, v, step=t, lr=0.0, exp_avg_scales=ms, exp_avg_sq_scales=vs)
    r = f64(v[0]) * np.repeat(f64(vs[0]), 256)
    r = r[np.arange(512) % 256 != 0]
    exact = math.sqrt(1 - 0.75 * 0.999 ** 3000)
    # in the mean it drifts as the exact one does; a single element is within two codes of it
    assert abs(r.mean() - exact) < 0.03 and np.abs(r - exact).max() < 0.25


def test_moments_in_8_bits_are_those_of_single_operations_bit_for_bit():
    """Each operation rounded to nearest in fp32 by numpy: the same codes and scales, over steps in which one difference would grow."""
    f = np.float32
    g = torch.Generator().manual_seed(21)
    n, (b1, b2) = 70000, (0.9, 0.999)
    p = [torch.zeros(n, device=DEV)]
    m, v, ms, vs = pb.adamw_state(p, 8)
    mc, rc, m_scale, r_scale = np.zeros(n, f), np.zeros(n, f), np.zeros(-(-n // 256), f), np.zeros(-(-n // 256), f)
    wide = lambda s: np.repeat(s, 256)[:n]                  # noqa: E731
    for t in range(1, 6):
        grad = (torch.randn(n, generator=g) * torch.exp(2 * torch.randn(n, generator=g))).to(DEV)
        grad[1000:1400] = 0.0
        pb.adamw(p, [grad], m, v, step=t, lr=1e-3, betas=(b1, b2), exp_avg_scales=ms, exp_avg_sq_scales=vs)
        x = grad.cpu().numpy()
        old, root = mc * wide(m_scale), rc * wide(r_scale)
        first = old * f(b1) + x * f(1 - b1)
        second = np.sqrt(root * root * f(b2) + x * x * f(1 - b2))
        u = oo.thresholds(n, t).astype(np.float64)
        for what, value, threshold, codes, scales in (("m", first, u, m, ms), ("r", second, (1 << 24) - 1 - u, v, vs)):
            top = np.array([np.abs(b).max() for b in oo.blocks(value)], f)
            with np.errstate(divide="ignore"):
                y = np.minimum(np.abs(value) * wide(np.where(top < f(2.0 ** -100), f(0), f(448) * (f(1) / top))), f(448)).astype(np.float64)
            apart = np.exp2(np.maximum(np.floor(np.log2(np.maximum(y, 2.0 ** -20))), -6) - 3)
            code = (np.floor(y / apart + threshold / (1 << 24)) * apart * np.sign(value)).astype(f)
            if what == "r":
                code = np.where(value > 0, np.maximum(code, f(2.0 ** -9)), f(0))
            scale = np.where(top < f(2.0 ** -100), f(0), top * f(1 / f(448)))
            assert np.array_equal(codes[0].float().cpu().numpy(), code) and np.array_equal(scales[0].cpu().numpy(), scale), (t, what)
            if what == "m":
                mc, m_scale = code, scale
            else:
                rc, r_scale = code, scale


@pytest.mark.parametrize("bits", [32, 8])
def test_clipped_and_scaled_gradients(bits):
    case = Case((3000, 17), torch.float32, torch.float16, bits, seed=6)
    norm = pb.grad_norm(case.grads)
    exact = oo.grad_norm([f64(g) for g in case.grads])
    for scale, most in ((1.0, exact / 3), (1.0, exact * 3), (1 / 128, exact / 512), (2.0, exact)):
        case.check(7, c=oo.coefficient(scale, float(norm), most), norm=norm, max_norm=most, grad_scale=scale)
    case.check(8, c=0.25, grad_scale=0.25)
    case.check(9, norm=norm)                               # no bound: the norm only says whether the step is taken
    case.check(10, c=1.0, norm=torch.zeros(1, device=DEV), max_norm=1.0)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("bad", [math.inf, math.nan, -math.inf])
def test_a_norm_that_is_no_number_skips_the_step(bits, bad):
    case = Case((3000, 17), torch.float32, torch.float32, bits, copy=torch.bfloat16, seed=7)
    flags = torch.zeros(1, dtype=torch.int32, device=DEV)
    every = [*case.params, *case.m, *case.v, *case.ms, *case.vs, *case.copies]
    before = [x.clone() for x in every]
    case.grads[0][5] = bad
    case.step(3, norm=pb.grad_norm(case.grads), max_norm=1.0, flags=flags)
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(every, before))
    assert int(flags) == pb.FLAG_NONFINITE
    flags.zero_()
    case.grads[0][5] = 0.0
    case.step(3, norm=pb.grad_norm(case.grads), max_norm=1.0, flags=flags)
    assert int(flags) == 0 and not torch.equal(before[0], case.params[0])


def test_what_is_no_number_stays_in_its_element_or_block():
    flags = torch.zeros(1, dtype=torch.int32, device=DEV)
    case = Case((1000,), torch.float32, torch.float32, 32, seed=8)
    case.grads[0][300] = math.nan
    case.step(3, flags=flags)
    assert int(flags) == pb.FLAG_NONFINITE and torch.isnan(case.params[0]).nonzero().flatten().tolist() == [300]
    case = Case((1000,), torch.float32, torch.float32, 8, seed=8)
    case.grads[0][300] = math.inf
    case.grads[0][999] = math.nan
    case.step(3)
    assert torch.isnan(case.params[0]).nonzero().flatten().tolist() == [300, 999]
    assert torch.isnan(case.ms[0]).tolist() == [False, True, False, True] == torch.isnan(case.vs[0]).tolist()
    case.step(4)                                          # the blocks' moments are unknown from then on
    lost = torch.isnan(case.params[0])
    assert bool(lost[256:512].all()) and bool(lost[768:].all()) and int(lost.sum()) == 256 + 232
    half = Case((100,), torch.float16, torch.float32, 32, seed=8)
    half.params[0].fill_(65504.0)
    flags.zero_()
    half.step(3, lr=1e3, weight_decay=0.0, flags=flags)    # some go beyond the type
    assert int(flags) == pb.FLAG_NONFINITE and bool(torch.isinf(half.params[0]).any())


@pytest.mark.parametrize("bits", [32, 8])
def test_zero_gradients_and_tiny_moments(bits):
    p = [torch.full((600,), 2.0, device=DEV)]
    m, v, ms, vs = pb.adamw_state(p, bits)
    kw = dict(exp_avg_scales=ms, exp_avg_sq_scales=vs)
    zero = [torch.zeros(600, device=DEV)]
    pb.adamw(p, zero, m, v, step=1, lr=0.1, weight_decay=0.5, **kw)
    assert torch.equal(p[0], torch.full_like(p[0], 2.0 * 0.95)) and float(m[0].float().abs().sum()) == 0
    # one gradient far below its block's largest: its root is held as something, so that the next step is no division by eps alone
    g = [torch.zeros(600, device=DEV)]
    g[0][0], g[0][1] = 1.0, 1e-7
    pb.adamw(p, g, m, v, step=1, lr=1e-3, weight_decay=0.0, **kw)
    before = p[0].clone()
    for t in range(2, 6):
        pb.adamw(p, zero, m, v, step=t, lr=1e-3, weight_decay=0.0, **kw)
    assert float((p[0] - before).abs().max()) <= 4 * 1e-3 * 2


def test_step_and_rate_from_the_device_and_a_replayed_graph():
    case, twin = (Case((5000, 3), torch.float32, torch.float32, 8, seed=10) for _ in range(2))
    step, rate = torch.zeros(1, dtype=torch.int64, device=DEV), torch.ones(1, device=DEV)
    norm = torch.zeros((), device=DEV)
    ws = torch.empty(8192, dtype=torch.uint8, device=DEV)

    def call():
        pb.grad_norm(case.grads, out=norm, workspace=ws)
        case.step(4, step_dev=step, lr_dev=rate, norm=norm, max_norm=1.0)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        call()
    torch.cuda.current_stream().wait_stream(s)
    twin.step(4, norm=pb.grad_norm(twin.grads), max_norm=1.0)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for k in range(1, 4):
        step.fill_(k)
        rate.fill_(0.5 ** k)
        graph.replay()
        twin.step(4 + k, lr=HYPER["lr"] * 0.5 ** k, norm=pb.grad_norm(twin.grads), max_norm=1.0)
    torch.cuda.synchronize()
    for a, b in zip((*case.m, *case.v), (*twin.m, *twin.v)):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    for a, b in zip((*case.params, *case.ms, *case.vs), (*twin.params, *twin.ms, *twin.vs)):
        assert torch.equal(a, b)


def test_many_tensors_take_several_launches_and_give_what_each_alone_does():
    g = torch.Generator().manual_seed(11)
    sizes = [int(n) for n in torch.randint(1, 600, (1000,), generator=g)]
    for bits in (32, 8):
        case = Case(sizes, torch.float32, torch.bfloat16, bits, copy=torch.float16, seed=12)
        alone = Case(sizes, torch.float32, torch.bfloat16, bits, copy=torch.float16, seed=12)
        case.step(5)
        for i in range(0, 1000, 97):
            pick = lambda x: x[i:i + 1] or None            # noqa: E731
            pb.adamw(pick(alone.params), pick(alone.grads), pick(alone.m), pick(alone.v), step=5, **HYPER, exp_avg_scales=pick(alone.ms), exp_avg_sq_scales=pick(alone.vs),
                     copies=pick(alone.copies))
            for a, b in ((case.params, alone.params), (case.m, alone.m), (case.v, alone.v), (case.copies, alone.copies)):
                assert torch.equal(a[i].view(torch.uint8), b[i].view(torch.uint8))


def test_arrays_that_begin_at_different_places_give_what_aligned_ones_do():
    for bits in (32, 8):
        a, b = (Case((3001,), torch.float32, torch.bfloat16, bits, seed=13) for _ in range(2))
        b.params = [place(b.params[0], 5)[0]]
        b.grads = [place(b.grads[0], 2)[0]]
        if bits == 8:
            codes = torch.zeros(4000, dtype=torch.uint8, device=DEV)[3:3004]
            codes.copy_(b.m[0].view(torch.uint8))
            b.m = [codes.view(torch.float8_e4m3fn)]
        a.step(3)
        b.step(3)
        for x, y in ((a.params, b.params), (a.m, b.m), (a.v, b.v), (a.ms, b.ms), (a.vs, b.vs)):
            assert all(torch.equal(s.view(torch.uint8), t.view(torch.uint8)) for s, t in zip(x, y))


def test_another_stream_and_modules_parameters():
    layer = torch.nn.Linear(40, 30).to(DEV)
    params = list(layer.parameters())
    layer(torch.randn(5, 40, device=DEV)).square().sum().backward()
    want = [p.detach().clone() for p in params]
    grads = [p.grad for p in params]
    for run, stream in ((want, None), (params, torch.cuda.Stream())):
        torch.cuda.synchronize()
        state = pb.adamw_state(run)
        torch.cuda.synchronize()
        norm = pb.grad_norm(grads, stream=stream)
        versions = [p._version for p in run]
        pb.adamw(run, grads, state[0], state[1], step=1, lr=0.1, norm=norm, max_norm=0.1, stream=stream)
        assert [p._version for p in run] == [v + 1 for v in versions]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(params, want))


@pytest.mark.parametrize("call", [
    lambda c: pb.grad_norm([]), lambda c: pb.grad_norm(c.grads[0]), lambda c: pb.grad_norm([c.grads[0], c.grads[0].half()]), lambda c: pb.grad_norm([c.grads[0][::2]]),
    lambda c: pb.grad_norm([c.grads[0].cpu()]), lambda c: pb.grad_norm([c.grads[0], c.grads[0].cpu()]), lambda c: pb.grad_norm([c.grads[0].double()]),
    lambda c: pb.grad_norm([None]), lambda c: pb.grad_norm(c.grads, out=torch.zeros(2, device=DEV)), lambda c: pb.grad_norm(c.grads, workspace=torch.zeros(64)),
    lambda c: pb.adamw([], [], [], [], step=1, lr=0.1), lambda c: c.step(0), lambda c: c.step(1.5), lambda c: c.step(1, lr=-1.0), lambda c: c.step(1, betas=(1.0, 0.9)),
    lambda c: c.step(1, betas=(0.9, -0.1)), lambda c: c.step(1, eps=0.0), lambda c: c.step(1, eps=2.0), lambda c: c.step(1, weight_decay=-1.0), lambda c: c.step(1, lr=math.nan),
    lambda c: c.step(1, grad_scale=0.0), lambda c: c.step(1, grad_scale=math.inf), lambda c: c.step(1, max_norm=1.0), lambda c: c.step(1, norm=torch.ones(1, device=DEV), max_norm=0.0),
    lambda c: c.step(1, norm=torch.ones(1)), lambda c: c.step(1, norm=1.0), lambda c: c.step(1, step_dev=torch.ones(1, device=DEV)), lambda c: c.step(1, flags=torch.ones(1, device=DEV)),
    lambda c: pb.adamw(c.params, c.grads[:1], c.m, c.v, step=1, lr=0.1), lambda c: pb.adamw(c.params, None, c.m, c.v, step=1, lr=0.1),
    lambda c: pb.adamw(c.params, c.grads, c.m, [c.v[0], c.v[1].half()], step=1, lr=0.1), lambda c: pb.adamw(c.params, c.grads, c.m, [c.v[0], c.v[1][:5]], step=1, lr=0.1),
    lambda c: pb.adamw([c.params[0]] * 2, [c.grads[0]] * 2, c.m, c.v, step=1, lr=0.1), lambda c: pb.adamw(c.params, c.grads, c.m, c.m, step=1, lr=0.1),
    lambda c: pb.adamw(c.params, c.grads, c.m, c.v, step=1, lr=0.1, copies=[p.clone() for p in c.params]),
    lambda c: pb.adamw(c.params, c.grads, c.m, c.v, step=1, lr=0.1, exp_avg_scales=c.m, exp_avg_sq_scales=c.m),
    lambda c: pb.adamw(c.params, c.grads, *([x.to(torch.float8_e4m3fn) for x in y] for y in (c.m, c.v)), step=1, lr=0.1),
    lambda c: pb.adamw(c.params, c.grads, *([x.to(torch.float8_e4m3fn) for x in y] for y in (c.m, c.v)), step=1, lr=0.1,
                       exp_avg_scales=[torch.zeros(2, device=DEV)] * 2, exp_avg_sq_scales=[torch.zeros(2, device=DEV)] * 2),
])
def test_refused_arguments(call):
    c = Case((256, 256), torch.float32, torch.float32, 32)
    with pytest.raises(pb.ParleError) as e:
        call(c)
    assert e.value.code == -1


@pytest.mark.parametrize("bits", [8, 32])
def test_past_32_bit_offsets(bits):
    """Elements from 2^32 on are stepped as those of a tensor of their own are (2^32 is a multiple of the thresholds' period and of a block)."""
    n, last = (1 << 32) + 5003, 5003
    big = [torch.zeros(n, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    g = torch.Generator().manual_seed(40)
    p, grad = (torch.randn(last, generator=g).bfloat16().to(DEV) for _ in range(2))
    big[0][-last:], big[1][-last:] = p, grad
    state, small = pb.adamw_state([big[0]], bits), pb.adamw_state([p], bits)
    assert float(pb.grad_norm([big[1]])) == float(pb.grad_norm([grad]))
    for t in (1, 2):
        pb.adamw([big[0]], [big[1]], state[0], state[1], step=t, lr=0.01, exp_avg_scales=state[2], exp_avg_sq_scales=state[3])
        pb.adamw([p], [grad], small[0], small[1], step=t, lr=0.01, exp_avg_scales=small[2], exp_avg_sq_scales=small[3])
    assert torch.equal(big[0][-last:], p) and not bool(big[0][:1 << 20].any()) and not bool(big[0][(1 << 32) - (1 << 20):1 << 32].any())
    for a, b in zip(state[:2], small[:2]):
        assert torch.equal(a[0][-last:].view(torch.uint8), b[0].view(torch.uint8))
    if bits == 8:
        assert all(torch.equal(a[0][-20:], b[0]) for a, b in zip(state[2:], small[2:]))


def test_calls_from_several_threads_and_streams():
    import threading
    cases = [Case((3000, 17, 40000), torch.float32, torch.bfloat16, 8, seed=50 + i) for i in range(4)]
    twins = [Case((3000, 17, 40000), torch.float32, torch.bfloat16, 8, seed=50 + i) for i in range(4)]
    torch.cuda.synchronize()

    def work(case):
        s = torch.cuda.Stream()
        for t in range(1, 20):
            case.step(t, norm=pb.grad_norm(case.grads, stream=s), max_norm=1.0, stream=s)
        s.synchronize()

    threads = [threading.Thread(target=work, args=(c,)) for c in cases]
    for th in threads:
        th.start()
    for th in threads:
        th.join()
    for case, twin in zip(cases, twins):
        for t in range(1, 20):
            twin.step(t, norm=pb.grad_norm(twin.grads), max_norm=1.0)
        for a, b in ((case.params, twin.params), (case.m, twin.m), (case.v, twin.v), (case.ms, twin.ms), (case.vs, twin.vs)):
            assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(a, b))
