"""AdamW with 8-bit moments over the whole range of fp32: gradients whose squares overflow or are subnormal numbers, blocks of any
magnitude.  Codes and scales are those of single operations in fp32, each rounded to nearest by numpy, bit for bit."""
import numpy as np
import pytest
import torch

import paper_1707_00424_b200 as pb
from oracle import optimizer_oracle as oo

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F = np.float32
U = 2.0 ** -24


class Single:
    """The definition in include/parle.h, an operation after another."""

    def __init__(self, n):
        self.n = n
        blocks = -(-n // 256)
        self.codes, self.scales = [np.zeros(n, F), np.zeros(n, F)], [np.zeros(blocks, F), np.zeros(blocks, F)]

    def wide(self, s):
        return np.repeat(s, 256)[:self.n]

    def step(self, grad, t, b1, b2):
        """New codes and scales; returns (m, v, sqrt(v))."""
        old, root = (c * self.wide(s) for c, s in zip(self.codes, self.scales))
        m = old * F(b1) + grad * F(1 - b1)
        v = root * root * F(b2) + grad * grad * F(1 - b2)
        r = np.sqrt(v)
        u = oo.thresholds(self.n, t).astype(np.float64)
        for k, (x, threshold) in enumerate(((m, u), (r, (1 << 24) - 1 - u))):
            top = np.array([np.abs(b).max() for b in oo.blocks(x)], F)
            none = top < F(2.0 ** -100)
            factor = self.wide(np.where(none, F(0), F(448) * (F(1) / top)))
            # the product to fp32's 24 bits, or to a multiple of 2^-29 below 2^-6
            exact = np.abs(x).astype(np.float64) * factor.astype(np.float64)
            y = np.where(exact < 2.0 ** -6, np.rint(exact * 2.0 ** 29) * 2.0 ** -29, exact.astype(F).astype(np.float64))
            y = np.where(np.isfinite(y), np.minimum(y, 448.0), 448.0)
            apart = np.exp2(np.maximum(np.floor(np.log2(np.maximum(y, 2.0 ** -20))), -6) - 3)
            code = (np.floor(y / apart + threshold / (1 << 24)) * apart * np.where(x < 0, -1, 1)).astype(F)
            if k == 1:
                code = np.where((x > 0) & ~self.wide(none), np.maximum(code, F(2.0 ** -9)), F(0))
            self.codes[k] = code
            self.scales[k] = np.where(np.isfinite(top), np.where(none, F(0), top * (F(1) / F(448))), F(np.nan))
        return m, v, r


def compare(n, gradients, betas=(0.9, 0.999), eps=1e-8, lr=1e-3, shift=0):
    """Steps with these gradients; the parameter's steps from the moments in 64 bits, where the largest of a block is a number."""
    with np.errstate(all="ignore"):
        p = torch.full((n + shift,), 0.5, device=DEV)[shift:]
        state, single = pb.adamw_state([p], 8), Single(n)
        for t, grad in enumerate(gradients, 1):
            before = p.double().cpu().numpy()
            pb.adamw([p], [torch.from_numpy(grad).to(DEV)], state[0], state[1], step=t, lr=lr, betas=betas, eps=eps, weight_decay=0.1,
                     exp_avg_scales=state[2], exp_avg_sq_scales=state[3])
            m, v, r = single.step(grad, t, *betas)
            for k in (0, 1):
                scales = state[2 + k][0].cpu().numpy()
                assert np.array_equal(scales, single.scales[k], equal_nan=True), (t, k)
                known = np.isfinite(single.wide(scales))
                got = state[k][0].float().cpu().numpy()
                assert np.array_equal(got[known], single.codes[k][known]), (t, k, np.argwhere(known & (got != single.codes[k]))[:5])
            den = r.astype(np.float64) / np.sqrt(1 - betas[1] ** t) + eps
            moved = lr / (1 - betas[0] ** t) * m.astype(np.float64) / den
            want = before * (1 - lr * 0.1) - moved
            # reciprocal 2^-22, root and products around it 8 u; factor of the correction and decay, the sum
            off = np.abs(moved) * (2.0 ** -22 + 16 * U) + 3 * U * (np.abs(before) + np.abs(moved))
            got = p.double().cpu().numpy()
            known = np.isfinite(want) & (np.abs(moved) < 1e38)
            assert (np.abs(got - want)[known] <= off[known]).all(), (t, np.abs(got - want)[known].max())
            assert np.array_equal(np.isfinite(got)[~np.isfinite(want)], np.isfinite(want)[~np.isfinite(want)])


def normal(n, seed, spread=0.0):
    g = np.random.default_rng(seed)
    return (g.normal(size=n) * np.exp(spread * g.normal(size=n))).astype(F)


# ---- the second moment's root at both ends of fp32 -------------------------------------------------------------------------------

@pytest.mark.parametrize("eps", [1e-8, 2.0 ** -60])
@pytest.mark.parametrize("size", [2.0 ** -40, 2.0 ** -50, 2.0 ** -58, 2.0 ** -62, 2.0 ** -66, 2.0 ** -70, 1e-20, 2.0 ** 40])
def test_gradients_whose_squares_are_small_or_subnormal(size, eps):
    for n, shift in ((5000, 0), (1000, 3)):
        compare(n, [normal(n, k, 1.0) * F(size) for k in range(3)], eps=eps, shift=shift)


@pytest.mark.parametrize("n", [300, 5000])
def test_small_and_ordinary_gradients_in_one_block(n):
    for eps in (1e-8, 1e-12, 2.0 ** -60):
        grad = normal(n, 5)
        grad[1::3] *= F(2.0 ** -60)
        grad[2::3] *= F(2.0 ** -68)
        grad[7::11] = 0
        compare(n, [grad, grad[::-1].copy()], eps=eps)


@pytest.mark.parametrize("n", [300, 5000])
def test_a_square_that_overflows_leaves_a_finite_parameter(n):
    """v is infinite, m / (sqrt(v) + eps) is 0: only the decay is left of the step.  The block's roots are lost from then on."""
    grad = normal(n, 6)
    grad[5], grad[100], grad[n - 1] = 1e20, -3e38, 2e19
    compare(n, [normal(n, 7), grad])
    p = torch.full((n,), 0.5, device=DEV)
    state = pb.adamw_state([p], 8)
    flags = torch.zeros(1, dtype=torch.int32, device=DEV)
    pb.adamw([p], [torch.from_numpy(grad).to(DEV)], state[0], state[1], step=1, lr=1e-3, weight_decay=0.1, exp_avg_scales=state[2], exp_avg_sq_scales=state[3], flags=flags)
    assert bool(torch.isfinite(p).all()) and int(flags) == 0
    assert p[[5, 100, n - 1]].tolist() == [float(F(0.5) * F(1 - 1e-4))] * 3


# ---- blocks of large numbers ---------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("n", [300, 5000])
@pytest.mark.parametrize("size", [2.0 ** 19, 2.0 ** 26, 2.0 ** 50, 2.0 ** 60])
def test_small_roots_in_blocks_of_large_ones(n, size):
    """Every root above 0 has at least the smallest code, however small it is beside the block's largest."""
    grad = normal(n, 8) * F(size)
    for i in range(1, 9):
        grad[i::16] = normal(len(grad[i::16]), i) * F(2.0 ** (13 * i - 70))
    grad[9::16] = 0
    compare(n, [grad, np.roll(grad, 3), np.roll(grad, 7)])
    p = torch.zeros(n, device=DEV)
    state = pb.adamw_state([p], 8)
    pb.adamw([p], [torch.from_numpy(grad).to(DEV)], state[0], state[1], step=1, lr=1e-3, exp_avg_scales=state[2], exp_avg_sq_scales=state[3])
    assert np.array_equal(state[1][0].float().cpu().numpy() > 0, grad * grad * F(1 - 0.999) > 0)


@pytest.mark.parametrize("size", [2.0 ** 14, 2.0 ** 40, 2.0 ** 74, 2.0 ** 75, 2.0 ** 100, 2.0 ** 125, 2.0 ** 126])
def test_first_moments_up_to_the_end_of_fp32(size):
    """beta1 = 0: m is the gradient.  1 / largest is a subnormal number at the end; small numbers lie at the borders between codes."""
    g = np.random.default_rng(11)
    grad = (g.uniform(0.5, 1, 4000) * np.exp2(-g.integers(0, 30, 4000)) * size * np.where(g.random(4000) < 0.5, -1, 1)).astype(F)
    grad[::256] = F(1.9 * size)
    compare(4000, [grad, grad[::-1].copy()], betas=(0.0, 0.999))


# ---- small numbers beside large ones: their place between two codes is a multiple of 2^-29 ----------------------------------------------

def test_many_numbers_far_below_their_blocks_largest():
    """Two of these codes would be others if the product were rounded to 24 bits there, too."""
    n = 1 << 21
    grad = normal(n, 1, 4.0)
    x = np.abs(grad * F(1 - 0.9))
    factor = np.repeat(F(448) * (F(1) / x.reshape(-1, 256).max(1)), 256)
    exact, u = x.astype(np.float64) * factor.astype(np.float64), oo.thresholds(n, 1).astype(np.float64) / (1 << 24)
    low = exact < 2.0 ** -6
    codes = [np.floor(y * 2.0 ** 9 + u)[low] for y in ((x * factor).astype(np.float64), np.rint(exact * 2.0 ** 29) * 2.0 ** -29)]
    assert (codes[0] != codes[1]).sum() == 2
    compare(n, [grad])
