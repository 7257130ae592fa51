"""The oracle of the operators over lists of tensors (CPU): torch's AdamW, the 8-bit type's numbers, rounding to neither side."""
import math

import numpy as np
import pytest
import torch

from oracle import optimizer_oracle as oo


def test_a_run_of_steps_is_torchs_adamw():
    g = torch.Generator().manual_seed(0)
    p = torch.randn(50, generator=g, dtype=torch.float64)
    q, m, v = p.numpy().copy(), np.zeros(50), np.zeros(50)
    p.requires_grad_()
    opt = torch.optim.AdamW([p], lr=0.01, betas=(0.8, 0.95), eps=1e-6, weight_decay=0.1)
    for t in range(1, 8):
        p.grad = torch.randn(50, generator=g, dtype=torch.float64)
        c = oo.coefficient(1.0, oo.grad_norm([p.grad.numpy()]), 5.0)
        m, v = oo.moments(c * p.grad.numpy(), m, v, 0.8, 0.95)
        q = oo.param(q, m, v, t, 0.01, 0.8, 0.95, 1e-6, 0.1)
        norm = torch.nn.utils.clip_grad_norm_([p], 5.0)
        assert abs(float(norm) - oo.grad_norm([p.grad.numpy()]) * max(1.0, float(norm) / 5.0)) < 1e-5
        opt.step()
    assert np.abs(q - p.detach().numpy()).max() < 1e-7             # (torch clips by max / (norm + 1e-6))


def test_the_numbers_of_the_8_bit_type():
    codes = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(codes, oo.E4M3) and oo.E4M3[-1] == 448 and oo.E4M3[1] == 2.0 ** -9


@pytest.mark.parametrize("root", [False, True])
def test_values_go_to_one_of_their_two_codes_and_over_the_steps_to_neither_side(root):
    rng = np.random.default_rng(1)
    x = np.abs(rng.normal(size=300)) * np.exp(rng.normal(size=300))
    if not root:
        x *= rng.choice([-1, 1], size=300)
    steps = 4000
    total, seen = np.zeros(300), []
    for t in range(1, steps + 1):
        code, s, _ = oo.quantise(x, t, root)
        value = code * np.repeat(s, oo.BLOCK)[:300]
        total += value
        if t < 50:
            seen.append(value)
    y = np.abs(x) / np.repeat(s, oo.BLOCK)[:300]
    low = oo.E4M3[np.searchsorted(oo.E4M3, y * (1 - 1e-12), side="right") - 1]
    apart = np.maximum(low / 8, 2.0 ** -9) * np.repeat(s, oo.BLOCK)[:300]
    assert (np.abs(np.array(seen) - x) <= apart * (1 + 1e-9)).all()
    # a sequence frac(u + t b) of N terms counts an interval to within a few log N / N of its length
    assert (np.abs(total / steps - x) <= apart * 4 * math.log(steps) / steps).all()


def test_a_second_moment_that_moves_by_less_than_half_a_code_a_step_arrives():
    """g = 1 from v = 0.25: v -> 1 with b2 = 0.999, beside an element that keeps the block's scale where it is.  Rounded to nearest, 0.1 %
    a step never leaves a code."""
    v, steps = np.array([0.25, 4.0]), 3000
    g = np.array([1.0, 2.0])
    for t in range(1, steps + 1):
        code, s, _ = oo.quantise(np.sqrt(oo.moments(g, np.zeros(2), v, 0.9, 0.999)[1]), t, True)
        v = (code * s[0]) ** 2
    exact = 1 - 0.75 * 0.999 ** steps
    assert abs(v[0] - exact) < 0.27, (v[0], exact)      # within a code (12.5 % of the root)


def test_blocks_of_nothing_and_of_no_numbers():
    x = np.zeros(600)
    x[300] = 1e-31
    x[550] = math.inf
    code, s, _ = oo.quantise(x, 3, False)
    assert s[0] == 0 and s[1] == 0 and math.isnan(s[2]) and not code.any()
