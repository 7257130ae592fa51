"""Calls of the operators over lists that their documentation allows: gradients that tensors share, clipping of scaled gradients at the ends of
fp32, workspaces of the documented size."""
import math

import numpy as np
import pytest
import torch

import paper_1707_00424_b200 as pb
from oracle import optimizer_oracle as oo

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24


def f64(t):
    return t.double().cpu().numpy()


@pytest.mark.parametrize("bits", [8, 32])
def test_tensors_may_share_a_gradient(bits):
    """Three replicas take one gradient; each ends as it does with a gradient of its own."""
    g = torch.Generator().manual_seed(1)
    grad = torch.randn(3000, generator=g).to(DEV)
    start = [torch.randn(3000, generator=g).to(DEV) for _ in range(3)]
    ends = []
    for grads in ([grad] * 3, [grad.clone() for _ in range(3)]):
        params = [p.clone() for p in start]
        state = pb.adamw_state(params, bits)
        for t in (1, 2):
            pb.adamw(params, grads, state[0], state[1], step=t, lr=0.1, exp_avg_scales=state[2], exp_avg_sq_scales=state[3])
        ends.append(params)
    assert all(torch.equal(a, b) for a, b in zip(*ends))
    with pytest.raises(pb.ParleError) as e:
        pb.adamw(params, [grad, params[0], grad], state[0], state[1], step=3, lr=0.1, exp_avg_scales=state[2], exp_avg_sq_scales=state[3])
    assert e.value.code == -1


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_the_norm_of_few_elements_is_correctly_rounded(dtype):
    """Of each list alone: the 64-bit norm rounded once, but where it lies as near to a tie as the sums' roundings of 2^-53 reach."""
    g = torch.Generator().manual_seed(5)
    for n in (1, 2, 3, 8, 9, 31, 64, 257, 5000):
        x = torch.randn(300 if n < 300 else 20, n, generator=g).to(dtype).to(DEV)
        out = torch.empty(len(x), device=DEV)
        for i in range(len(x)):
            pb.grad_norm([x[i].contiguous()], out=out[i:i + 1])
        for got, row in zip(f64(out), f64(x)):
            want = math.sqrt(math.fsum(v * v for v in row))
            assert abs(got - want) <= 2.0 ** (math.floor(math.log2(want)) - 24) * (1 + 1e-12) + n * 2.0 ** -53 * want, (n, got, want)


@pytest.mark.parametrize("size", [1, 16376, 16377, 16378, 16384, 16385, 2 * 16376, 32768, 10 * 16384])
@pytest.mark.parametrize("shift", [0, 1, 7])
def test_a_workspace_of_the_documented_size_is_enough(size, shift):
    flat = torch.ones(40, size + 8, dtype=torch.bfloat16, device=DEV)
    grads = [row[shift:shift + size] for row in flat.unbind()]
    ws = torch.empty(8 * 40 * -(-size // 16376) + 128, dtype=torch.uint8, device=DEV)
    assert abs(float(pb.grad_norm(grads, workspace=ws)) - math.sqrt(40 * size)) <= 2 * U * math.sqrt(40 * size)


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("size, scale, most", [(1e30, 1e10, 1.0), (1e37, 1e30, 1e3), (1e37, 64.0, 1e-3), (1e30, 2.0 ** 30, math.inf), (1e-30, 1e-12, 1.0), (1e-10, 1e20, 2.0)])
def test_a_scaled_norm_beyond_fp32_is_clipped(bits, size, scale, most):
    """max_norm / norm is an ordinary number where grad_scale norm is none."""
    n = 700
    grad = (torch.randn(n, generator=torch.Generator().manual_seed(2)) * size / 26).to(DEV)
    p = torch.zeros(n, device=DEV)
    state = pb.adamw_state([p], bits)
    norm = pb.grad_norm([grad])
    pb.adamw([p], [grad], state[0], state[1], step=1, lr=0.1, weight_decay=0.0, exp_avg_scales=state[2], exp_avg_sq_scales=state[3], norm=norm, max_norm=most, grad_scale=scale)
    g = f64(grad) * oo.coefficient(scale, float(norm), most)
    with np.errstate(over="ignore"):
        v = np.where(0.001 * np.square(g) > 3.4e38, np.inf, 0.001 * np.square(g))
    if not np.isfinite(0.1 * np.abs(g)).all() or np.abs(g).max() > 3.4e38:
        return                                              # (the gradient itself is none then)
    want = -0.1 * g / (np.sqrt(v / 0.001) + 1e-8)
    # of steps of at most 0.1: root and reciprocal 2^-22 each, the coefficient 4 u (its reciprocal is a subnormal number from 2^126 on: 2^-21), 8 products;
    # squares that are subnormal numbers are off by 2^-150 beside eps = 1e-8: nothing
    assert np.abs(f64(p) - want).max() <= 0.1 * (2.0 ** -20 + 12 * U) + 1e-12
