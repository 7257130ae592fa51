"""Pins of the token operators' oracle (CPU): known answers of Philox, finite differences, closed forms, torch in fp64."""
import math

import numpy as np
import pytest
import torch

from oracle import token_oracle as to


@pytest.mark.parametrize("counter, key, want", [      # known answers published with the generator (Random123's kat_vectors)
    ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
    ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
    ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0), (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1)),
])
def test_philox_known_answers(counter, key, want):
    assert tuple(to.philox4x32_10(counter, key)) == want


def test_dropout_keeps_a_share_of_one_minus_p_and_its_expectation():
    n, p = 40000, 0.3
    f = to.dropout_fields(n, 12345, 6)
    threshold = math.floor(p * 65536 + 0.5)
    share = (f >= threshold).mean()
    assert abs(share - (1 - threshold / 65536)) < 5 * math.sqrt(p * (1 - p) / n)       # five standard deviations
    y = to.dropout(np.ones((200, 200)), p, 12345, 6)
    assert set(np.unique(y)) == {0.0, 65536 / (65536 - threshold)}
    assert (to.dropout_fields(50, 12345, 6, first=13) == f[13:63]).all()
    assert (to.dropout_fields(64, 12345, 7) != f[:64]).any() and (to.dropout_fields(64, 12346, 6) != f[:64]).any()
    assert (to.dropout(np.full((3, 5), np.nan), 1.0, 1, 2) == 0).all()


def test_log_probabilities_against_torch_and_closed_forms():
    rng = np.random.default_rng(0)
    x = rng.normal(size=(5, 17)) * 3
    x[1, ::2] = -np.inf
    t = np.array([3, 1, -1, 16, 99])
    lp, h, top, toplp = to.token_logprobs(x, t, 0.7, 4)
    want = torch.log_softmax(0.7 * torch.from_numpy(x), dim=1)
    for r in range(5):
        assert lp[r] == (pytest.approx(want[r, t[r]].item(), abs=1e-12) if 0 <= t[r] < 17 else 0)
        p = want[r].exp()
        assert h[r] == pytest.approx(torch.special.entr(p).sum().item(), abs=1e-12)
        v, i = want[r].topk(4)
        assert top[r].tolist() == i.tolist() and np.allclose(toplp[r], v.numpy(), atol=1e-12)
    lp, h, top, toplp = to.token_logprobs(np.zeros((1, 8)), [5], 2.0, 3)
    assert lp[0] == pytest.approx(-math.log(8)) and h[0] == pytest.approx(math.log(8)) and top[0].tolist() == [0, 1, 2]
    lp, h, top, toplp = to.token_logprobs(np.array([[-np.inf] * 3, [0.0, np.nan, 1.0], [-np.inf, 2.0, -np.inf]]), [0, 0, 1], 1.0, 2)
    assert lp[0] == -np.inf and h[0] == 0 and top[0].tolist() == [-1, -1]
    assert math.isnan(lp[1]) and math.isnan(h[1]) and top[1].tolist() == [-1, -1]
    assert lp[2] == 0 and h[2] == 0 and top[2].tolist() == [1, -1] and toplp[2].tolist() == [0, -np.inf]


def test_gradient_against_differences():
    rng = np.random.default_rng(1)
    x, t, s = rng.normal(size=(3, 6)), np.array([2, -1, 5]), 1.3
    g, h = rng.normal(size=3), rng.normal(size=3)

    def loss(x):
        lp, ent, _, _ = to.token_logprobs(x, t, s)
        return float((g * lp + h * ent).sum())

    got = to.token_logprobs_grad(x, t, g, h, s)
    step = 1e-5
    for r in range(3):
        for j in range(6):
            a, b = x.copy(), x.copy()
            a[r, j] += step
            b[r, j] -= step
            assert got[r, j] == pytest.approx((loss(a) - loss(b)) / (2 * step), abs=1e-9)
    assert np.allclose(got.sum(axis=1), 0, atol=1e-15)


def test_embedding_and_its_gradient_are_adjoint_and_match_torch():
    rng = np.random.default_rng(2)
    table, tokens = rng.normal(size=(2, 7, 3)), rng.integers(-1, 9, size=(2, 11))       # -1, 7, 8: no token
    out, dout = to.embedding(table, tokens, 1.5), rng.normal(size=(2, 11, 3))
    grad, size, count = to.embedding_grad(dout, tokens, 7, 1.5)
    assert (out * dout).sum() == pytest.approx((table * grad).sum())                    # the lookup is linear in the table
    ok = torch.from_numpy((tokens >= 0) & (tokens < 7))
    w = torch.from_numpy(table).requires_grad_()
    y = torch.stack([torch.nn.functional.embedding(torch.from_numpy(tokens[g]).clamp(0, 6), w[g]) for g in range(2)]) * 1.5 * ok[..., None]
    y.backward(torch.from_numpy(dout))
    assert np.allclose(y.detach().numpy(), out) and np.allclose(w.grad.numpy(), grad) and (size >= np.abs(grad) - 1e-12).all()
    assert count.sum() == int(ok.sum())
