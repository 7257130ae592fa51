"""Token operators on the GPU against the fp64 oracle: types, odd sizes, pitches, masked rows, ties, replicas, streams, graphs.

Tolerances come from the arithmetic: u = 2^-24 is half a step of fp32 relative to the value; a base-2 exponential is off by at
most 2^-22; the last rounding of a 16-bit result by eps / 2 of it."""
import math

import numpy as np
import pytest
import torch

import paper_1707_00424_b200 as pb
from oracle import token_oracle as to

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U, E2 = 2.0 ** -24, 2.0 ** -22
TYPES = (torch.float32, torch.bfloat16, torch.float16)


def half_step(dtype, value):
    """Largest error of rounding `value` (an array) to dtype: relative, or half the smallest number."""
    if dtype == torch.float32:
        return np.zeros_like(value)
    return np.maximum(torch.finfo(dtype).eps / 2 * np.abs(value), torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps / 2)


def close(got, want, tol):
    """Equal where not finite, else within tol (an array).  A number beyond fp32's largest (a lowest-value mask times a scale
    above 1) is infinite in every type tested here."""
    got, want, tol = np.asarray(got, np.float64), np.asarray(want, np.float64), np.broadcast_to(np.asarray(tol, np.float64), np.shape(want))
    want = np.where(np.abs(want) > float(np.finfo(np.float32).max), np.copysign(np.inf, want), want)
    fine = np.isfinite(want)
    assert (np.isfinite(got) == fine).all(), np.argwhere(np.isfinite(got) != fine)[:5]
    assert np.array_equal(got[~fine], want[~fine], equal_nan=True)
    off = np.abs(got[fine] - want[fine]) - tol[fine]
    assert (off <= 0).all(), (off.max(), got[fine][off.argmax()], want[fine][off.argmax()])


def f64(t):
    return t.detach().double().cpu().numpy()


def strided(x, pad, shift=0):
    """x [rows, cols] inside a wider, shifted buffer of NaN."""
    rows, cols = x.shape
    buf = torch.full((rows * (cols + pad) + shift + 64,), math.nan, dtype=x.dtype, device=x.device)
    view = buf[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    view.copy_(x)
    return view


# ---- log probabilities ----------------------------------------------------------------------------------------------------------

def lse_error(logp, vocab, scale_range):
    """Bound on the error of log S, relative error of S: one exponential per logit (its argument is a difference, the rounded
    scale log2 e and a product: 3 u of |d|, weighted by p), sums of at most vocab / 64 terms in a thread, and at most 40 + vocab / 1024
    rescalings by an exponential on the way from a thread's sums to the row's."""
    steps = 40 + vocab / 1024
    return E2 * (1 + steps) + U * (3 * scale_range + vocab / 64 + steps)


def check_logprobs(x, tokens, scale, k, **kw):
    """x a GPU tensor [rows, vocab] (any pitch), tokens a numpy array."""
    rows, vocab = x.shape
    tok = torch.from_numpy(np.asarray(tokens, np.int32)).to(DEV)
    lp, h, top, toplp = pb.token_logprobs(x, tok, k=k, scale=scale, **kw)
    torch.cuda.synchronize()
    xs = f64(x)
    wlp, wh, wtop, wtoplp = to.token_logprobs(xs, tokens, scale, k)
    assert np.array_equal(top.cpu().numpy(), wtop)
    for r in range(rows):
        logp = to.log_softmax(xs[r], scale)
        real = logp[np.isfinite(logp)]
        p = np.exp(real)
        spread = float((p * np.abs(real - real.max())).sum()) if real.size else 0.0      # sum of p |d|
        err = lse_error(logp, vocab, spread)
        tol = lambda want: err + 4 * U * np.abs(np.where(np.isfinite(want), want, 0))    # noqa: E731
        close(f64(lp)[r], wlp[r], tol(wlp[r]))
        close(f64(toplp)[r], wtoplp[r], tol(wtoplp[r]))
        # H = log S - sum e d / S: the second quotient has twice the relative error, its terms 3 u more
        close(f64(h)[r], wh[r], err + spread * (2 * err + 6 * U) + 4 * U * (abs(wh[r]) if np.isfinite(wh[r]) else 0))


def random_rows(rows, vocab, dtype, seed, spread=3.0):
    rng = np.random.default_rng(seed)
    x = torch.from_numpy(rng.normal(size=(rows, vocab)) * spread).to(dtype).to(DEV)
    return x, rng.integers(0, vocab, size=rows), rng


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows, vocab, pad, shift, k", [
    (1, 1, 0, 0, 1), (3, 2, 0, 1, 3), (5, 7, 0, 0, 32), (4, 64, 1, 3, 5), (9, 100, 0, 0, 0), (33, 257, 0, 5, 32), (130, 1000, 0, 0, 5),
    (7, 2047, 2, 1, 20), (6, 2049, 0, 0, 20), (5, 4097, 7, 7, 32), (4, 8193, 0, 0, 8), (3, 16385, 3, 2, 32), (160, 12289, 0, 1, 3),
    (2, 33333, 0, 0, 20), (1, 50021, 0, 3, 32), (40, 50021, 0, 0, 20), (1, 131072, 0, 0, 20), (2, 131071, 0, 1, 32),
])
def test_logprobs_over_sizes(dtype, rows, vocab, pad, shift, k):
    x, tokens, rng = random_rows(rows, vocab, dtype, vocab * 31 + rows)
    tokens[rng.random(rows) < 0.2] = -1
    check_logprobs(strided(x, pad, shift), tokens, 1.0 if rows % 2 else 0.6, k)


def special_rows(vocab, dtype):
    rng = np.random.default_rng(vocab)
    low = torch.finfo(dtype).min
    base = rng.normal(size=vocab) * 2
    rows = [np.full(vocab, -np.inf), np.full(vocab, low), np.zeros(vocab), np.full(vocab, 3.25)]
    some = base.copy(); some[rng.random(vocab) < 0.7] = -np.inf; rows.append(some)
    one = np.full(vocab, -np.inf); one[vocab // 2] = -5.0; rows.append(one)
    masked = base.copy(); masked[rng.random(vocab) < 0.7] = low; rows.append(masked)
    nan = base.copy(); nan[vocab // 3] = np.nan; rows.append(nan)
    rows.append(np.where(np.arange(vocab) == vocab // 3, np.nan, -np.inf))
    inf = base.copy(); inf[vocab - 1] = np.inf; rows.append(inf)
    rows.append(np.full(vocab, np.inf))
    rows.append(np.sort(base)); rows.append(np.sort(base)[::-1].copy())
    rows.append(np.round(base))                                       # many ties
    rows.append(np.where(rng.random(vocab) < 0.5, 0.0, -0.0))         # equal zeros of both signs
    few = np.full(vocab, low); few[::max(1, vocab // 3)] = 1.0; rows.append(few)
    rows.append(base * 0 + np.where(np.arange(vocab) == vocab - 1, 60.0, 0))
    return torch.from_numpy(np.stack(rows)).to(dtype).to(DEV)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [5, 100, 1031, 9001, 70001])
@pytest.mark.parametrize("split", [False, True])
def test_logprobs_of_masked_tied_and_undefined_rows(dtype, vocab, split):
    x = special_rows(vocab, dtype)
    tokens = np.array([(7 * r + 1) % vocab for r in range(x.shape[0])])
    tokens[5] = vocab // 2
    if split:                                                         # one row at a time: few rows are shared among blocks
        for r in range(x.shape[0]):
            check_logprobs(x[r:r + 1], tokens[r:r + 1], 1.0, 7)
    else:
        for scale in (1.0, 2.5):                                      # 2.5 x the lowest number is -inf
            check_logprobs(x, tokens, scale, 32)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows", [1, 200])
def test_top_alternatives_gathered_in_few_places(dtype, rows):
    """The largest logits lie where a few threads read them: more of them pass the bound than are ranked at once."""
    vocab = 65536
    x, tokens, rng = random_rows(rows, vocab, dtype, 5)
    per = 16 // x.element_size()
    hot = (torch.arange(vocab, device=DEV) // per) % 64 < 3           # three of every 64 granules
    x = torch.where(hot, x.abs() + 20, x)
    got = pb.token_logprobs(x, k=32)[2].cpu().numpy()
    xs = f64(x)
    for r in range(0, rows, 37):
        assert got[r].tolist() == np.lexsort((np.arange(vocab), -xs[r]))[:32].tolist()


def test_logprobs_shapes_and_optional_outputs():
    x = torch.randn(3, 4, 50, device=DEV)
    t = torch.randint(0, 50, (3, 4), device=DEV, dtype=torch.int32)
    want = torch.log_softmax(x.double(), -1)
    lp, h, top, toplp = pb.token_logprobs(x, t, k=2)
    assert lp.shape == (3, 4) and top.shape == (3, 4, 2)
    assert torch.allclose(lp.double(), want.gather(-1, t.long()[..., None])[..., 0], atol=1e-5)
    lp, h, top, toplp = pb.token_logprobs(x)
    assert lp is None and top.shape == (3, 4, 0)
    one = pb.token_logprobs(x[0, 0], t[0, 0], k=1)
    assert one[0].shape == () and one[2].shape == (1,)
    assert pb.token_logprobs(x[:0], t[:0], k=3)[2].shape == (0, 4, 3)
    # only the alternatives, through the C entry point: nothing else is written
    out = torch.full((12, 2), -7, dtype=torch.int32, device=DEV)
    rc = pb.lib().parle_token_logprobs(x.data_ptr(), 0, 12, 50, 50, None, 1.0, 2, None, None, out.data_ptr(), None, None,
                                       torch.cuda.current_stream().cuda_stream)
    assert rc == 0 and torch.equal(out.view(3, 4, 2).long(), want.topk(2).indices)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [5, 1031, 9001])
@pytest.mark.parametrize("scale", [1e-6, 1e6])
def test_logprobs_at_the_smallest_and_largest_scale(dtype, vocab, scale):
    x = special_rows(vocab, dtype)
    check_logprobs(x, np.array([(7 * r + 1) % vocab for r in range(x.shape[0])]), scale, 9)


def check_grad(x, tokens, g, h, scale, inplace=False, pad=0, shift=0, outputs=False):
    rows, vocab = x.shape
    tok = torch.from_numpy(np.asarray(tokens, np.int32)).to(DEV)
    dev = lambda a: None if a is None else torch.from_numpy(np.asarray(a, np.float32)).to(DEV)      # noqa: E731
    xs = f64(x)
    gd, hd = dev(g), dev(h)
    g32, h32 = (None if a is None else f64(a) for a in (gd, hd))
    buf = x if inplace else strided(torch.zeros_like(x), pad, shift)
    lp = torch.empty(rows, device=DEV) if outputs else None
    ent = torch.empty(rows, device=DEV) if outputs else None
    assert pb.token_logprobs_grad(x, tok, gd, hd, scale, dlogits=buf, logprob=lp, entropy=ent) is buf
    torch.cuda.synchronize()
    want, got = to.token_logprobs_grad(xs, tokens, g32, h32, scale), f64(buf)
    wlp, wh, _, _ = to.token_logprobs(xs, tokens, scale)
    for r in range(rows):
        logp = to.log_softmax(xs[r], scale)
        real = logp[np.isfinite(logp)]
        spread = float((np.exp(real) * np.abs(real - real.max())).sum()) if real.size else 0.0
        err = lse_error(logp, vocab, spread)
        eh = err + spread * (2 * err + 6 * U) + 4 * U * spread
        gr = abs(float(g32[r])) if g32 is not None and 0 <= tokens[r] < vocab else 0.0
        hr = abs(float(h32[r])) if h32 is not None else 0.0
        lo = np.where(np.isfinite(logp), logp, 0.0)
        p = np.where(np.isfinite(logp), np.exp(lo), 0.0)
        d = np.abs(lo - (real.max() if real.size else 0.0))
        rel = E2 + 3 * U * d + err + 4 * U                            # of p_j = e_j / S
        H = wh[r] if np.isfinite(wh[r]) else 0.0
        # p ( a + b d ): a = -(g + h (H - log S)), b d: products and sums of terms of at most g, h (|log p| + H + d), a few u each
        tol = scale * (gr * p * rel + 4 * U * gr * (p + (np.arange(vocab) == tokens[r])) +
                       hr * p * ((np.abs(lo) + H) * rel + eh + err + 8 * U * (np.abs(lo) + H + d + abs(math.log(vocab)))))
        tol = tol + 1e-37 * (1 + scale * (gr + hr * 100))             # probabilities below fp32's smallest normal count as 0
        close(got[r], want[r], tol + half_step(x.dtype, want[r]))
        if outputs:
            close(f64(lp)[r], wlp[r], err + 4 * U * abs(np.nan_to_num(wlp[r], posinf=0, neginf=0)))
            close(f64(ent)[r], wh[r], eh + 4 * U * H)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows, vocab, pad, shift", [
    (1, 1, 0, 0), (3, 2, 0, 1), (4, 64, 1, 3), (20, 100, 0, 0), (9, 257, 0, 5), (65, 1000, 0, 0), (7, 2047, 2, 1), (6, 4097, 7, 7),
    (3, 16385, 3, 2), (2, 33333, 0, 1), (40, 50021, 0, 0), (1, 131072, 0, 0), (2, 131071, 0, 1),
])
def test_gradient_over_sizes(dtype, rows, vocab, pad, shift):
    x, tokens, rng = random_rows(rows, vocab, dtype, vocab * 17 + rows)
    tokens[rng.random(rows) < 0.2] = -1
    g, h = rng.normal(size=rows), rng.normal(size=rows) * 0.3
    g[rng.random(rows) < 0.2] = 0
    check_grad(strided(x, pad, shift), tokens, g, None, 1.0, pad=pad, shift=shift, outputs=True)
    check_grad(strided(x, pad, shift), tokens, g, h, 0.6, pad=0, shift=2, outputs=False)
    check_grad(strided(x, 0, shift), tokens, None, h, 1.7, inplace=True, outputs=True)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [5, 100, 1031, 9001, 70001])
@pytest.mark.parametrize("split", [False, True])
def test_gradient_of_masked_and_undefined_rows(dtype, vocab, split):
    x = special_rows(vocab, dtype)
    rows = x.shape[0]
    tokens = np.array([(7 * r + 1) % vocab for r in range(rows)])
    tokens[5] = vocab // 2
    rng = np.random.default_rng(3)
    g, h = rng.normal(size=rows), rng.normal(size=rows)
    for r in range(rows) if split else (slice(None),):
        cut = slice(r, r + 1) if split else r
        check_grad(x[cut], tokens[cut], g[cut], h[cut], 1.0, outputs=True)
        check_grad(x[cut], tokens[cut], g[cut], None, 1.0)
        check_grad(x[cut].clone(), tokens[cut], g[cut] * 0, None, 1.0, inplace=True, outputs=True)


def test_logprobs_beyond_32_bit_offsets():
    rows, vocab = 33000, 131072                                            # 4.3e9 logits
    x = torch.zeros(rows, vocab, dtype=torch.bfloat16, device=DEV)
    pick = torch.tensor([0, 16383, 16384, 32767, 32768, rows - 1], device=DEV)
    x[pick] = torch.randn(6, vocab, device=DEV).bfloat16()
    t = torch.randint(0, vocab, (rows,), device=DEV, dtype=torch.int32)
    lp, h, top, toplp = pb.token_logprobs(x, t, k=3)
    few = pb.token_logprobs(x[pick].contiguous(), t[pick].contiguous(), k=3)
    # the few rows are summed by other blocks: another order of the same sums
    assert torch.allclose(lp[pick], few[0], atol=1e-5) and torch.allclose(h[pick], few[1], atol=1e-4) and torch.equal(top[pick], few[2])
    g = torch.randn(rows, device=DEV)
    want = pb.token_logprobs_grad(x[pick].contiguous(), t[pick].contiguous(), g[pick].contiguous())
    pb.token_logprobs_grad(x, t, g, dlogits=x)
    assert torch.allclose(x[pick].float(), want.float(), rtol=2 ** -7, atol=1e-7)       # a step of bf16
    del x, want
    torch.cuda.empty_cache()


def test_rows_without_an_incoming_gradient_are_zero_whatever_their_logits():
    x = torch.full((3, 70001), math.nan, device=DEV, dtype=torch.bfloat16)
    x[1] = 1.0
    t = torch.tensor([4, -1, -1], dtype=torch.int32, device=DEV)
    d = pb.token_logprobs_grad(x, t, torch.tensor([0.0, 5.0, math.nan], device=DEV))
    assert (d == 0).all()


def test_gradient_against_differences_of_the_kernel_itself():
    torch.manual_seed(0)
    x = torch.randn(6, 40, device=DEV)
    t = torch.randint(0, 40, (6,), device=DEV, dtype=torch.int32)
    g, h = torch.randn(6, device=DEV), torch.randn(6, device=DEV)
    got = pb.token_logprobs_grad(x, t, g, h, 1.3)
    step = 2.0 ** -5
    for j in (0, 7, 39):
        v = []
        for sign in (1, -1):
            y = x.clone()
            y[:, j] += sign * step
            lp, ent, _, _ = pb.token_logprobs(y, t, scale=1.3)
            v.append((g * lp + h * ent).double())
        # third derivative of log p and H times s^3 is at most a few; outputs are off by 1e-6 each
        assert torch.allclose((v[0] - v[1]) / (2 * step), got[:, j].double(), atol=step ** 2 * 10 + 2e-6 / step)


def test_bad_tokens_set_the_flag_and_count_as_none():
    x = torch.randn(4, 30, device=DEV)
    flags = torch.zeros(1, dtype=torch.int32, device=DEV)
    t = torch.tensor([0, -1, 29, 5], dtype=torch.int32, device=DEV)
    pb.token_logprobs(x, t, flags=flags)
    pb.token_logprobs_grad(x, t, torch.ones(4, device=DEV), flags=flags)
    pb.embedding(x, t % 4, flags=flags); pb.embedding(x, t.clamp(max=3), flags=flags); pb.embedding_grad(x, t, 30, flags=flags)
    assert flags.item() == 0
    for length in (1500, 6000, 40000):                                    # each way of sorting
        many, rows = torch.randint(-1, 30, (length,), dtype=torch.int32, device=DEV), torch.randn(length, 8, device=DEV)
        want = pb.embedding_grad(rows, many, 30, flags=flags)
        assert flags.item() == 0
        wrong = torch.where(many == -1, torch.full_like(many, 30), many)
        assert torch.equal(pb.embedding_grad(rows, wrong, 30, flags=flags), want) and flags.item() == pb.FLAG_BAD_LABEL
        flags.zero_()
    bad = torch.tensor([30, -2, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device=DEV)
    for call in (lambda: pb.token_logprobs(x, bad, flags=flags)[0], lambda: pb.embedding(x, bad, flags=flags),
                 lambda: pb.embedding_grad(x, bad, 30, flags=flags), lambda: pb.token_logprobs_grad(x, bad, torch.ones(4, device=DEV), flags=flags)):
        flags.zero_()
        assert (call() == 0).all() and flags.item() == pb.FLAG_BAD_LABEL


# ---- embedding ------------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("out_type", TYPES)
@pytest.mark.parametrize("table_type", TYPES)
@pytest.mark.parametrize("n, length, vocab, dim, pad, scale", [
    (1, 1, 1, 1, 0, 1.0), (1, 1, 50, 4096, 0, 1.0), (1, 7, 30, 33, 1, 2.5), (2, 5, 11, 64, 0, -0.3), (3, 129, 100, 100, 4, 1.0),
    (1, 300, 20, 2056, 8, 11.3), (64, 2, 3, 8, 0, 1.0),
])
def test_embedding_rows(table_type, out_type, n, length, vocab, dim, pad, scale):
    rng = np.random.default_rng(n * 100 + length)
    tokens = rng.integers(-1, vocab + 2, size=(n, length)).astype(np.int32)
    table = torch.from_numpy(rng.normal(size=(n, vocab, dim + pad))).to(table_type).to(DEV)[:, :, :dim]
    out = torch.full((n, length, dim + pad), math.nan, dtype=out_type, device=DEV)
    got = pb.embedding(table, torch.from_numpy(tokens).to(DEV), scale, out=out[:, :, :dim])
    want = to.embedding(f64(table), tokens, scale)
    close(f64(got), want, 3 * U * np.abs(want) + half_step(out_type, want))
    assert torch.isnan(out[:, :, dim:]).all()                          # what lies between the rows is left alone


def test_embedding_layouts():
    torch.manual_seed(1)
    table = torch.randn(40, 24, device=DEV)
    t = torch.randint(0, 40, (3, 5), device=DEV, dtype=torch.int32)
    assert torch.equal(pb.embedding(table, t), table[t.long()])
    assert pb.embedding(table, t[0, 0]).shape == (24,) and pb.embedding(table, t[:0]).shape == (0, 5, 24)
    assert pb.embedding(table, t, dtype=torch.bfloat16).dtype == torch.bfloat16
    # replicas side by side in every row of the output, tables expanded from one
    out = torch.empty(5, 3, 24, device=DEV)
    pb.embedding(table.expand(3, 40, 24), t, out=out.transpose(0, 1))
    assert torch.equal(out.transpose(0, 1), table[t.long()])
    # a table inside parameter vectors [n, stride]
    flat = torch.randn(3, 40 * 24 + 32, device=DEV)
    tables = flat[:, 32:].view(3, 40, 24)
    assert torch.equal(pb.embedding(tables, t), torch.stack([tables[g][t[g].long()] for g in range(3)]))


def test_embedding_beyond_32_bit_offsets():
    table = torch.zeros(300000, 8192, dtype=torch.bfloat16, device=DEV)      # 2.46e9 elements
    last = torch.tensor([299999, 262144, 0], dtype=torch.int32, device=DEV)
    table[last.long()] = torch.arange(3, device=DEV, dtype=torch.bfloat16)[:, None] + 1
    assert torch.equal(pb.embedding(table, last), table[last.long()])
    del table
    torch.cuda.empty_cache()
    grad = torch.full((300000, 8192), 7.0, device=DEV)
    dout = torch.ones(3, 8192, device=DEV)
    pb.embedding_grad(dout, last, 300000, 2.0, dtable=grad)
    assert (grad[last.long()] == 2).all() and grad.sum(dtype=torch.float64).item() == 3 * 8192 * 2
    pb.embedding_grad(dout, last, 300000, 1.0, dtable=grad, accumulate=True)
    assert (grad[last.long()] == 3).all()
    del grad
    torch.cuda.empty_cache()


def test_embedding_gradient_of_an_input_beyond_32_bit_offsets():
    length, vocab, dim = 540000, 700, 8192                                # 4.4e9 elements
    dout = torch.zeros(length, dim, dtype=torch.bfloat16, device=DEV)
    pick = [0, 262143, 262144, 524287, 524288, length - 1]
    t = torch.randint(0, vocab, (length,), device=DEV, dtype=torch.int32)
    want = torch.zeros(vocab, device=DEV)
    for i, at in enumerate(pick):
        dout[at] = i + 1
        want[t[at]] += i + 1
    got = pb.embedding_grad(dout, t, vocab)
    assert torch.equal(got, want[:, None].expand(vocab, dim))
    del dout, got
    torch.cuda.empty_cache()


def check_embedding_grad(dout, tokens, vocab, scale, accumulate=False, pad=0, start=None):
    n, length, dim = dout.shape
    buf = torch.full((n, vocab, dim + pad), 0.75 if accumulate else math.nan, device=DEV)
    before = buf.clone()
    got = pb.embedding_grad(dout, torch.from_numpy(tokens).to(DEV), vocab, scale, dtable=buf[:, :, :dim], accumulate=accumulate)
    again = before.clone()
    pb.embedding_grad(dout, torch.from_numpy(tokens).to(DEV), vocab, scale, dtable=again[:, :, :dim], accumulate=accumulate)
    assert torch.equal(buf.view(torch.int32), again.view(torch.int32))         # the same bits every time
    want, size, count = to.embedding_grad(f64(dout), tokens, vocab, scale)
    # a sum of c terms in any order is off by at most (c - 1) u of the terms' sizes; the scale, its product and an addition: 3 u
    tol = U * (count[:, :, None] + 3) * size
    if accumulate:
        tol, want = tol + 2 * U * (np.abs(want) + 0.75), want + 0.75
        absent = count == 0
        assert (f64(got)[absent] == 0.75).all()
    close(f64(got), want, tol)
    assert torch.equal(buf[:, :, dim:].contiguous().view(torch.int32), before[:, :, dim:].contiguous().view(torch.int32))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n, length, vocab, dim, pad", [
    (1, 1, 1, 1, 0), (1, 1, 100, 64, 0), (1, 31, 40, 33, 1), (2, 32, 7, 8, 0), (1, 33, 5, 100, 4), (3, 65, 1000, 16, 0), (1, 257, 3, 264, 8),
    (8, 640, 100, 101, 0), (1, 1000, 1, 24, 0), (1, 8192, 37, 8, 0), (2, 8193, 300, 9, 0), (1, 16384, 300, 520, 0), (1, 20000, 70000, 8, 0), (1, 1025, 17000000, 1, 0),
])
def test_embedding_gradient(dtype, n, length, vocab, dim, pad):
    rng = np.random.default_rng(length + vocab)
    tokens = rng.integers(-1, vocab + 1, size=(n, length)).astype(np.int32)
    dout = torch.from_numpy(rng.normal(size=(n, length, dim + pad))).to(dtype).to(DEV)[:, :, :dim]
    check_embedding_grad(dout, tokens, vocab, 1.0, pad=pad)
    check_embedding_grad(dout, tokens, vocab, -2.3, accumulate=True, pad=pad)


@pytest.mark.parametrize("length", [1, 32, 33, 64, 100, 1024, 1025, 4099, 32768, 32769, 40001])
def test_embedding_gradient_of_skewed_tokens(length):
    """All positions the same token, none at all, a block of one token amid others, tokens in ascending and descending order."""
    vocab, dim = 50, 40 if length <= 4099 else 8
    rng = np.random.default_rng(length)
    dout = torch.from_numpy(rng.normal(size=(5, length, dim))).to(torch.bfloat16).to(DEV)
    tokens = np.empty((5, length), np.int32)
    tokens[0], tokens[1] = 17, -1
    tokens[2] = rng.integers(0, vocab, size=length)
    tokens[2, length // 4:length // 2 + 1] = 3
    tokens[3] = np.arange(length) * vocab // length
    tokens[4] = (vocab - 1) - tokens[3]
    check_embedding_grad(dout, tokens, vocab, 1.0)
    check_embedding_grad(dout, tokens, vocab, 0.5, accumulate=True)


def test_embedding_gradient_forms():
    torch.manual_seed(2)
    t = torch.randint(0, 9, (4, 6), device=DEV, dtype=torch.int32)
    d = torch.randn(4, 6, 16, device=DEV)
    want = torch.zeros(9, 16, device=DEV, dtype=torch.float64).index_add_(0, t.flatten().long(), d.flatten(0, 1).double())
    assert torch.allclose(pb.embedding_grad(d, t, 9).double(), want, atol=1e-5)
    per = pb.embedding_grad(d, t, 9, n=4)
    assert per.shape == (4, 9, 16) and torch.allclose(per.double().sum(0), want, atol=1e-5)
    assert (pb.embedding_grad(d[:0], t[:0], 9) == 0).all()
    keep = torch.full((9, 16), 3.0, device=DEV)
    assert (pb.embedding_grad(d[:0], t[:0], 9, dtable=keep, accumulate=True) == 3).all()
    # a gradient that is one row for every position (as after a sum)
    row = torch.randn(16, device=DEV)
    wide = pb.embedding_grad(row.expand(4, 6, 16), t, 9)
    count = torch.bincount(t.flatten(), minlength=9).double()
    assert torch.allclose(wide.double(), count[:, None] * row.double(), atol=1e-5)
    # a given workspace that held something else
    t, d = torch.randint(0, 9, (17000,), device=DEV, dtype=torch.int32), torch.randn(17000, 16, device=DEV)
    ws = torch.full((pb.embedding_grad_workspace_bytes(1, 17000, 9, 16),), 255, dtype=torch.uint8, device=DEV)
    assert torch.equal(pb.embedding_grad(d, t, 9, workspace=ws), pb.embedding_grad(d, t, 9))
    with pytest.raises(pb.ParleError) as e:
        pb.embedding_grad(d, t, 9, workspace=ws[:-1])
    assert e.value.code == -6


# ---- dropout --------------------------------------------------------------------------------------------------------------------

def check_dropout(x, p, seed, offset, residual=None, **kw):
    got = pb.dropout(x, p, seed, offset, residual=residual, **kw)
    flat = lambda t: None if t is None else f64(t).reshape(-1, t.shape[-1])      # noqa: E731
    want = to.dropout(flat(x), p, seed, offset, flat(residual))
    r = 0 if residual is None else np.abs(flat(residual))
    size = np.abs(np.nan_to_num(want)) + 2 * r                         # |x scale| <= |y| + |r|
    close(flat(got), want, 3 * U * size + half_step(x.dtype, np.nan_to_num(want)))
    return got


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows, cols, pad, shift", [
    (1, 1, 0, 0), (1, 7, 0, 1), (1, 8, 0, 0), (1, 4099, 0, 0), (3, 5, 0, 0), (7, 16, 0, 0), (5, 16, 8, 0), (5, 24, 3, 1), (17, 255, 0, 3),
    (9, 257, 1, 0), (33, 1001, 22, 5), (64, 64, 0, 0), (100, 3, 2, 0), (3, 9000, 8, 0), (2, 20011, 3, 1), (5, 248, 1, 0), (40, 8, 8, 0),
])
def test_dropout(dtype, rows, cols, pad, shift):
    rng = np.random.default_rng(rows * cols)
    x = torch.from_numpy(rng.normal(size=(rows, cols))).to(dtype).to(DEV)
    r = torch.from_numpy(rng.normal(size=(rows, cols))).to(dtype).to(DEV)
    for p, seed, offset in ((0.1, 1, 0), (0.5, 2 ** 64 - 1, 2 ** 64 - 1), (0.9, 0x123456789ABCDEF, 1 << 40)):
        check_dropout(strided(x, pad, shift), p, seed, offset)
        check_dropout(strided(x, pad, shift), p, seed, offset, residual=strided(r, pad, shift + 1))
        out = strided(torch.zeros_like(x), pad, shift)
        check_dropout(strided(x, pad, shift), p, seed, offset, residual=r, out=out)
    for p, want in ((0.0, x), (1.0, torch.zeros_like(x))):
        assert torch.equal(pb.dropout(strided(x, pad, shift), p, 5), want)
        assert torch.equal(pb.dropout(x, p, 5, residual=r), (want.float() + r.float()).to(dtype))
    # in place, over x and over the residual
    y = pb.dropout(x, 0.5, 3, 4, residual=r)
    a, b = strided(x, pad, shift), strided(r, pad, shift)
    assert torch.equal(pb.dropout(a, 0.5, 3, 4, residual=r, out=a), y) and torch.equal(pb.dropout(x, 0.5, 3, 4, residual=b, out=b), y)


@pytest.mark.parametrize("dtype", TYPES)
def test_dropout_mask_does_not_depend_on_type_or_pitch_and_drops_nan(dtype):
    ones = torch.ones(50, 72, device=DEV)
    want = pb.dropout(ones, 0.3, 11, 2) > 0
    x = ones.to(dtype)
    assert torch.equal(pb.dropout(x, 0.3, 11, 2) > 0, want)
    assert torch.equal(pb.dropout(strided(x, 5, 3), 0.3, 11, 2) > 0, want)
    assert torch.equal(pb.dropout(x.view(5, 10, 72), 0.3, 11, 2).view(50, 72) > 0, want)
    nan = torch.full_like(x, math.nan)
    assert torch.equal(torch.isnan(pb.dropout(nan, 0.3, 11, 2)), want) and (pb.dropout(nan, 0.3, 11, 2)[~want] == 0).all()
    assert not torch.equal(pb.dropout(x, 0.3, 11, 3) > 0, want)


def test_dropout_beyond_32_bit_offsets():
    n = (1 << 32) + 4099
    x = torch.ones(n, dtype=torch.bfloat16, device=DEV)
    pb.dropout(x, 0.5, 9, 1, out=x)
    for first in (0, (1 << 31) - 40, (1 << 32) - 40, n - 100):
        field = to.dropout_fields(100, 9, 1, first=first)
        assert np.array_equal(f64(x[first:first + 100]) > 0, field >= 32768)
    del x
    torch.cuda.empty_cache()


def test_dropout_gradient_is_the_same_call():
    torch.manual_seed(3)
    x, dy = torch.randn(20, 40, device=DEV), torch.randn(20, 40, device=DEV)
    dx = pb.dropout(dy, 0.4, 77, 5)
    # linear in x: <dy, dropout(x)> = <dropout(dy), x>, element by element
    assert torch.allclose(dy * pb.dropout(x, 0.4, 77, 5), dx * x, rtol=3 * 2 ** -23)


# ---- streams, graphs, refusals --------------------------------------------------------------------------------------------------

def every_call(stream=None):
    """(name, call(out) -> tuple of outputs) of every operator on fixed inputs."""
    torch.manual_seed(4)
    x, t = torch.randn(40, 9000, device=DEV, dtype=torch.bfloat16), torch.randint(0, 9000, (40,), device=DEV, dtype=torch.int32)
    g, one = torch.randn(40, device=DEV), torch.randn(1, 70000, device=DEV)
    e, long = torch.randn(40, 9000, device=DEV), torch.randint(0, 300, (34000,), device=DEV, dtype=torch.int32)
    rows = torch.randn(34000, 40, device=DEV)
    torch.cuda.synchronize()
    return {
        "logprobs": lambda: pb.token_logprobs(x, t, k=9, stream=stream),
        "logprobs split": lambda: pb.token_logprobs(one, k=9, stream=stream)[1:],
        "gradient": lambda: (pb.token_logprobs_grad(x, t, g, g, stream=stream),),
        "embedding": lambda: (pb.embedding(e, t % 40, stream=stream),),
        "embedding gradient": lambda: (pb.embedding_grad(e, t, 9000, stream=stream),),
        "embedding gradient, long": lambda: (pb.embedding_grad(rows, long, 300, stream=stream),),
        "embedding gradient, middle": lambda: (pb.embedding_grad(rows[:5000], long[:5000], 300, stream=stream),),
        "dropout": lambda: (pb.dropout(e, 0.2, 8, 1, residual=e, stream=stream),),
    }


def test_calls_on_another_stream_and_two_at_once():
    want = {name: call() for name, call in every_call().items()}
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    first, second = every_call(a), every_call(b)
    got = {name: (first[name](), second[name]()) for name in want}
    torch.cuda.synchronize()
    for name in want:
        for pair in got[name]:
            for u, v in zip(want[name], pair):
                assert torch.equal(u, v), name


def test_captured_calls_replay():
    calls = every_call()
    want = {name: call() for name, call in calls.items()}
    for name, call in calls.items():
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = call()
        for _ in range(2):
            for o in out:
                o.fill_(-5)
            graph.replay()
            torch.cuda.synchronize()
            for u, v in zip(want[name], out):
                assert torch.equal(u, v), name


def test_a_replayed_dropout_draws_a_new_mask_when_the_caller_advances_the_offset():
    x, step = torch.ones(1000, device=DEV), torch.zeros(1, dtype=torch.int64, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = pb.dropout(x, 0.5, 6, 100, offset_dev=step)
        step.add_(1)
    for k in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, pb.dropout(x, 0.5, 6, 100 + k))


def test_the_functions_refuse():
    x, t = torch.zeros(4, 8, device=DEV), torch.zeros(4, dtype=torch.int32, device=DEV)
    bad = [
        lambda: pb.token_logprobs(x.double(), t), lambda: pb.token_logprobs(x, t.long()), lambda: pb.token_logprobs(x, t[:3]),
        lambda: pb.token_logprobs(x.t(), t), lambda: pb.token_logprobs(x, t, k=33), lambda: pb.token_logprobs(x, logprob=torch.zeros(4, device=DEV)),
        lambda: pb.token_logprobs(x, t, scale=0.0), lambda: pb.token_logprobs(x, t, entropy=torch.zeros(8, device=DEV)[::2]),
        lambda: pb.token_logprobs(x, t.cpu()), lambda: pb.token_logprobs(x, t, flags=torch.zeros(1, device=DEV)),
        lambda: pb.token_logprobs(x[:, :0], t), lambda: pb.token_logprobs(torch.zeros(2, 3, 8, device=DEV).transpose(0, 1), t),
        lambda: pb.token_logprobs_grad(x, t), lambda: pb.token_logprobs_grad(x, None, torch.zeros(4, device=DEV)),
        lambda: pb.token_logprobs_grad(x, t, torch.zeros(4, device=DEV), dlogits=x.bfloat16()),
        lambda: pb.token_logprobs_grad(x, t, torch.zeros(4, device=DEV), dlogits=torch.zeros(1, 8, device=DEV).expand(4, 8)),
        lambda: pb.embedding(x, t.long()), lambda: pb.embedding(x[0], t), lambda: pb.embedding(x[None].expand(3, 4, 8), t),
        lambda: pb.embedding(x, t, out=torch.zeros(4, 9, device=DEV)), lambda: pb.embedding(x, t, math.nan),
        lambda: pb.embedding(x, t, out=torch.zeros(1, 8, device=DEV).expand(4, 8)),
        lambda: pb.embedding_grad(x, t[:3], 5), lambda: pb.embedding_grad(x, t, 5, accumulate=True),
        lambda: pb.embedding_grad(x, t, 5, dtable=torch.zeros(6, 8, device=DEV)), lambda: pb.embedding_grad(x, t, 0),
        lambda: pb.embedding_grad(x, t, 5, dtable=torch.zeros(5, 8, device=DEV).bfloat16()),
        lambda: pb.embedding_grad(x, t, 5, dtable=torch.zeros(1, 8, device=DEV).expand(5, 8)),
        lambda: pb.embedding_grad(torch.zeros(1, device=DEV).expand(4, 8), t, 5),
        lambda: pb.dropout(x, 1.5, 1), lambda: pb.dropout(x, 0.5, -1), lambda: pb.dropout(x, 0.5, 1, 1 << 64), lambda: pb.dropout(x, 0.5, 1, residual=x[:2]),
        lambda: pb.dropout(x, 0.5, 1, out=x.half()), lambda: pb.dropout(x.t(), 0.5, 1), lambda: pb.dropout(x, 0.5, 1, offset_dev=t),
        lambda: pb.dropout(x, 0.5, 1, offset_dev=torch.zeros(1, dtype=torch.int64)), lambda: pb.dropout(x.int(), 0.5, 1),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(pb.ParleError) as e:
            call()
        assert e.value.code == -1, i
    torch.cuda.synchronize()


# ---- together, as they are used -------------------------------------------------------------------------------------------------

def test_a_bigram_model_trained_by_flat_replicas():
    """n replicas of a table of logits [vocab, vocab] in flat parameter vectors: lookup of the previous token's row, dropout, log
    probabilities of the next token, gradient back through both into `grad`, and the library's own inner update -- against the
    same steps in fp64."""
    n, vocab, length, steps, p = 3, 37, 200, 3, 0.25
    m = pb.Parle(n, (vocab * vocab,), 0, eta=0.5, eta_prime=0.5, gamma=2.0, rho=1.0).alloc(DEV)
    rng = np.random.default_rng(0)
    x0 = rng.normal(size=(n, vocab * vocab)).astype(np.float32)
    m.x[:, :vocab * vocab] = torch.from_numpy(x0).to(DEV)
    m.mean()
    tables = lambda flat: flat[:, :vocab * vocab].view(n, vocab, vocab)                  # noqa: E731
    seq = rng.integers(0, vocab, size=(steps, n, length + 1)).astype(np.int32)
    seq[:, :, -20:] = -1                                                # padding
    weight = np.float32(-1.0 / (n * length))
    m.round_begin()
    x, y, z = x0.astype(np.float64), x0.astype(np.float64), x0.astype(np.float64)
    for k in range(steps):
        prev, nxt = (torch.from_numpy(np.ascontiguousarray(seq[k][:, a:a + length])).to(DEV) for a in (0, 1))
        e = pb.embedding(tables(m.x if k == 0 else m.y), prev, 1.5)
        logits = pb.dropout(e, p, 42, k)
        d = pb.token_logprobs_grad(logits, nxt, torch.full((n, length), float(weight), device=DEV), dlogits=logits)
        pb.dropout(d, p, 42, k, out=d)
        pb.embedding_grad(d, prev, vocab, 1.5, dtable=tables(m.grad))
        m.inner_update(m.grad)
        # the same in fp64
        we = to.embedding(y.reshape(n, vocab, vocab), seq[k][:, :length], 1.5)
        mask = to.dropout(np.ones((n * length, vocab)), p, 42, k).reshape(n, length, vocab)
        wd = to.token_logprobs_grad((we * mask).reshape(-1, vocab), seq[k][:, 1:].reshape(-1), np.full(n * length, weight), None)
        wg, _, _ = to.embedding_grad(wd.reshape(n, length, vocab) * mask, seq[k][:, :length], vocab, 1.5)
        y = y - 0.5 * (wg.reshape(n, -1) + (y - x) / 2.0)
        z = 0.75 * z + 0.25 * y
    torch.cuda.synchronize()
    assert m.status() == 0
    # y moves by gradients of at most a few 1e-2 a step, each off by some 1e-5 relative; y itself is rounded three times a step
    for got, want in ((m.y, y), (m.z, z)):
        assert np.abs(f64(got)[:, :vocab * vocab] - want).max() < 1e-5
    assert (m.grad[:, vocab * vocab:] == 0).all()


def test_embedded_and_dropped_minibatches_through_an_inner_step():
    """Contexts of three tokens from replicas' tables, input dropout, the MLP's inner step, and the alternatives to its labels from
    the step's logits."""
    n, B, ctx, vocab, dim, classes = 2, 16, 3, 29, 8, 29
    m = pb.Parle(n, (ctx * dim, 64, classes), B).alloc(DEV)
    gen = torch.Generator(device=DEV).manual_seed(1)
    for layer in range(2):                                              # the padding between the segments stays zero
        w, _ = m.layer_offset(layer)
        m.x[:, w:w + m.dims[layer] * m.dims[layer + 1]].normal_(0, 0.2, generator=gen)
    m.mean()
    tables = torch.randn(n, vocab, dim, device=DEV, generator=gen)
    tokens = torch.randint(0, vocab, (n, B, ctx), device=DEV, generator=gen, dtype=torch.int32)
    labels = torch.randint(0, classes, (n, B), device=DEV, generator=gen, dtype=torch.int32)
    inputs = torch.empty(n, B, ctx * dim, device=DEV)
    pb.embedding(tables, tokens, out=inputs.view(n, B, ctx, dim))
    pb.dropout(inputs, 0.1, 5, 0, out=inputs)
    loss = torch.empty(n, device=DEV)
    m.round_begin()
    m.inner_step(inputs, labels, loss)
    logits = m.debug_buffer(m.DBG_LOGITS)
    lp, h, top, toplp = pb.token_logprobs(logits, labels, k=5)
    torch.cuda.synchronize()
    # the step's loss is the mean of -log p of its labels, both from the same logits: fp32 rounding of the step's own kernel
    assert torch.allclose(loss, -lp.mean(dim=1), rtol=1e-5, atol=1e-5)
    assert torch.equal(top.long(), logits.topk(5).indices) and (h > 0).all() and (toplp[..., 0] >= lp).all()


# ---- rows by larger blocks, two groups of logits a thread -----------------------------------------------------------------------

LONG = {torch.float32: 100003, torch.bfloat16: 200001, torch.float16: 200001}      # longer than eight blocks of 256 threads hold


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows, pad, shift, k", [(1, 0, 0, 32), (13, 1, 3, 8), (20, 0, 0, 0), (50, 0, 1, 5)])
def test_logprobs_of_very_long_rows(dtype, rows, pad, shift, k):
    x, tokens, rng = random_rows(rows, LONG[dtype], dtype, rows)
    check_logprobs(strided(x, pad, shift), tokens, 0.7, k)


@pytest.mark.parametrize("dtype", TYPES)
def test_masked_tied_and_undefined_rows_of_very_long_rows(dtype):
    vocab = LONG[dtype]
    x = special_rows(vocab, dtype)
    tokens = np.array([(7 * r + 1) % vocab for r in range(x.shape[0])])
    check_logprobs(x, tokens, 1.0, 9)
    rng = np.random.default_rng(1)
    g, h = rng.normal(size=x.shape[0]), rng.normal(size=x.shape[0])
    for inplace in (False, True):
        check_grad(x.clone(), tokens, g, h, 1.0, inplace=inplace)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows, granules, pad, shift", [(1, 1300, 0, 0), (148, 1025, 1, 1), (149, 2047, 0, 0), (1, 2049, 0, 0), (5, 4095, 3, 2),
                                                        (296, 2100, 0, 0), (297, 2100, 0, 0), (3, 16700, 0, 0), (20, 20000, 5, 1)])
def test_gradient_of_few_rows_by_larger_blocks(dtype, rows, granules, pad, shift):
    vocab = granules * (4 if dtype == torch.float32 else 8) - 3
    x, tokens, rng = random_rows(rows, vocab, dtype, granules)
    tokens[rng.random(rows) < 0.2] = -1
    g, h = rng.normal(size=rows), rng.normal(size=rows) * (rows % 2)
    check_grad(x, tokens, g, h, 0.8, inplace=rows % 3 == 0, pad=pad, shift=shift)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows, vocab, pad, shift, k", [(300, 150, 0, 0, 20), (70, 150, 3, 1, 32), (50, 500, 0, 0, 25), (9, 1011, 0, 2, 32), (6, 2039, 0, 0, 32),
                                                        (40, 33, 0, 0, 32), (40, 31, 1, 0, 32), (17, 8, 0, 0, 2), (17, 9, 0, 1, 2)])
def test_many_alternatives_of_short_rows(dtype, rows, vocab, pad, shift, k):
    x, tokens, rng = random_rows(rows, vocab, dtype, vocab)
    x[::3] = x[::3].round()                                           # ties
    x[1::3] = torch.where(torch.rand(x[1::3].shape, generator=torch.Generator().manual_seed(vocab)).to(DEV) < 0.8, -math.inf, x[1::3])
    check_logprobs(strided(x, pad, shift), tokens, 1.0, k)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n, length, vocab, dim, pad", [
    (1, 1025, 40, 256, 1), (1, 1056, 3, 257, 0), (2, 1100, 500, 511, 1), (1, 2000, 33, 512, 2), (1, 1500, 700, 513, 0), (1, 1300, 50, 769, 0),
    (3, 1057, 9, 1023, 1), (1, 4200, 2000, 1025, 0), (1, 1040, 64, 2051, 0), (1, 9000, 11, 900, 4),
])
def test_embedding_gradient_of_rows_off_16_byte_boundaries(dtype, n, length, vocab, dim, pad):
    """Skewed tokens: runs inside a chunk, over one border and over many."""
    rng = np.random.default_rng(dim)
    tokens = np.minimum(np.exp(rng.random((n, length)) * math.log(vocab + 1)) - 1, vocab - 1).astype(np.int32)
    tokens[rng.random((n, length)) < 0.05] = -1
    dout = torch.from_numpy(rng.normal(size=(n, length, dim + pad))).to(dtype).to(DEV)[:, :, :dim]
    check_embedding_grad(dout, tokens, vocab, 0.9, pad=pad)
    check_embedding_grad(dout, tokens, vocab, -1.7, accumulate=True, pad=pad)


@pytest.mark.parametrize("dtype", TYPES)
def test_dropout_of_rows_at_every_place_against_16_byte_boundaries(dtype):
    rng = np.random.default_rng(8)
    for shift in range(9):
        for cols, pad in ((100, 1), (33, 0), (257, 5), (600, 3), (40, 4), (9, 2)):
            x = torch.from_numpy(rng.normal(size=(5, cols))).to(dtype).to(DEV)
            r = torch.from_numpy(rng.normal(size=(5, cols))).to(dtype).to(DEV)
            want = pb.dropout(x, 0.4, 6, 1, residual=r)               # contiguous, on 16-byte boundaries
            out = torch.full((5 * (cols + 3) + 40,), 7.0, dtype=dtype, device=DEV)
            view = out[8 - shift:8 - shift + 5 * (cols + 3)].view(5, cols + 3)[:, :cols]
            pb.dropout(strided(x, pad, shift), 0.4, 6, 1, residual=strided(r, pad + 1, 2 * shift + 1), out=view)
            assert torch.equal(view, want)
            left = torch.ones_like(out, dtype=torch.bool)
            left[8 - shift:8 - shift + 5 * (cols + 3)].view(5, cols + 3)[:, :cols] = False
            assert bool((out[left] == 7).all())                       # nothing beside the rows is written
            for at in (strided(x, pad, shift), strided(x, 0, shift)):
                assert torch.equal(pb.dropout(at, 0.4, 6, 1, residual=r, out=at), want)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows, cols, pad, shift", [(5001, 1003, 2, 1), (9000, 33, 5, 0), (3000, 95, 1, 3), (2800, 96, 1, 0), (1, 300007, 0, 3), (700, 1001, 0, 1),
                                                    (1100, 247, 0, 2), (1100, 248, 1, 0), (20100, 121, 0, 5)])
def test_dropout_of_many_elements_off_16_byte_boundaries(dtype, rows, cols, pad, shift):
    rng = np.random.default_rng(cols)
    x = torch.from_numpy(rng.normal(size=(rows, cols))).to(dtype).to(DEV)
    r = torch.from_numpy(rng.normal(size=(rows, cols))).to(dtype).to(DEV)
    check_dropout(strided(x, pad, shift), 0.3, 99, 7)
    a = strided(x, pad, shift)
    check_dropout(strided(x, pad, shift), 0.3, 99, 7, residual=r, out=a)
    assert torch.equal(pb.dropout(strided(x, pad, shift), 0.3, 99, 7, residual=strided(r, 1, shift + 2)), a)
    b = strided(x, pad, shift)
    assert torch.equal(pb.dropout(b, 0.3, 99, 7, residual=r, out=b), a)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("x_shift, out_shift, x_pad, out_pad", [(0, 1, 0, 0), (1, 0, 0, 0), (0, 2, 0, 0), (3, 0, 4, 4), (0, 4, 0, 0), (0, 5, 1, 0), (7, 0, 0, 3), (2, 1, 8, 1)])
def test_gradient_at_another_place_of_16_bytes_than_the_logits(dtype, x_shift, out_shift, x_pad, out_pad):
    """The given token is each of a row's in turn; rows of a warp, of a block, of a cluster and streamed."""
    rng = np.random.default_rng(x_shift * 8 + out_shift)
    for rows, vocab in ((297, 297), (21, 21), (5, 1000), (4, 8000), (3, 17000), (2, 70001)):
        x, tokens, _ = random_rows(rows, vocab, dtype, vocab)
        tokens = np.arange(rows) if rows == vocab else (np.arange(rows) * 7919 + 13) % vocab
        check_grad(strided(x, x_pad, x_shift), tokens, rng.normal(size=rows), rng.normal(size=rows), 1.1, pad=out_pad, shift=out_shift, outputs=True)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows, vocab", [(600, 8211), (300, 33001), (300, 70003)])
def test_gradient_of_many_rows_at_another_pitch(dtype, rows, vocab):
    """Against the same call at the same pitch, which the tests above hold to the oracle: the same bits."""
    x, tokens, rng = random_rows(rows, vocab, dtype, 3)
    tok = torch.from_numpy(np.asarray(tokens, np.int32)).to(DEV)
    g, h = (torch.from_numpy(rng.normal(size=rows).astype(np.float32)).to(DEV) for _ in range(2))
    g[::5] = 0
    h[::5] = 0
    want = pb.token_logprobs_grad(x, tok, g, h)
    for pad, shift in ((1, 0), (3, 5), (8, 1)):
        buf = torch.full((rows * (vocab + pad) + 16,), 5.0, dtype=dtype, device=DEV)
        out = buf[shift:shift + rows * (vocab + pad)].view(rows, vocab + pad)
        pb.token_logprobs_grad(x, tok, g, h, dlogits=out[:, :vocab])
        assert torch.equal(out[:, :vocab], want)
        assert bool((out[:, vocab:] == 5).all()) and bool((buf[:shift] == 5).all()) and bool((buf[shift + rows * (vocab + pad):] == 5).all())


def test_beyond_32_bit_offsets_off_16_byte_boundaries():
    n = (1 << 32) + 4099
    x = torch.ones(n + 3, dtype=torch.bfloat16, device=DEV)
    pb.dropout(x[3:], 0.5, 9, 1, out=x[3:])
    assert bool((x[:3] == 1).all())
    for first in (0, (1 << 31) - 40, (1 << 32) - 40, n - 100):
        field = to.dropout_fields(100, 9, 1, first=first)
        assert np.array_equal(f64(x[3 + first:103 + first]) > 0, field >= 32768)
    del x
    rows, vocab = 33000, 131071
    logits = torch.zeros(rows, vocab + 1, dtype=torch.bfloat16, device=DEV)
    logits[-3:].normal_()
    dlogits = torch.ones(rows, vocab, dtype=torch.bfloat16, device=DEV)
    tokens = torch.full((rows,), vocab - 1, dtype=torch.int32, device=DEV)
    g = torch.zeros(rows, device=DEV)
    g[-3:] = torch.tensor([1.0, -2.0, 0.5])                           # (rows without a gradient are not read)
    pb.token_logprobs_grad(logits[:, :vocab], tokens, g, dlogits=dlogits)
    want = pb.token_logprobs_grad(logits[-3:, :vocab].contiguous(), tokens[-3:], g[-3:])
    assert torch.equal(dlogits[-3:], want) and not bool(dlogits[:-3].any())
    del logits, dlogits
    torch.cuda.empty_cache()
