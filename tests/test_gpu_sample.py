"""Sampling of tokens on the GPU against the fp64 oracle: types, sizes, limits alone and together, ties, masks, rows and parameters without
an answer, pitches, streams, graphs; and a model of tokens that is trained and answers.

Tokens and numbers kept are compared exactly, but where a sum of weights lies as near to what it is compared with as the whole numbers'
roundings reach: vocab roundings of 2^-45 against sums of at least 1, and 2^-48 for exponentials on either side."""
import math

import numpy as np
import pytest
import torch

import paper_1707_00424_b200 as pb
from oracle import optimizer_oracle as oo
from oracle import token_oracle as to

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
TYPES = (torch.float32, torch.bfloat16, torch.float16)


def check(x, u, scale=1.0, top_k=0, top_p=1.0, min_p=0.0, most_near=0.02):
    """x [rows, vocab] and u on the GPU; parameters numbers or tensors."""
    rows, vocab = x.shape
    token, logprob, kept = pb.sample_tokens(x, u, scale=scale, top_k=top_k, top_p=top_p, min_p=min_p)
    assert token.dtype == torch.int32 == kept.dtype and logprob.dtype == torch.float32
    host, z = x.double().cpu().numpy(), u.cpu().numpy()
    row = lambda v, r: v[r].item() if isinstance(v, torch.Tensor) else v      # noqa: E731
    left = 0
    for r in range(rows):
        want = to.sample(host[r], z[r], *(row(v, r) for v in (scale, top_k, top_p, min_p)))
        got = int(token[r]), float(logprob[r]), int(kept[r])
        if want[3] <= vocab * 2.0 ** -45 + 2.0 ** -47:
            left += 1
            continue
        assert (got[0], got[2]) == (want[0], want[2]), (r, got, want)
        assert (math.isnan(got[1]) and math.isnan(want[1])) or got[1] == want[1] or abs(got[1] - want[1]) <= U * abs(want[1]) + 1e-9, (r, got, want)
    assert left <= most_near * rows
    return token, logprob, kept


def logits(rows, vocab, dtype, seed, spread=2.5, liked=0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, vocab, generator=g) * spread
    if liked:
        x.scatter_(1, torch.randint(vocab, (rows, liked), generator=g), 8 + 8 * torch.rand(rows, liked, generator=g))
    return x.to(dtype).to(DEV), torch.rand(rows, generator=g).to(DEV)


LIMITS = [dict(), dict(top_k=1), dict(top_k=5), dict(top_k=50), dict(top_p=0.5), dict(top_p=0.95), dict(min_p=0.02), dict(min_p=1.0), dict(top_p=0.0),
          dict(top_k=50, top_p=0.9), dict(top_k=300, top_p=0.99, min_p=0.001), dict(top_p=0.9, min_p=0.1), dict(top_k=1 << 30, top_p=0.999), dict(top_k=700)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("limits", LIMITS, ids=str)
def test_limits_and_sizes(dtype, limits):
    for i, (rows, vocab) in enumerate(((3, 1), (3, 2), (5, 7), (6, 50), (4, 257), (9, 1000), (3, 4096), (3, 4097), (4, 20001), (2, 50021), (2, 131072), (1, 300007))):
        x, u = logits(rows, vocab, dtype, 31 * i, liked=20 if i % 2 else 0)
        check(x, u, scale=(1.0, 1 / 0.7, 0.3)[i % 3], **limits, most_near=1 / rows)


@pytest.mark.parametrize("vocab", [5, 1000, 40000])
def test_ties_go_to_the_lower_token(vocab):
    u = torch.arange(16, device=DEV) / 16
    for dtype in TYPES:
        flat = torch.full((16, vocab), 1.5, dtype=dtype, device=DEV)
        two = flat.clone()
        two[:, ::3] = 3.0
        coarse = (torch.arange(16 * vocab, device=DEV).view(16, vocab) * 7919 % 13).to(dtype)
        for x in (flat, two, coarse):
            for limits in ({}, dict(top_k=3), dict(top_k=vocab // 2 + 1), dict(top_p=0.37), dict(top_p=0.37, top_k=vocab - 2), dict(min_p=0.9), dict(top_k=vocab // 3 + 2, top_p=0.9)):
                check(x, u, **limits, most_near=1)          # (sums of equal weights are whole: the oracle's comparisons are exact, or nearly)
    token, _, kept = pb.sample_tokens(flat, u, top_k=4)
    assert kept.tolist() == [4] * 16 and token.tolist() == [i // 4 for i in range(16)]
    token, _, kept = pb.sample_tokens(flat, u, top_p=0.5)   # half of an even number of equal ones, exactly
    assert kept.tolist() == [(vocab + 1) // 2] * 16


def test_zeros_of_both_signs_are_equal():
    x = torch.tensor([[-0.0, 0.0, -0.0, -1.0]] * 3, device=DEV)
    token, _, kept = pb.sample_tokens(x, torch.tensor([0.0, 0.4, 0.7], device=DEV), top_k=3)
    assert token.tolist() == [0, 1, 2] and kept.tolist() == [3] * 3
    token, _, kept = pb.sample_tokens(x, torch.tensor([0.0, 0.4, 0.7], device=DEV), min_p=1.0)
    assert token.tolist() == [0, 1, 2] and kept.tolist() == [3] * 3


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [40, 5000])
def test_masks(dtype, vocab):
    low = torch.finfo(dtype).min
    x, u = logits(40, vocab, dtype, 5)
    g = torch.Generator().manual_seed(6)
    hide = (torch.rand(40, vocab, generator=g) < 0.6).to(DEV)
    for mask in (-math.inf, low):
        y = x.masked_fill(hide, mask)
        y[0], y[1], y[2, 1:], y[3, :-1] = mask, -math.inf, mask, mask
        for limits in ({}, dict(top_k=vocab - 3), dict(top_k=30, top_p=0.9), dict(top_p=0.99), dict(min_p=0.01)):
            check(y, u, **limits)
    token, logprob, kept = pb.sample_tokens(torch.full((2, vocab), -math.inf, dtype=dtype, device=DEV), u[:2], top_p=0.5, top_k=2)
    assert token.tolist() == [-1] * 2 and logprob.tolist() == [-math.inf] * 2 and kept.tolist() == [0] * 2


def test_rows_without_an_answer_and_their_neighbours():
    for vocab in (30, 9000, 100000):
        x, u = logits(8, vocab, torch.float32, 7)
        x[1, vocab // 2], x[3, -1], x[5, 0], x[6, 3] = math.nan, math.inf, -math.nan, -math.inf
        flags = torch.zeros(1, dtype=torch.int32, device=DEV)
        for limits in ({}, dict(top_k=7), dict(top_p=0.8)):
            token, logprob, kept = check(x, u, **limits)
            assert token[[1, 3, 5]].tolist() == [-1] * 3 and torch.isnan(logprob[[1, 3, 5]]).all() and kept[[1, 3, 5]].tolist() == [0] * 3
        pb.sample_tokens(x, u, flags=flags)
        assert int(flags) == 0


def test_parameters_of_each_row_and_invalid_ones():
    nan = math.nan
    x, _ = logits(14, 3000, torch.bfloat16, 8)
    f = lambda v: torch.tensor(v, device=DEV)              # noqa: E731
    scale = f([1.0, 0.5, 2.0, 0.0, nan, 1.0, 1.0, 1.0, 1.0, 1.0, 1e7, -1.0, 1e-6, 1e6])
    top_k = torch.tensor([0, -5, 3, 1, 1, 10, 10, 10, 2, 2, 2, 2, 0, 0], dtype=torch.int32, device=DEV)
    top_p = f([1.0, 2.0, -1.0, 0.5, 0.5, nan, 0.5, 0.5, 0.3, 1.0, 1.0, 1.0, 0.7, 0.9])
    min_p = f([0.0, -1.0, 0.0, 0.0, 0.0, 0.0, nan, 0.0, 2.0, 0.1, 0.1, 0.1, 0.0, 0.0])
    u = f([0.1, 0.9, 0.5, 0.5, 0.5, 0.5, 0.5, 1.0, 0.99, 0.5, 0.5, 0.5, 0.3, 0.4])
    token, _, _ = check(x, u, scale, top_k, top_p, min_p)
    assert (token == -1).nonzero().flatten().tolist() == [3, 4, 5, 6, 7, 10, 11]
    flags = torch.zeros(1, dtype=torch.int32, device=DEV)
    pb.sample_tokens(x, u, scale=scale, flags=flags)
    assert int(flags) == pb.FLAG_BAD_SAMPLING
    for bad in (-0.1, nan, math.inf, 1.0):
        flags.zero_()
        assert int(pb.sample_tokens(x[0], f(bad), flags=flags)[0]) == -1 and int(flags) == pb.FLAG_BAD_SAMPLING


def test_random_numbers_at_the_ends():
    tiny = [0.0, 2.0 ** -149, 2.0 ** -126, 2.0 ** -60, 2.0 ** -24, 0.5, 1 - 2.0 ** -23, 1 - 2.0 ** -24]
    u = torch.tensor(tiny, device=DEV)
    for vocab in (3, 2000, 70000):
        x, _ = logits(1, vocab, torch.float32, 9)
        for limits in ({}, dict(top_p=0.7), dict(top_k=2)):
            check(x.expand(len(tiny), vocab), u, **limits)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("apart", [0.5, 3.0, 6.0, 10.0, 10.9, 11.1, 14.0, 60.0, 1000.0])
def test_rows_whose_beginning_says_little_about_the_rest(dtype, apart):
    """The first logits are lower, or higher, than all others by some nats: what is guessed from them is wrong."""
    g = torch.Generator().manual_seed(30)
    for vocab in (20000, 131072, 300007):
        x = torch.randn(4, vocab, generator=g) * 0.3
        x[0, vocab // 3:] += apart
        x[1, :vocab // 3] += apart
        x[2, vocab - 5000:] += apart
        x[3, -1] += apart
        x = x.to(dtype).to(DEV)
        u = torch.rand(4, generator=g).to(DEV)
        for limits in ({}, dict(top_k=40), dict(top_p=0.9), dict(min_p=0.3), dict(top_k=200, top_p=0.8, min_p=0.01)):
            check(x, u, **limits, most_near=0.25)


def test_logits_of_any_size_and_extreme_temperatures():
    g = torch.Generator().manual_seed(10)
    u = torch.rand(6, generator=g).to(DEV)
    for size in (1e-30, 1e-5, 1e4, 1e30, 3e38):
        x = (torch.randn(6, 3000, generator=g).clamp(-1, 1) * size).to(DEV)
        for scale in (1e-6, 1.0, 1e6):
            for limits in ({}, dict(top_p=0.6), dict(top_k=100), dict(min_p=0.3)):
                check(x, u, scale=scale, **limits, most_near=1)


@pytest.mark.parametrize("dtype", TYPES)
def test_pitches_and_places(dtype):
    for vocab, pad, shift in ((1001, 3, 1), (1001, 7, 5), (40000, 1, 3), (9, 0, 7)):
        x, u = logits(5, vocab, dtype, 11)
        buf = torch.full((5 * (vocab + pad) + 40,), math.nan, dtype=dtype, device=DEV)
        view = buf[shift:shift + 5 * (vocab + pad)].view(5, vocab + pad)[:, :vocab]
        view.copy_(x)
        for limits in ({}, dict(top_k=20, top_p=0.9), dict(top_p=0.9)):
            a, b = check(view, u, **limits), pb.sample_tokens(x, u, **limits)
            assert all(torch.equal(s, t) for s, t in zip(a, b))
    x, u = logits(6, 500, dtype, 12)
    a = pb.sample_tokens(x.view(2, 3, 500), u.view(2, 3), top_k=9)
    assert a[0].shape == (2, 3) and torch.equal(a[0].flatten(), pb.sample_tokens(x, u, top_k=9)[0])
    one = pb.sample_tokens(x[0], u[0])
    assert one[0].shape == () and int(one[0]) == int(pb.sample_tokens(x, u)[0][0])
    assert pb.sample_tokens(x[:0], u[:0])[0].shape == (0,)


def test_many_rows():
    x, u = logits(3000, 333, torch.bfloat16, 13, liked=5)
    check(x, u, top_k=40, top_p=0.9, most_near=1e-3)
    check(x, u, most_near=1e-3)


def test_past_32_bit_offsets():
    rows, vocab = 9000, 250000                              # 2.25 10^9 bf16 logits
    x = torch.zeros(rows, vocab, dtype=torch.bfloat16, device=DEV)
    at = torch.arange(rows, device=DEV) * 7919 % vocab
    x[torch.arange(rows, device=DEV), at] = 30.0
    token, _, kept = pb.sample_tokens(x, torch.full((rows,), 0.5, device=DEV), min_p=0.5)
    assert torch.equal(token.long(), at) and bool((kept == 1).all())


def test_evenly_spread_numbers_give_each_token_its_share():
    """u = (i + 1/2) / N: a token is sampled N p times to within one."""
    x, _ = logits(1, 900, torch.float32, 14)
    n = 4096
    u = (torch.arange(n, device=DEV) + 0.5) / n
    for limits in ({}, dict(top_k=30), dict(top_p=0.8)):
        token, logprob, kept = pb.sample_tokens(x.expand(n, 900), u, **limits)
        count = torch.bincount(token.long(), minlength=900)
        p = torch.zeros(900, device=DEV).scatter_(0, token.long(), logprob.exp())
        assert bool(((count - n * p).abs() <= 1.001).all()) and bool((token[1:] >= token[:-1]).all())
        assert int((count > 0).sum()) <= int(kept[0])


def test_given_results_streams_and_a_replayed_graph():
    x, u = logits(12, 30000, torch.bfloat16, 15)
    want = pb.sample_tokens(x, u, top_k=50, top_p=0.9)
    out = [torch.empty_like(t) for t in want]
    got = pb.sample_tokens(x, u, top_k=50, top_p=0.9, token=out[0], logprob=out[1], kept=out[2], stream=torch.cuda.Stream())
    torch.cuda.synchronize()
    assert all(a is b and torch.equal(a, c) for a, b, c in zip(got, out, want)) and out[0]._version == 1
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pb.sample_tokens(x, u, top_k=50, top_p=0.9, token=out[0], logprob=out[1], kept=out[2])
    for seed in (16, 17):
        y, v = logits(12, 30000, torch.bfloat16, seed)
        x.copy_(y)
        u.copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, pb.sample_tokens(y, v, top_k=50, top_p=0.9)))


@pytest.mark.parametrize("call", [
    lambda x, u: pb.sample_tokens(x, u, scale=0.0), lambda x, u: pb.sample_tokens(x, u, scale=1e7), lambda x, u: pb.sample_tokens(x, u, scale=math.nan),
    lambda x, u: pb.sample_tokens(x, u, top_k=-1), lambda x, u: pb.sample_tokens(x, u, top_k=1 << 31), lambda x, u: pb.sample_tokens(x, u, top_k=2.5),
    lambda x, u: pb.sample_tokens(x, u, top_p=1.5), lambda x, u: pb.sample_tokens(x, u, top_p=-0.1), lambda x, u: pb.sample_tokens(x, u, min_p=math.nan),
    lambda x, u: pb.sample_tokens(x, u, min_p="low"), lambda x, u: pb.sample_tokens(x, u[:3]), lambda x, u: pb.sample_tokens(x, u.double()), lambda x, u: pb.sample_tokens(x, None),
    lambda x, u: pb.sample_tokens(x, u.cpu()), lambda x, u: pb.sample_tokens(x, u, top_k=u), lambda x, u: pb.sample_tokens(x, u, scale=u.double()),
    lambda x, u: pb.sample_tokens(x, u, top_p=u[:2]), lambda x, u: pb.sample_tokens(x.t(), u), lambda x, u: pb.sample_tokens(x.double(), u),
    lambda x, u: pb.sample_tokens(x, u, token=torch.zeros(4, device=DEV)), lambda x, u: pb.sample_tokens(x[:, :0], u), lambda x, u: pb.sample_tokens(x, u, flags=u),
])
def test_refused_arguments(call):
    x, u = torch.zeros(4, 8, device=DEV), torch.zeros(4, device=DEV)
    with pytest.raises(pb.ParleError) as e:
        call(x, u)
    assert e.value.code == -1


@pytest.mark.parametrize("bits", [32, 8])
def test_a_model_of_tokens_takes_a_step_and_answers(bits):
    """Lookup, log probabilities' gradient, the table's gradient, its norm, AdamW with a bf16 copy, and tokens sampled from that one:
    each against the oracle, on the values that the call before it left."""
    rng = np.random.default_rng(18)
    vocab, length = 60, 200
    table = torch.from_numpy(rng.normal(size=(vocab, vocab)).astype(np.float32)).to(DEV)
    served = table.bfloat16()
    state = pb.adamw_state([table], bits)
    prev, following = (torch.from_numpy(rng.integers(0, vocab, length).astype(np.int32)).to(DEV) for _ in range(2))
    for t in range(1, 4):
        before, scores = table.double().cpu().numpy(), pb.embedding(served, prev, dtype=torch.float32)
        assert torch.equal(scores, served[prev.long()].float())
        d = pb.token_logprobs_grad(scores, following, torch.full((length,), -1.0 / length, device=DEV))
        grad = pb.embedding_grad(d, prev, vocab)
        s = scores.double().cpu().numpy()
        wd = to.token_logprobs_grad(s, following.cpu().numpy(), np.full(length, -1.0 / length), None)
        wg, _, _ = to.embedding_grad(wd[None], prev.cpu().numpy()[None], vocab, 1.0)
        assert np.abs(grad.double().cpu().numpy() - wg[0]).max() < 1e-5
        norm = pb.grad_norm([grad])
        g = grad.double().cpu().numpy()
        assert abs(float(norm) - oo.grad_norm([g])) < 1e-5 * float(norm)
        def moment(k):
            x = state[k][0].double().cpu().numpy().reshape(-1)
            x = x if bits == 32 else x * np.repeat(state[k + 2][0].double().cpu().numpy(), 256)[:len(x)]
            return (x if bits == 32 or k == 0 else x ** 2).reshape(vocab, vocab)
        m0, v0 = moment(0), moment(1)
        pb.adamw([table], [grad], state[0], state[1], step=t, lr=0.02, exp_avg_scales=state[2], exp_avg_sq_scales=state[3], copies=[served], norm=norm, max_norm=0.05)
        c = oo.coefficient(1.0, float(norm), 0.05)
        want = oo.param(before, *oo.moments(c * g, m0, v0, 0.9, 0.999), t, 0.02, 0.9, 0.999, 1e-8, 0.01)
        # the ratio of the moments is below 10; each of a dozen roundings, the root and the reciprocal move it by less than 2^-20
        assert np.abs(table.double().cpu().numpy() - want).max() < 0.02 * 10 * 2.0 ** -20 + 4 * 3 * U + 1e-7
        assert torch.equal(served, table.bfloat16())
        u = torch.from_numpy(rng.random(length).astype(np.float32)).to(DEV)
        answers = pb.embedding(served, prev, dtype=torch.bfloat16)
        token, logprob, kept = check(answers, u, scale=1 / 0.8, top_k=20, top_p=0.9)
        full, _, _, _ = pb.token_logprobs(answers, token, scale=1 / 0.8)
        assert bool((logprob >= full - 1e-5).all()) and bool((kept <= 20).all())
        prev = token


def test_calls_from_several_threads_and_streams():
    import threading
    x, u = logits(40, 60000, torch.bfloat16, 33)
    y, v = logits(500, 300, torch.float16, 34)
    limits = [{}, dict(top_k=30), dict(top_p=0.9), dict(min_p=0.01), dict(top_k=5000, top_p=0.95)]
    want = [[pb.sample_tokens(a, b, **k) for k in limits] for a, b in ((x, u), (y, v))]
    torch.cuda.synchronize()
    wrong = []

    def work():
        s = torch.cuda.Stream()
        for _ in range(10):
            got = [[pb.sample_tokens(a, b, **k, stream=s) for k in limits] for a, b in ((x, u), (y, v))]
        s.synchronize()
        if not all(torch.equal(p, q) for a, b in zip(got, want) for c, d in zip(a, b) for p, q in zip(c, d)):
            wrong.append(1)

    threads = [threading.Thread(target=work) for _ in range(4)]
    for th in threads:
        th.start()
    for th in threads:
        th.join()
    assert not wrong


def test_short_and_long_rows_around_the_borders_between_kernels():
    """Around 4096 tokens (blocks of 128 or 512 threads), lists' lengths and blocks' parts."""
    for rows, vocab in ((3, 255), (3, 256), (3, 257), (2, 1023), (2, 1025), (2, 4095), (2, 4096), (2, 4097), (2, 16383), (1, 16384), (2, 32767), (3, 32768), (2, 131071)):
        for dtype in TYPES:
            x, u = logits(rows, vocab, dtype, vocab, spread=1.0)
            for k in (dict(top_k=64), dict(top_k=65), dict(top_k=256), dict(top_k=257), dict(top_k=vocab - 1), dict(top_k=vocab), dict(top_p=0.97), dict(min_p=0.05), dict(top_k=vocab // 2, top_p=0.5, min_p=0.2)):
                check(x, u, **k, most_near=1 / rows)
