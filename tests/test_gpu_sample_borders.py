"""Sampling where a border is hard to place: rows whose large logits have low numbers under all three limits, borders at a logit of zero,
logits so large that their distances are coarse.  Against the fp64 oracle; comparisons of sums as near as the whole numbers' roundings reach
(vocab of 2^-45 against sums of at least 1, 2^-47 for the exponentials) are left out."""
import math

import numpy as np
import pytest
import torch

import paper_1707_00424_b200 as pb
from oracle import token_oracle as to

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
TYPES = (torch.float32, torch.bfloat16, torch.float16)


def check(x, u, scale=1.0, most_near=0.02, **limits):
    token, logprob, kept = (t.cpu().numpy() for t in pb.sample_tokens(x, u, scale=scale, **limits))
    host, z, left = x.double().cpu().numpy(), u.cpu().numpy(), 0
    for r in range(len(host)):
        want = to.sample(host[r], z[r], scale, limits.get("top_k", 0), limits.get("top_p", 1.0), limits.get("min_p", 0.0))
        if want[3] <= host.shape[1] * 2.0 ** -45 + 2.0 ** -47:
            left += 1
            continue
        assert (token[r], kept[r]) == (want[0], want[2]), (r, token[r], kept[r], want)
        # the result's rounding; the sum is at least 1 and each weight in it off by 2^-45 (equal ones by the same)
        assert abs(float(logprob[r]) - want[1]) <= U * abs(want[1]) + host.shape[1] * 2.0 ** -45 + 1e-9, (r, logprob[r], want)
    assert left <= most_near * len(host)
    return token, logprob, kept


# ---- top-k, top-p and min-p together: all of top-k's weights count towards top-p's total ---------------------------------------

@pytest.mark.parametrize("dtype", TYPES)
def test_a_list_that_holds_fewer_than_top_k_is_no_basis_for_top_p(dtype):
    """The first logits tell of a bound that min_p reaches, but fewer than top_k logits are from it on."""
    rows, vocab = 160, 131072
    x = torch.full((rows, vocab), -30.0, dtype=dtype, device=DEV)
    x[:, 0], x[:, 1], x[:, 8:488:8], x[:, 20000:21000] = 0.0, -3.5, -7.0, -7.5
    u = (torch.arange(rows, device=DEV) + 0.5) / rows
    _, _, kept = check(x, u, top_k=200, top_p=0.9, min_p=0.02, most_near=0)
    assert (kept == 2).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("top_k, min_p", [(50, 0.05), (200, 0.02), (256, 0.001)])
def test_rows_whose_large_logits_have_low_numbers(dtype, top_k, min_p):
    """As real vocabularies are ordered: frequent tokens first."""
    for rows, vocab in ((160, 131072), (160, 40000), (20, 131072), (400, 20001)):
        g = torch.Generator(device=DEV).manual_seed(rows + vocab)
        x = torch.randn(rows, vocab, generator=g, device=DEV) * 2.5
        x = (x - 1.5 * torch.log1p(torch.arange(vocab, device=DEV) / 100)).to(dtype)
        some = slice(None) if dtype == torch.bfloat16 and vocab > 100000 else slice(0, None, 5)
        u = torch.rand(rows, generator=g, device=DEV)
        got = pb.sample_tokens(x, u, top_k=top_k, top_p=0.9, min_p=min_p)
        host, z = x[some].double().cpu().numpy(), u[some].cpu().numpy()
        for r in range(len(host)):
            # (nothing below the 1024 largest matters to top_k; in their order by number)
            first = np.sort(np.argpartition(-host[r], 1024)[:1024])
            want = to.sample(host[r][first], z[r], 1.0, top_k, 0.9, min_p)
            if want[3] > vocab * 2.0 ** -45 + 2.0 ** -47:
                assert (int(got[0][some][r]), int(got[2][some][r])) == (first[want[0]], want[2]), (rows, vocab, r)


# ---- borders at a logit of zero --------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [256, 257, 4096, 4097, 20001, 131072])
def test_min_p_of_one_keeps_all_zeros(dtype, vocab):
    """More of them than a list holds; a row that is masked altogether counts as zeros, and so does min_p above 1 of a row."""
    x = torch.zeros(5, vocab, dtype=dtype, device=DEV)
    x[1] = torch.finfo(dtype).min
    x[2, ::2] = -1.0
    x[3, ::2] = -0.0
    x[4, vocab // 2:] = -math.inf
    u = (torch.arange(5, device=DEV) + 0.25) / 5
    for _ in range(2):
        check(x, u, min_p=1.0, most_near=1)
        few = torch.tensor([vocab, vocab, vocab // 2, vocab, vocab // 2], device=DEV)
        marked = [torch.full((5,), -7, device=DEV, dtype=t) for t in (torch.int32, torch.float32, torch.int32)]
        token, logprob, kept = pb.sample_tokens(x, u, min_p=torch.full((5,), 2.0, device=DEV), token=marked[0], logprob=marked[1], kept=marked[2])
        assert torch.equal(kept, few.int())
        want = (u.double() * few).floor().long()
        want[2] = 2 * want[2] + 1
        assert torch.equal(token.long(), want)
        assert bool(((logprob.double() + few.double().log()).abs() <= U * few.double().log() + 1e-9).all())
        u = u.flip(0)


def test_zeros_that_are_listed_already_are_kept_once():
    """top_p's border lies just below the zeros that the first pass has listed."""
    rows, vocab = 4, 20000
    x = torch.full((rows, vocab), -20.0, dtype=torch.bfloat16, device=DEV)
    x[:, :1200:8] = 0.0                                     # in the first granules of one or two blocks, one a thread
    x[:, 10000:11200:8] = 0.0
    x[:, 8500:8800], x[:, 18500:18800] = -0.003, -0.004
    u = torch.rand(rows, generator=torch.Generator().manual_seed(3)).to(DEV)
    for k in (1, 40):
        for top_p in (0.2, 0.35, 0.4, 0.52, 0.75, 0.95):
            check(x.repeat(k, 1), u.repeat(k), top_p=top_p, most_near=1)


# ---- logits whose distances are coarse -----------------------------------------------------------------------------------------------

@pytest.mark.parametrize("vocab", [20000, 131072, 300007])
@pytest.mark.parametrize("size, apart, scale", [(1e8, 8, 1.0), (1e8, 8, 0.7), (1e8, 8, 1.2), (5e7, 4, 2.0), (5e7, 8, 0.7), (3e7, 4, 1 / 0.7), (100.0, 2.0 ** -17, 1e6), (-1e8, 8, 1.1), (6e5, 2.0 ** -4, 100.0)])
def test_the_largest_logits_are_one_step_above_all_others(vocab, size, apart, scale):
    """The first logits do not show them; few, so that sums relative to the first logits would stand."""
    for rows in (3, 170) if vocab == 131072 else (3,):
        x = torch.full((rows, vocab), size, device=DEV)
        x[:, -100:-60] += apart
        x[0, vocab - 3000::100] += apart
        u = (torch.arange(rows, device=DEV) + 0.3) / rows
        check(x, u, scale=scale, most_near=1)


# ---- very long rows: whole numbers of less than 2^-44 ----------------------------------------------------------------------------------

def test_weights_of_less_than_half_a_unit_count_nothing():
    """Of 2^23 tokens' weights in units of 2^-39 all but some hundreds are rounded to 0.  Together they would be 7 10^-6 of the sum, enough to move
    top_p's border."""
    vocab = 1 << 23
    x = torch.full((1, vocab), math.log(0.45 * 2.0 ** -39), device=DEV)
    for at in range(0, vocab, 1 << 20):                     # some that the first pass lists, of 4 10^-11 each
        x[0, at + 3:at + 24576:256] = -24.0
    x[0, 5], x[0, 7000000] = 0.0, -14 * math.log(2)
    for top_p, want in ((1 - 6.23e-5, 1), (1 - 5.9e-5, 2)):
        total = (1 + 2.0 ** -14) * float(np.float32(top_p))
        assert abs(total - 1) > 1e-6 and (total > 1) == (want == 2)
        token, _, kept = pb.sample_tokens(x, torch.full((1,), 0.25, device=DEV), top_p=top_p)
        assert (int(token), int(kept)) == (5, want)
