"""Equal logits among the alternatives: the lower token first, wherever the equal ones lie against each other and against 16 bytes.

Whole-number logits, exact in every type, so that (logit, -token) is one integer key and the alternatives are its largest: the tokens
have to be equal."""
import pytest
import torch

import paper_1707_00424_b200 as pb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = (torch.float32, torch.bfloat16, torch.float16)


def ranked(whole):
    """Tokens by falling logit, equal ones by token: whole int64 [rows, vocab]."""
    key = whole * 4096 - torch.arange(whole.shape[1], device=DEV)
    return key.argsort(dim=1, descending=True).int()


def placed(whole, dtype, pad, shift):
    """The logits in rows of pitch vocab + pad that begin `shift` elements behind a 16-byte boundary, amid large numbers."""
    rows, vocab = whole.shape
    buf = torch.full((rows * (vocab + pad) + shift + 16,), 1000.0, dtype=dtype, device=DEV)
    view = buf[shift:shift + rows * (vocab + pad)].view(rows, vocab + pad)[:, :vocab]
    view.copy_(whole)
    return view


def wrong(x, k, want):
    got = pb.token_logprobs(x, k=k)[2]
    here = min(k, x.shape[1])                             # (no alternatives behind the last token)
    return (got[:, :here] != want[:, :here]).any(dim=1) | (got[:, here:] != pb.NO_TOKEN).any(dim=1)


def pairs(vocab, near):
    """A row for each pair of tokens at most `near` apart."""
    i, j = torch.triu_indices(vocab, vocab, 1, device=DEV)
    some = j - i <= near
    return i[some], j[some]


def test_the_smallest_rows():
    for dtype, vocab in ((torch.float32, 4), (torch.bfloat16, 8), (torch.float16, 8)):
        row = torch.zeros(1, vocab, device=DEV, dtype=dtype)
        row[0, 1:3] = 5
        assert pb.token_logprobs(row, k=1)[2].tolist() == [[1]]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab, k", [(v, k) for v in (2, 3, 4, 5, 7, 8, 9, 12, 15, 16, 17, 24, 33) for k in (1, 2, 3)] +
                         [(50, 6), (64, 12), (100, 20), (150, 20), (150, 32), (300, 32), (500, 25), (500, 32), (1000, 32), (2000, 32)])
def test_two_equal_logits_at_the_last_rank(dtype, vocab, k):
    """k - 1 larger logits, spread over the row, and two equal ones, of which the lower token has the last place."""
    i, j = pairs(vocab, 16 if vocab <= 200 else 9)
    if vocab > 200:                                       # enough rows for one warp each
        i, j = i[:6000], j[:6000]
    r = torch.arange(len(i), device=DEV)
    for turn in (1, 7):
        whole = torch.zeros(len(i), vocab, dtype=torch.int64, device=DEV)
        at = (torch.arange(k - 1, device=DEV) * vocab // max(1, k - 1))[None, :].expand(len(i), -1)
        at = (at + r[:, None] * turn) % vocab             # (some fall on the pair, and leave fewer before it)
        whole.scatter_(1, at, torch.arange(20, 20 + k - 1, device=DEV).expand(len(i), -1))
        whole[r, i] = 5
        whole[r, j] = 5
        want = ranked(whole)
        for shift in range(16 // dtype.itemsize):
            for pad in (0, shift + 1):
                bad = wrong(placed(whole, dtype, pad, shift), k, want)
                assert not bool(bad.any()), (shift, pad, int(bad.sum()), whole[bad][0].tolist())


@pytest.mark.parametrize("dtype", TYPES)
def test_whole_numbers_over_all_short_vocabularies(dtype):
    gen = torch.Generator(device=DEV).manual_seed(1)
    bad = []
    for vocab in range(1, 65):
        whole = torch.randn(1000, vocab, device=DEV, generator=gen).round().long()
        want = ranked(whole)
        for shift in range(16 // dtype.itemsize):
            x = placed(whole, dtype, shift % 3, shift)
            for k in range(1, min(vocab, 32) + 1):
                bad.append(wrong(x, k, want).sum())
    assert int(torch.stack(bad).sum()) == 0


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows, vocab, k", [(4000, 50, 6), (4000, 100, 19), (4000, 150, 20), (2000, 387, 32), (1500, 500, 32), (1300, 1000, 30), (1300, 2032, 32),
                                            (700, 500, 12), (300, 1900, 20), (64, 3000, 32), (5, 9001, 8), (300, 9001, 8), (2, 4095, 32)])
def test_whole_numbers_of_more_classes(dtype, rows, vocab, k):
    gen = torch.Generator(device=DEV).manual_seed(vocab)
    for spread in (1.0, 3.0, 20.0):
        whole = (torch.randn(rows, vocab, device=DEV, generator=gen) * spread).round().long()
        want = torch.empty(rows, k, dtype=torch.int32, device=DEV)
        key = whole * 16384 - torch.arange(vocab, device=DEV)
        want.copy_(key.topk(k, dim=1).indices)
        for shift, pad in ((0, 0), (1, 3)):
            assert int(wrong(placed(whole, dtype, pad, shift), k, want).sum()) == 0


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab, k", [(8, 1), (16, 2), (50, 6)])
def test_logits_whose_ties_arise_by_rounding(dtype, vocab, k):
    gen = torch.Generator(device=DEV).manual_seed(2)
    x = torch.randn(20000, vocab, device=DEV, generator=gen).to(dtype)
    # 16-bit numbers as whole ones: ordered by their bits
    value = x.double()
    rank = torch.unique(value, return_inverse=True)[1]
    key = rank * 64 - torch.arange(vocab, device=DEV)
    assert int(wrong(x, k, key.argsort(dim=1, descending=True).int()).sum()) == 0
