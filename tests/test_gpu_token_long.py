"""The tables' gradient of long sequences: tiles of the sort whose counts every block adds up, and more of them, whose counts are scanned.

Whole numbers whose sums stay below 2^24: fp32 sums in any order are exact, so the results have to be equal."""
import pytest
import torch

import paper_1707_00424_b200 as pb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TILE = 4096                                               # positions of a block of the sort


def case(n, length, vocab, dim, dtype, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    tokens = torch.randint(-1, vocab, (n, length), generator=gen, device=DEV, dtype=torch.int32)
    dout = torch.randint(-8, 9, (n, length, dim), generator=gen, device=DEV).to(dtype)
    return tokens, dout


def sums(tokens, dout, vocab):
    n, length, dim = dout.shape
    out = torch.zeros(n, vocab + 1, dim, dtype=torch.int64, device=DEV)          # row `vocab` takes the positions without a token
    for g in range(n):
        at = torch.where(tokens[g] >= 0, tokens[g], vocab).long()
        out[g].index_add_(0, at, dout[g].long())
    assert int(out.abs().max()) < 1 << 24
    return out[:, :vocab]


@pytest.mark.parametrize("n, length, vocab, dim, dtype", [
    (1, 64 * TILE, 300, 3, torch.float32), (1, 64 * TILE + 1, 300, 3, torch.bfloat16), (1, 65 * TILE, 300, 8, torch.float16),
    (3, 66 * TILE - 1, 70000, 2, torch.bfloat16), (2, 97 * TILE + 17, 7, 9, torch.float32), (1, 300001, 20000000, 1, torch.float32),
    (1, (1 << 22) + 5, 5000, 1, torch.bfloat16), (1, 1 << 23, 100000, 4, torch.float16), (5, 128 * TILE + 4095, 1, 1, torch.bfloat16),
])
def test_sums_of_many_positions(n, length, vocab, dim, dtype):
    tokens, dout = case(n, length, vocab, dim, dtype, length % 1000)
    want = sums(tokens, dout, vocab)
    got = pb.embedding_grad(dout, tokens, vocab, n=n)
    assert torch.equal(got.long(), want)
    more = torch.full_like(got, 3.0)
    pb.embedding_grad(dout, tokens, vocab, dtable=more, accumulate=True)
    assert torch.equal(more.long(), want + 3)


@pytest.mark.parametrize("order", ["ascending", "descending", "one token", "two far tokens"])
def test_sums_of_many_positions_in_order(order):
    length, vocab = 200 * TILE + 77, 1 << 17
    _, dout = case(1, length, vocab, 2, torch.bfloat16, 5)
    at = torch.arange(length, device=DEV)
    tokens = {"ascending": at * vocab // length, "descending": vocab - 1 - at * vocab // length, "one token": torch.full_like(at, vocab - 1),
              "two far tokens": torch.where(at % 3 == 0, vocab - 1, 0)}[order][None].int()
    assert torch.equal(pb.embedding_grad(dout, tokens, vocab, n=1).long(), sums(tokens, dout, vocab))


def test_the_time_of_long_sequences_grows_with_their_length():
    """Eight times the positions take eight times as long; were every tile's counts read for every tile, some twenty-five times."""
    def time(length):
        tokens, dout = case(1, length, 1000, 1, torch.bfloat16, 1)
        out = torch.empty(1000, 1, device=DEV)
        scratch = torch.empty(pb.embedding_grad_workspace_bytes(1, length, 1000, 1), dtype=torch.uint8, device=DEV)
        each = []
        for _ in range(5):
            a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            a.record()
            pb.embedding_grad(dout[0], tokens[0], 1000, dtable=out, workspace=scratch)
            b.record()
            b.synchronize()
            each.append(a.elapsed_time(b))
        return min(each)
    assert time(1 << 26) < 16 * time(1 << 23)
