"""Calls of the token operators' functions: which strided tensors they take, what they refuse, calls from several threads."""
import itertools
import threading

import pytest
import torch

import paper_1707_00424_b200 as pb

pytestmark = pytest.mark.gpu
EINVAL, ETOOBIG = -1, -8


def viewable(t):
    """Whether t is rows of one pitch with a dense last dimension, by torch's own rules."""
    try:
        v = t.view(-1 if t.numel() else 0, t.shape[-1])
    except RuntimeError:
        return False
    return t.shape[-1] <= 1 or v.stride(1) == 1


def strided():
    """Tensors of one to four dimensions with steps, broadcasts, swapped and single dimensions."""
    base = torch.arange(4096, device="cuda:0", dtype=torch.float32)
    for shape in ((7,), (1,), (3, 5), (1, 5), (5, 1), (2, 3, 4), (2, 1, 4), (1, 3, 4), (3, 2, 1), (2, 3, 1, 4), (1, 1, 1, 1), (2, 2, 2, 2)):
        for steps in itertools.product((0, 1, 4, 5, 8, 12, 24), repeat=len(shape) - 1):
            yield base.as_strided(shape, (*steps, 1))
        yield base.as_strided(shape, (*(1 for _ in shape[1:]), 2))


def test_strided_tensors_are_taken_or_refused_as_views_are():
    taken = refused = 0
    for x in strided():
        if viewable(x):
            assert torch.equal(pb.dropout(x, 0.0, 1), x), (x.shape, x.stride())
            taken += 1
        else:
            with pytest.raises(pb.ParleError) as e:
                pb.dropout(x, 0.0, 1)
            assert e.value.code == EINVAL
            refused += 1
    assert taken > 100 and refused > 100


def test_strided_tables_of_replicas():
    g = torch.Generator().manual_seed(1)
    base = torch.randn(3, 2, 11, 16, generator=g).cuda()
    tokens = torch.randint(0, 11, (3, 4, 5), generator=g, dtype=torch.int32).cuda()
    for table in (base[:, 1], base[:, 0, :, :7], base[::2, 1, :, 8:], base[1:2, 1]):
        n = table.shape[0]
        out = torch.full((n, 4, 5, table.shape[2] + 3), 9.0, device="cuda:0")
        want = torch.stack([table[i][tokens[i].long()] for i in range(n)])
        assert torch.equal(pb.embedding(table, tokens[:n]), want)
        pb.embedding(table, tokens[:n], out=out[..., :-3])
        assert torch.equal(out[..., :-3], want) and bool((out[..., -3:] == 9).all())
    with pytest.raises(pb.ParleError):
        pb.embedding(base[:, :, ::2].flatten(0, 1)[:3].transpose(0, 1).contiguous().transpose(0, 1).transpose(1, 2), tokens)


@pytest.mark.parametrize("call", [
    lambda x, t: pb.token_logprobs(x, t, k=-1), lambda x, t: pb.token_logprobs(x, t, k=33), lambda x, t: pb.token_logprobs(x, t, k=1 << 70),
    lambda x, t: pb.token_logprobs(x, t, k=1.5), lambda x, t: pb.token_logprobs(x, t.long()), lambda x, t: pb.token_logprobs(x, t.cpu()),
    lambda x, t: pb.token_logprobs(x, [1, 2]), lambda x, t: pb.token_logprobs(None, t), lambda x, t: pb.token_logprobs(x.double(), t),
    lambda x, t: pb.token_logprobs(x, t, scale="warm"), lambda x, t: pb.token_logprobs(x, logprob=torch.zeros(4, device="cuda:0")),
    lambda x, t: pb.token_logprobs(x[0, 0], t), lambda x, t: pb.token_logprobs(x.t(), t), lambda x, t: pb.token_logprobs(x, t, flags=t),
    lambda x, t: pb.token_logprobs(x, t, entropy=torch.zeros(4)), lambda x, t: pb.token_logprobs_grad(x, t, x[:, 0]),
    lambda x, t: pb.token_logprobs_grad(x, t, torch.zeros(4, device="cuda:0"), dlogits=x.half()),
    lambda x, t: pb.token_logprobs_grad(x, t, torch.zeros(4, device="cuda:0"), dlogits=x[:3]),
    lambda x, t: pb.embedding(x[0], t), lambda x, t: pb.embedding(x, t, dtype=torch.float64), lambda x, t: pb.embedding(x, t, dtype="float32"),
    lambda x, t: pb.embedding(x, t, out=torch.zeros(4, 7, device="cuda:0")), lambda x, t: pb.embedding(x[None], t),
    lambda x, t: pb.embedding(x, t, out=torch.zeros(4, 8, device="cuda:0"), dtype=torch.float16),
    lambda x, t: pb.embedding_grad(x, t, 0), lambda x, t: pb.embedding_grad(x, t, 1 << 40), lambda x, t: pb.embedding_grad(x, t, 5, accumulate=True),
    lambda x, t: pb.embedding_grad(x, t, 5, n=1), lambda x, t: pb.embedding_grad(x, t, 5, n=-1),
    lambda x, t: pb.embedding_grad(x, t[:3], 5), lambda x, t: pb.embedding_grad(x, t, 5, dtable=torch.zeros(5, 8, device="cuda:0").bfloat16()),
    lambda x, t: pb.embedding_grad(x, t, 5, dtable=torch.zeros(5, 9, device="cuda:0")),
    lambda x, t: pb.embedding_grad(x, t, 5, n=2, dtable=torch.zeros(5, 8, device="cuda:0")),
    lambda x, t: pb.embedding_grad(x, t, 5, workspace=torch.zeros(64)), lambda x, t: pb.dropout(x, 0.5, -1), lambda x, t: pb.dropout(x, 0.5, 1 << 64),
    lambda x, t: pb.dropout(x, 0.5, 1, 2.5), lambda x, t: pb.dropout(x, 1.5, 1), lambda x, t: pb.dropout(x, "half", 1),
    lambda x, t: pb.dropout(x, 0.5, 1, residual=x[:, :7]), lambda x, t: pb.dropout(x, 0.5, 1, out=x.half()),
    lambda x, t: pb.dropout(x, 0.5, 1, offset_dev=t[:1]), lambda x, t: pb.dropout(x, 0.5, 1, offset_dev=torch.zeros(1, dtype=torch.int64)),
])
def test_refused_arguments(call):
    x, t = torch.zeros(4, 8, device="cuda:0"), torch.zeros(4, dtype=torch.int32, device="cuda:0")
    with pytest.raises(pb.ParleError) as e:
        call(x, t)
    assert e.value.code == EINVAL


def test_one_position_for_each_of_several_tables():
    x, t = torch.randn(4, 8, device="cuda:0"), torch.arange(4, dtype=torch.int32, device="cuda:0")
    want = torch.zeros(4, 5, 8, device="cuda:0")
    want[torch.arange(4), torch.arange(4)] = x
    assert torch.equal(pb.embedding_grad(x, t, 5, n=4), want)


def test_a_vocabulary_beyond_32_bits_is_refused():
    x = torch.empty((1 << 32) + 8, device="cuda:0", dtype=torch.float16)          # as 32 bits: 8
    for call in (lambda: pb.token_logprobs(x[None]), lambda: pb.embedding(x[:, None], torch.zeros(1, dtype=torch.int32, device="cuda:0"))):
        with pytest.raises(pb.ParleError) as e:
            call()
        assert e.value.code == ETOOBIG


def test_arguments_by_name_and_position_and_the_results_given():
    x, t = torch.randn(4, 8, device="cuda:0"), torch.arange(4, dtype=torch.int32, device="cuda:0")
    a = pb.token_logprobs(x, t, 2, 0.5)
    out = [torch.empty_like(v) for v in a]
    b = pb.token_logprobs(logits=x, tokens=t, k=2, scale=0.5, logprob=out[0], entropy=out[1], top_token=out[2], top_logprob=out[3])
    assert all(v is w for v, w in zip(b, out)) and all(torch.equal(v, w) for v, w in zip(a, b))
    none, entropy, top_token, top_logprob = pb.token_logprobs(x)
    assert none is None and entropy.shape == (4,) and top_token.shape == (4, 0) == top_logprob.shape
    table = torch.zeros(8, 8, device="cuda:0")
    assert pb.embedding_grad(x, t, 8, dtable=table, accumulate=True) is table
    assert pb.embedding(x, t, dtype=torch.bfloat16).dtype is torch.bfloat16


def test_calls_from_several_threads():
    """Each thread on a stream of its own; each result is the one of a call alone."""
    g = torch.Generator().manual_seed(2)
    x, t = torch.randn(64, 1001, generator=g).cuda(), torch.randint(0, 1001, (64,), generator=g, dtype=torch.int32).cuda()
    want = [pb.token_logprobs(x, t, k=3), pb.embedding_grad(x, t, 1001), pb.dropout(x, 0.3, 5)]
    torch.cuda.synchronize()
    wrong = []

    def work():
        s = torch.cuda.Stream()
        for _ in range(50):
            got = [pb.token_logprobs(x, t, k=3, stream=s), pb.embedding_grad(x, t, 1001, stream=s), pb.dropout(x, 0.3, 5, stream=s)]
        s.synchronize()
        if not (all(torch.equal(a, b) for a, b in zip(got[0], want[0])) and torch.equal(got[1], want[1]) and torch.equal(got[2], want[2])):
            wrong.append(threading.get_ident())

    threads = [threading.Thread(target=work) for _ in range(4)]
    for th in threads:
        th.start()
    for th in threads:
        th.join()
    assert not wrong
