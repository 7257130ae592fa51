"""What the token operators refuse, on the CPU: every call here returns before it touches the device."""
import ctypes as C
import math

import pytest
import torch

import paper_1707_00424_b200 as pb

EINVAL, EALIGN, EWORKSPACE, ETOOBIG = -1, -3, -6, -8
P = 1 << 20                                               # an aligned address that is never read
F32, BF16, F16 = 0, 1, 2


def logprobs(logits=P, dtype=F32, rows=2, vocab=8, ld=8, tokens=P, scale=1.0, k=0, logprob=P, entropy=None, top_token=None,
             top_logprob=None, flags=None):
    return pb.lib().parle_token_logprobs(logits, dtype, rows, vocab, ld, tokens, scale, k, logprob, entropy, top_token, top_logprob, flags, None)


def logprobs_grad(logits=P, dtype=F32, rows=2, vocab=8, ld=8, tokens=P, scale=1.0, d_logprob=P, d_entropy=None, logprob=None,
                  entropy=None, dlogits=2 * P, ld_d=8, flags=None):
    return pb.lib().parle_token_logprobs_grad(logits, dtype, rows, vocab, ld, tokens, scale, d_logprob, d_entropy, logprob, entropy, dlogits,
                                              ld_d, flags, None)


def embedding(table=P, table_dtype=F32, table_gs=32, ld_table=4, n=2, vocab=8, dim=4, tokens=P, length=5, scale=1.0, out=2 * P,
              out_dtype=F32, out_gs=20, ld_out=4, flags=None):
    return pb.lib().parle_embedding(table, table_dtype, table_gs, ld_table, n, vocab, dim, tokens, length, scale, out, out_dtype, out_gs,
                                    ld_out, flags, None)


def embedding_grad(dout=P, dtype=F32, dout_gs=20, ld_dout=4, tokens=P, n=2, length=5, vocab=8, dim=4, scale=1.0, dtable=2 * P,
                   dtable_gs=32, ld_dtable=4, accumulate=0, workspace=3 * P, nbytes=1 << 20, flags=None):
    return pb.lib().parle_embedding_grad(dout, dtype, dout_gs, ld_dout, tokens, n, length, vocab, dim, scale, dtable, dtable_gs, ld_dtable,
                                         accumulate, workspace, nbytes, flags, None)


def dropout(x=P, ld_x=8, residual=None, ld_r=0, y=2 * P, ld_y=8, dtype=F32, rows=2, cols=8, p=0.5, seed=1, offset=0, offset_dev=None):
    return pb.lib().parle_dropout(x, ld_x, residual, ld_r, y, ld_y, dtype, rows, cols, p, seed, offset, offset_dev, None)


@pytest.mark.parametrize("call, kw, code", [
    (logprobs, dict(logits=None), EINVAL), (logprobs, dict(dtype=3), EINVAL), (logprobs, dict(rows=-1), EINVAL),
    (logprobs, dict(vocab=0), EINVAL), (logprobs, dict(ld=-1), EINVAL), (logprobs, dict(scale=0.0), EINVAL),
    (logprobs, dict(scale=-1.0), EINVAL), (logprobs, dict(scale=math.nan), EINVAL), (logprobs, dict(scale=math.inf), EINVAL),
    (logprobs, dict(scale=3e38), EINVAL), (logprobs, dict(scale=1e-60), EINVAL), (logprobs, dict(scale=9e-7), EINVAL), (logprobs, dict(scale=1.1e6), EINVAL), (logprobs, dict(tokens=None), EINVAL),
    (logprobs, dict(k=33, top_token=P), EINVAL), (logprobs, dict(k=-1), EINVAL), (logprobs, dict(k=0, top_token=P), EINVAL),
    (logprobs, dict(logprob=None), EINVAL), (logprobs, dict(rows=1 << 31), ETOOBIG), (logprobs, dict(vocab=(1 << 30) + 1), ETOOBIG),
    (logprobs, dict(logits=P + 2), EALIGN), (logprobs, dict(logits=P + 1, dtype=BF16), EALIGN), (logprobs, dict(tokens=P + 2), EALIGN),
    (logprobs, dict(logprob=P + 2), EALIGN), (logprobs, dict(entropy=P + 1), EALIGN), (logprobs, dict(flags=P + 2), EALIGN),
    (logprobs_grad, dict(d_logprob=None), EINVAL), (logprobs_grad, dict(tokens=None), EINVAL), (logprobs_grad, dict(dlogits=None), EINVAL),
    (logprobs_grad, dict(d_logprob=None, d_entropy=P, tokens=None, logprob=P), EINVAL), (logprobs_grad, dict(ld_d=7), EINVAL),
    (logprobs_grad, dict(dlogits=P, ld_d=9), EINVAL), (logprobs_grad, dict(scale=-2.0), EINVAL), (logprobs_grad, dict(dlogits=P + 2), EALIGN),
    (logprobs_grad, dict(d_logprob=P + 2), EALIGN), (logprobs_grad, dict(d_entropy=P + 2), EALIGN),
    (embedding, dict(n=0), EINVAL), (embedding, dict(n=65), EINVAL), (embedding, dict(vocab=0), EINVAL), (embedding, dict(dim=0), EINVAL),
    (embedding, dict(length=-1), EINVAL), (embedding, dict(table=None), EINVAL), (embedding, dict(tokens=None), EINVAL),
    (embedding, dict(out=None), EINVAL), (embedding, dict(table_dtype=5), EINVAL), (embedding, dict(out_dtype=-1), EINVAL),
    (embedding, dict(scale=math.inf), EINVAL), (embedding, dict(scale=1e39), EINVAL), (embedding, dict(ld_table=-4), EINVAL),
    (embedding, dict(table_gs=-32), EINVAL), (embedding, dict(ld_out=3), EINVAL), (embedding, dict(out_gs=19), EINVAL),
    (embedding, dict(out_gs=0), EINVAL), (embedding, dict(out_gs=4, ld_out=7), EINVAL),
    (embedding, dict(length=1 << 30), ETOOBIG), (embedding, dict(vocab=(1 << 30) + 1), ETOOBIG), (embedding, dict(dim=(1 << 24) + 1), ETOOBIG),
    (embedding, dict(table=P + 2), EALIGN), (embedding, dict(out=P + 1, out_dtype=F16), EALIGN),
    (embedding, dict(tokens=P + 2), EALIGN), (embedding, dict(flags=P + 3), EALIGN),
    (embedding_grad, dict(dout=None), EINVAL), (embedding_grad, dict(dtable=None), EINVAL), (embedding_grad, dict(workspace=None, length=20000, dout_gs=80000), EINVAL),
    (embedding_grad, dict(dtype=3), EINVAL), (embedding_grad, dict(scale=math.nan), EINVAL), (embedding_grad, dict(ld_dout=-1), EINVAL),
    (embedding_grad, dict(dtable_gs=31), EINVAL), (embedding_grad, dict(ld_dtable=3), EINVAL), (embedding_grad, dict(nbytes=64, length=20000), EWORKSPACE),
    (embedding_grad, dict(length=1 << 30), ETOOBIG), (embedding_grad, dict(vocab=(1 << 30) + 1), ETOOBIG),
    (embedding_grad, dict(dim=(1 << 24) + 1), ETOOBIG), (embedding_grad, dict(workspace=3 * P + 64), EALIGN),
    (embedding_grad, dict(dout=P + 2), EALIGN), (embedding_grad, dict(dtable=P + 2), EALIGN),
    (dropout, dict(x=None), EINVAL), (dropout, dict(y=None), EINVAL), (dropout, dict(p=-0.1), EINVAL), (dropout, dict(p=1.1), EINVAL),
    (dropout, dict(p=math.nan), EINVAL), (dropout, dict(dtype=9), EINVAL), (dropout, dict(rows=-1), EINVAL), (dropout, dict(ld_y=7), EINVAL),
    (dropout, dict(ld_x=-8), EINVAL), (dropout, dict(y=P, ld_y=9), EINVAL), (dropout, dict(residual=2 * P, ld_r=9), EINVAL),
    (dropout, dict(rows=1 << 40, cols=2, ld_x=2, ld_y=2), ETOOBIG), (dropout, dict(x=P + 2), EALIGN), (dropout, dict(offset_dev=P + 4), EALIGN),
])
def test_the_c_entry_points_refuse(call, kw, code):
    assert call(**kw) == code


def test_nothing_to_do_is_no_error():
    assert logprobs(rows=0) == 0 and logprobs_grad(rows=0) == 0 and embedding(length=0, out_gs=4) == 0
    assert dropout(rows=0) == 0 and dropout(cols=0) == 0


def test_workspace_sizes():
    size = pb.embedding_grad_workspace_bytes
    assert size(1, 0, 10, 4) == 0 and size(0, 5, 10, 4) == 0 and size(1, -1, 10, 4) == 0 and size(1, 5, 0, 4) == 0
    assert size(2, 1 << 30, 10, 4) == 0
    assert size(1, 1, 1000, 64) == 0 and size(64, 1024, 1000, 64) == 0           # up to this length the gradient needs none
    for n, length in ((1, 1025), (4, 100000)):
        assert size(n, length, 1000, 64) >= n * length * 8 and size(n, length, 1000, 64) % 128 == 0



def test_the_functions_refuse_tensors_that_are_not_on_a_gpu():
    x, t = torch.zeros(2, 8), torch.zeros(2, dtype=torch.int32)
    for call in (lambda: pb.token_logprobs(x, t), lambda: pb.token_logprobs_grad(x, t, torch.zeros(2)), lambda: pb.embedding(x, t),
                 lambda: pb.embedding_grad(x, t, 5), lambda: pb.dropout(x, 0.5, 1)):
        with pytest.raises(pb.ParleError) as e:
            call()
        assert e.value.code == EINVAL and "CUDA device" in str(e.value)


def test_constants_match_the_header():
    assert pb.NO_TOKEN == -1 and pb.TOP_MAX == 32
    assert C.sizeof(C.c_size_t) == 8
