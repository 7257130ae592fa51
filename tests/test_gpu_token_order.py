"""The order of the table gradient's sums is a matter of the tokens alone: a column has the same bits whatever columns stand beside it."""
import pytest
import torch

import paper_1707_00424_b200 as pb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16, torch.float16))
@pytest.mark.parametrize("n, length", [(1, 17), (1, 200), (3, 640), (1, 1024), (1, 1025), (2, 6000), (1, 40000)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_columns_have_the_same_bits_in_wider_and_narrower_rows(dtype, n, length, accumulate):
    gen = torch.Generator(device=DEV).manual_seed(length)
    vocab, dim = 30, 600                                  # tokens more and less frequent than a row's noted positions
    tokens = (torch.rand(n, length, generator=gen, device=DEV) ** 3 * vocab).int()
    dout = torch.randn(n, length, dim, generator=gen, device=DEV).to(dtype)
    before = torch.randn(n, vocab, dim, generator=gen, device=DEV)

    def grad(cut):
        out = before[..., cut].clone()
        return pb.embedding_grad(dout[..., cut], tokens, vocab, 0.7, dtable=out, accumulate=accumulate)

    want = grad(slice(None))
    for cut in (slice(0, 256), slice(0, 257), slice(0, 200), slice(256, 600), slice(100, 101), slice(3, 515), slice(0, 512), slice(8, 600), slice(88, 600)):
        assert torch.equal(grad(cut).view(torch.int32), want[..., cut].contiguous().view(torch.int32)), cut
