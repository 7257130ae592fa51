"""The token operators stand outside autograd: results have no graph, and torch's own check sees that a given tensor was overwritten."""
import pytest
import torch

import paper_1707_00424_b200 as pb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def inputs():
    torch.manual_seed(0)
    x, t = torch.randn(6, 16, device=DEV), torch.randint(0, 16, (6,), device=DEV, dtype=torch.int32)
    return x, t, torch.randn(6, device=DEV)


CALLS = {
    "logprobs": lambda x, t, g, o: pb.token_logprobs(x, t, k=2, logprob=o["row"], entropy=o["row2"], top_token=o["whole"], top_logprob=o["pairs"], flags=o["flags"]),
    "gradient": lambda x, t, g, o: pb.token_logprobs_grad(x, t, g, g, dlogits=o["like"], logprob=o["row"], entropy=o["row2"], flags=o["flags"]),
    "embedding": lambda x, t, g, o: pb.embedding(x, t, out=o["like"], flags=o["flags"]),
    "embedding gradient": lambda x, t, g, o: pb.embedding_grad(x, t, 16, dtable=o["table"], workspace=o["bytes"], flags=o["flags"]),
    "accumulated": lambda x, t, g, o: pb.embedding_grad(x, t, 16, dtable=o["table"], accumulate=True),
    "dropout": lambda x, t, g, o: pb.dropout(x, 0.5, 1, residual=x, out=o["like"]),
}
WRITTEN = {
    "logprobs": {"row", "row2", "whole", "pairs", "flags"}, "gradient": {"like", "row", "row2", "flags"}, "embedding": {"like", "flags"},
    "embedding gradient": {"table", "bytes", "flags"}, "accumulated": {"table"}, "dropout": {"like"},
}


def outputs():
    return {"row": torch.zeros(6, device=DEV), "row2": torch.zeros(6, device=DEV), "whole": torch.zeros(6, 2, dtype=torch.int32, device=DEV),
            "pairs": torch.zeros(6, 2, device=DEV), "like": torch.zeros(6, 16, device=DEV), "table": torch.zeros(16, 16, device=DEV),
            "bytes": torch.zeros(1 << 12, dtype=torch.uint8, device=DEV), "flags": torch.zeros(1, dtype=torch.int32, device=DEV)}


@pytest.mark.parametrize("name", CALLS)
def test_given_tensors_count_as_written_and_inputs_do_not(name):
    given, out = inputs(), outputs()
    before = {k: v._version for k, v in out.items()}
    CALLS[name](*given, out)
    assert {k for k, v in out.items() if v._version != before[k]} == WRITTEN[name]
    assert all(v._version == w._version for v, w in zip(given, inputs()))


@pytest.mark.parametrize("call", [
    lambda y, t, g: pb.dropout(y, 0.5, 1, out=y), lambda y, t, g: pb.token_logprobs_grad(y, t, g, dlogits=y),
    lambda y, t, g: pb.embedding(y.clone(), t, out=y), lambda y, t, g: pb.embedding_grad(y.clone(), t, 6, dtable=y, accumulate=True),
    lambda y, t, g: pb.token_logprobs(y.clone(), t, entropy=y[:, 0].as_strided((6,), (1,))),
])
def test_a_saved_tensor_that_was_overwritten_is_torchs_error(call):
    x, t, g = inputs()
    t %= 6
    y = x.requires_grad_().exp()                          # saves its result
    call(y.detach(), t, g)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


def test_results_have_no_graph():
    x, t, g = inputs()
    x.requires_grad_()
    results = [*pb.token_logprobs(x, t, k=2), pb.token_logprobs_grad(x, t, g), pb.embedding(x, t % 6), pb.embedding_grad(x, t, 16), pb.dropout(x, 0.5, 1)]
    assert not any(r.requires_grad for r in results)
    assert "autograd" in pb.token_ops.__doc__


def test_inference_tensors_are_written_too():
    with torch.inference_mode():
        x, t, g = inputs()
        out = outputs()
        for name, call in CALLS.items():
            call(x, t, g, out)
    for name, call in CALLS.items():
        call(x, t, g, out)
    assert torch.equal(pb.dropout(x, 0.0, 1, out=x), x)
