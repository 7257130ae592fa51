"""Token operators of libparle.so: embedding lookup and its gradient, counter-based dropout, log probabilities of given tokens
with entropy, top alternatives and gradient, sampling of tokens.

Each function checks its tensors, then makes one call of the C ABI (include/parle.h has the definitions) on `stream`, or on the
current stream of the tensors' device: both in the module _token_ops (csrc/token_bindings.cpp).  Results go to the tensors given
for them; those not given are allocated with torch.  Tensors are strided as they come: only the last dimension has to be dense.

The functions stand outside autograd, as all of this package: what they return has no graph, whether an input requires a gradient or not;
their gradients are calls of their own.  Tensors given for results count as modified in place, so that a backward pass of torch that
saved one of them raises its usual error."""
from __future__ import annotations

from .binding import ParleError, lib

NO_TOKEN = -1
TOP_MAX = 32
_MODULE = None


def load():
    """The compiled module, built first if it is missing or was built from other sources or for another torch."""
    global _MODULE
    if _MODULE is None:
        from . import build
        build.build_module()
        lib()
        from . import _token_ops as module
        if not module.built_from.startswith(build.module_stamp()):
            raise RuntimeError("_token_ops.so changed while it was loaded: start again")
        module.set_error(ParleError)
        _MODULE = module
    return _MODULE


def token_logprobs(logits, tokens=None, k: int = 0, scale: float = 1.0, *, logprob=None, entropy=None, top_token=None,
                   top_logprob=None, flags=None, stream=None):
    """(logprob, entropy, top_token, top_logprob) of logits [..., vocab] at the inverse temperature `scale`
    (parle_token_logprobs): log probability of tokens [...] (int32, NO_TOKEN where there is none; logprob is None without
    tokens), entropy, and the k <= TOP_MAX most probable tokens with their log probabilities, [..., k]."""
    return (_MODULE or load()).token_logprobs(logits, tokens, k, scale, logprob, entropy, top_token, top_logprob, flags, stream)


def token_logprobs_grad(logits, tokens=None, d_logprob=None, d_entropy=None, scale: float = 1.0, *, dlogits=None, logprob=None,
                        entropy=None, flags=None, stream=None):
    """dlogits of sum(d_logprob * logprob + d_entropy * entropy) (parle_token_logprobs_grad); dlogits may be logits itself.
    logprob and entropy are formed in the same pass when given."""
    return (_MODULE or load()).token_logprobs_grad(logits, tokens, d_logprob, d_entropy, scale, dlogits, logprob, entropy, flags, stream)


def sample_tokens(logits, u, *, scale=1.0, top_k=0, top_p=1.0, min_p=0.0, token=None, logprob=None, kept=None, flags=None, stream=None):
    """(token, logprob, kept) of logits [..., vocab] by random numbers u [...] (fp32, in [0, 1)) (parle_sample_tokens): a token sampled at
    the inverse temperature `scale` among the top_k most probable (0: all), of these the most probable that make up top_p, of these those
    at least min_p times as probable as the best; its log probability among them, and their number.  scale, top_k, top_p and min_p are
    numbers, or tensors [...] (fp32; int32 for top_k) with one for each row."""
    return (_MODULE or load()).sample_tokens(logits, u, scale, top_k, top_p, min_p, token, logprob, kept, flags, stream)


def embedding(table, tokens, scale: float = 1.0, *, out=None, dtype=None, flags=None, stream=None):
    """out[..., :] = scale * table[tokens[...], :] (parle_embedding): table [vocab, dim] with tokens of any shape, or one table per
    replica, [n, vocab, dim], with tokens [n, ...].  out: tokens' shape + [dim], of type `dtype` (the table's)."""
    return (_MODULE or load()).embedding(table, tokens, scale, out, dtype, flags, stream)


def embedding_grad_workspace_bytes(n: int, length: int, vocab: int, dim: int) -> int:
    """Bytes of scratch that embedding_grad() needs for n tables and `length` positions each; 0 for sizes that it refuses."""
    if min(n, length, vocab, dim) < 0 or max(n, vocab, dim) >= 1 << 31 or length >= 1 << 63:      # (ctypes would cut them off)
        return 0
    return lib().parle_embedding_grad_workspace_bytes(n, length, vocab, dim)


def embedding_grad(dout, tokens, vocab: int, scale: float = 1.0, *, n=None, dtable=None, accumulate: bool = False, workspace=None,
                   flags=None, stream=None):
    """dtable[v, :] = scale * sum of the rows of dout [..., dim] whose token is v (parle_embedding_grad): fp32 [vocab, dim], or
    [n, vocab, dim] when dtable has three dimensions or n is given (tokens and dout then begin with n).  accumulate adds to
    dtable.  workspace: scratch of embedding_grad_workspace_bytes(), allocated when not given."""
    return (_MODULE or load()).embedding_grad(dout, tokens, vocab, scale, n, dtable, accumulate, workspace, flags, stream)


def dropout(x, p: float, seed: int, offset: int = 0, *, residual=None, out=None, offset_dev=None, stream=None):
    """residual + dropout(x), the mask a function of (seed, offset + *offset_dev, element number) (parle_dropout).  out may be x or
    residual.  The gradient of x is dropout(gradient of the output, p, seed, offset)."""
    return (_MODULE or load()).dropout(x, p, seed, offset, residual, out, offset_dev, stream)
