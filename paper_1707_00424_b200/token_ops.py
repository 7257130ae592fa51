"""Token operators of libparle.so: embedding lookup and its gradient, counter-based dropout, log probabilities of given tokens
with entropy, top alternatives and gradient.

Each function checks its tensors, then makes one call of the C ABI (include/parle.h has the definitions) on `stream`, or on the
current stream of the tensors' device.  Results go to the tensors given for them; those not given are allocated with torch.
Tensors are strided as they come: only the last dimension has to be dense."""
from __future__ import annotations

import torch

from .binding import ParleError, lib

NO_TOKEN = -1
TOP_MAX = 32
_EINVAL = -1
_DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}


def _refuse(call: str, why: str):
    raise ParleError(_EINVAL, f"{call}: {why}")


def _dtype(call: str, name: str, t) -> int:
    d = _DTYPES.get(t.dtype)
    if d is None:
        _refuse(call, f"{name} has type {t.dtype}: fp32, bf16 and fp16 are supported")
    return d


def _on(call: str, device, **tensors):
    """Every given tensor is on the CUDA device `device`."""
    if device.type != "cuda":
        _refuse(call, f"the tensors are on {device}: a CUDA device is needed")
    for name, t in tensors.items():
        if t is not None and t.device != device:
            _refuse(call, f"{name} is on {t.device}, the others on {device}")


def _dense(call: str, name: str, t, shape, dtype):
    """A contiguous tensor of this shape and type."""
    if t.shape != shape or t.dtype != dtype or not t.is_contiguous():
        _refuse(call, f"{name} has to be a contiguous {dtype} tensor of shape {tuple(shape)}, not {t.dtype} {tuple(t.shape)} with strides {t.stride()}")


def _flags(call: str, flags):
    if flags is not None and (flags.numel() != 1 or flags.dtype != torch.int32):
        _refuse(call, "flags has to be one int32")


def _groups(call: str, name: str, t, *shape):
    """t as [.., .., dim] of this shape, its last dimension dense, without a copy."""
    if t.shape != shape:
        try:
            t = t.view(shape)
        except RuntimeError:
            _refuse(call, f"{name} of shape {tuple(t.shape)} and strides {t.stride()} is no {shape} without a copy")
    if shape[-1] > 1 and t.stride(-1) != 1:
        _refuse(call, f"the last dimension of {name} is not dense (strides {t.stride()})")
    return t


def _pitch(t, dim: int) -> int:
    """Pitch of dimension `dim`; that of a dimension of one element has no meaning and becomes the dense one."""
    if t.shape[dim] > 1:
        return t.stride(dim)
    return max(1, t.shape[-1]) * (t.shape[-2] if dim == t.dim() - 3 else 1)


def _rows(call: str, name: str, t):
    """t [..., cols] as [rows, cols]."""
    if t.dim() == 2:
        return _groups(call, name, t, *t.shape)
    if t.dim() == 0:
        _refuse(call, f"{name} has no dimension")
    return _groups(call, name, t, t.numel() // t.shape[-1] if t.shape[-1] else 0, t.shape[-1])


def _call(call: str, device, stream, *args):
    """lib().<call>(*args, stream) with `device` current."""
    fn = getattr(lib(), call)
    if stream is None:
        stream = torch.cuda.current_stream(device)
    elif stream.device != device:
        _refuse(call, f"the stream is on {stream.device}, the tensors on {device}")
    if torch.cuda.current_device() == device.index:
        rc = fn(*args, stream.cuda_stream)
    else:
        with torch.cuda.device(device):
            rc = fn(*args, stream.cuda_stream)
    if rc != 0:
        raise ParleError(rc, call)


def _new(device, stream, shape, dtype):
    """Memory for a result: of the stream that the call runs on."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _ptr(t) -> int:
    return 0 if t is None else t.data_ptr()


def token_logprobs(logits, tokens=None, k: int = 0, scale: float = 1.0, *, logprob=None, entropy=None, top_token=None,
                   top_logprob=None, flags=None, stream=None):
    """(logprob, entropy, top_token, top_logprob) of logits [..., vocab] at the inverse temperature `scale`
    (parle_token_logprobs): log probability of tokens [...] (int32, NO_TOKEN where there is none; logprob is None without
    tokens), entropy, and the k <= TOP_MAX most probable tokens with their log probabilities, [..., k]."""
    call = "parle_token_logprobs"
    _on(call, logits.device, tokens=tokens, logprob=logprob, entropy=entropy, top_token=top_token, top_logprob=top_logprob, flags=flags)
    dtype, x, lead, device = _dtype(call, "logits", logits), _rows(call, "logits", logits), logits.shape[:-1], logits.device
    if not 0 <= k <= TOP_MAX:
        _refuse(call, f"k = {k} is not in [0, {TOP_MAX}]")
    if tokens is not None:
        _dense(call, "tokens", tokens, lead, torch.int32)
        if logprob is None:
            logprob = _new(device, stream, lead, torch.float32)
        else:
            _dense(call, "logprob", logprob, lead, torch.float32)
    elif logprob is not None:
        _refuse(call, "logprob needs tokens")
    if entropy is None:
        entropy = _new(device, stream, lead, torch.float32)
    else:
        _dense(call, "entropy", entropy, lead, torch.float32)
    if top_token is None:
        top_token = _new(device, stream, (*lead, k), torch.int32)
    else:
        _dense(call, "top_token", top_token, (*lead, k), torch.int32)
    if top_logprob is None:
        top_logprob = _new(device, stream, (*lead, k), torch.float32)
    else:
        _dense(call, "top_logprob", top_logprob, (*lead, k), torch.float32)
    _flags(call, flags)
    _call(call, device, stream, x.data_ptr(), dtype, x.shape[0], x.shape[1], _pitch(x, 0), _ptr(tokens), scale, k, _ptr(logprob),
          entropy.data_ptr(), top_token.data_ptr() if k else 0, top_logprob.data_ptr() if k else 0, _ptr(flags))
    return logprob, entropy, top_token, top_logprob


def token_logprobs_grad(logits, tokens=None, d_logprob=None, d_entropy=None, scale: float = 1.0, *, dlogits=None, logprob=None,
                        entropy=None, flags=None, stream=None):
    """dlogits of sum(d_logprob * logprob + d_entropy * entropy) (parle_token_logprobs_grad); dlogits may be logits itself.
    logprob and entropy are formed in the same pass when given."""
    call = "parle_token_logprobs_grad"
    _on(call, logits.device, tokens=tokens, d_logprob=d_logprob, d_entropy=d_entropy, dlogits=dlogits, logprob=logprob, entropy=entropy, flags=flags)
    dtype, x, lead, device = _dtype(call, "logits", logits), _rows(call, "logits", logits), logits.shape[:-1], logits.device
    if tokens is not None:
        _dense(call, "tokens", tokens, lead, torch.int32)
    for name, t in (("d_logprob", d_logprob), ("d_entropy", d_entropy), ("logprob", logprob), ("entropy", entropy)):
        if t is not None:
            _dense(call, name, t, lead, torch.float32)
    if dlogits is None:
        dlogits = _new(device, stream, logits.shape, logits.dtype)
    elif dlogits.shape != logits.shape or dlogits.dtype != logits.dtype:
        _refuse(call, f"dlogits is {dlogits.dtype} {tuple(dlogits.shape)}, logits {logits.dtype} {tuple(logits.shape)}")
    d = _rows(call, "dlogits", dlogits)
    _flags(call, flags)
    _call(call, device, stream, x.data_ptr(), dtype, x.shape[0], x.shape[1], _pitch(x, 0), _ptr(tokens), scale, _ptr(d_logprob),
          _ptr(d_entropy), _ptr(logprob), _ptr(entropy), d.data_ptr(), _pitch(d, 0), _ptr(flags))
    return dlogits


def embedding(table, tokens, scale: float = 1.0, *, out=None, dtype=None, flags=None, stream=None):
    """out[..., :] = scale * table[tokens[...], :] (parle_embedding): table [vocab, dim] with tokens of any shape, or one table per
    replica, [n, vocab, dim], with tokens [n, ...].  out: tokens' shape + [dim], of type `dtype` (the table's)."""
    call = "parle_embedding"
    _on(call, table.device, tokens=tokens, out=out, flags=flags)
    if table.dim() not in (2, 3):
        _refuse(call, f"table has {table.dim()} dimensions, not [vocab, dim] or [n, vocab, dim]")
    t3 = table if table.dim() == 3 else table[None]
    n, vocab, dim = t3.shape
    t3 = _groups(call, "table", t3, n, vocab, dim)
    if table.dim() == 3 and (tokens.dim() == 0 or tokens.shape[0] != n):
        _refuse(call, f"{n} tables and tokens of shape {tuple(tokens.shape)}")
    _dense(call, "tokens", tokens, tokens.shape, torch.int32)
    if out is None:
        out = _new(table.device, stream, (*tokens.shape, dim), dtype or table.dtype)
    elif out.shape != (*tokens.shape, dim) or (dtype is not None and out.dtype != dtype):
        _refuse(call, f"out is {out.dtype} {tuple(out.shape)}, not {dtype or out.dtype} {(*tokens.shape, dim)}")
    length = tokens.numel() // n if n else 0
    o = _groups(call, "out", out, n, length, dim)
    _flags(call, flags)
    _call(call, table.device, stream, t3.data_ptr(), _dtype(call, "table", table), _pitch(t3, 0), _pitch(t3, 1), n, vocab, dim,
          tokens.data_ptr(), length, scale, o.data_ptr(), _dtype(call, "out", out), _pitch(o, 0), _pitch(o, 1), _ptr(flags))
    return out


def embedding_grad_workspace_bytes(n: int, length: int, vocab: int, dim: int) -> int:
    """Bytes of scratch that embedding_grad() needs for n tables and `length` positions each."""
    return lib().parle_embedding_grad_workspace_bytes(n, length, vocab, dim)


def embedding_grad(dout, tokens, vocab: int, scale: float = 1.0, *, n=None, dtable=None, accumulate: bool = False, workspace=None,
                   flags=None, stream=None):
    """dtable[v, :] = scale * sum of the rows of dout [..., dim] whose token is v (parle_embedding_grad): fp32 [vocab, dim], or
    [n, vocab, dim] when dtable has three dimensions or n is given (tokens and dout then begin with n).  accumulate adds to
    dtable.  workspace: uint8 scratch of embedding_grad_workspace_bytes(), allocated when not given."""
    call = "parle_embedding_grad"
    device = dout.device
    _on(call, device, tokens=tokens, dtable=dtable, workspace=workspace, flags=flags)
    _dense(call, "tokens", tokens, tokens.shape, torch.int32)
    if dout.shape[:-1] != tokens.shape or dout.dim() == 0:
        _refuse(call, f"dout of shape {tuple(dout.shape)} and tokens of shape {tuple(tokens.shape)}")
    dim = dout.shape[-1]
    if dtable is None:
        if accumulate:
            _refuse(call, "accumulate needs a dtable")
        dtable = _new(device, stream, (vocab, dim) if n is None else (n, vocab, dim), torch.float32)
    grouped = dtable.dim() == 3
    groups = dtable.shape[0] if grouped else 1
    if dtable.dtype != torch.float32 or dtable.shape[-2:] != (vocab, dim) or dtable.dim() not in (2, 3) or (n is not None and (not grouped or n != groups)):
        _refuse(call, f"dtable is {dtable.dtype} {tuple(dtable.shape)}: fp32 [{vocab}, {dim}] or [n, {vocab}, {dim}] is needed")
    if grouped and (tokens.dim() == 0 or tokens.shape[0] != groups):
        _refuse(call, f"{groups} tables and tokens of shape {tuple(tokens.shape)}")
    length = tokens.numel() // groups if groups else 0
    d = _groups(call, "dout", dout, groups, length, dim)
    t = _groups(call, "dtable", dtable if grouped else dtable[None], groups, vocab, dim)
    need = lib().parle_embedding_grad_workspace_bytes(groups, length, vocab, dim)
    if workspace is None:
        workspace = _new(device, stream, need, torch.uint8)
    elif not workspace.is_contiguous():
        _refuse(call, "workspace is not contiguous")
    _flags(call, flags)
    _call(call, device, stream, d.data_ptr(), _dtype(call, "dout", dout), _pitch(d, 0), _pitch(d, 1), tokens.data_ptr(), groups, length,
          vocab, dim, scale, t.data_ptr(), _pitch(t, 0), _pitch(t, 1), 1 if accumulate else 0, workspace.data_ptr(),
          workspace.numel() * workspace.element_size(), _ptr(flags))
    return dtable


def dropout(x, p: float, seed: int, offset: int = 0, *, residual=None, out=None, offset_dev=None, stream=None):
    """residual + dropout(x), the mask a function of (seed, offset + *offset_dev, element number) (parle_dropout).  out may be x or
    residual.  The gradient of x is dropout(gradient of the output, p, seed, offset)."""
    call = "parle_dropout"
    _on(call, x.device, residual=residual, out=out, offset_dev=offset_dev)
    dtype, device = _dtype(call, "x", x), x.device
    if out is None:
        out = _new(device, stream, x.shape, x.dtype)
    for name, t in (("residual", residual), ("out", out)):
        if t is not None and (t.shape != x.shape or t.dtype != x.dtype):
            _refuse(call, f"{name} is {t.dtype} {tuple(t.shape)}, x {x.dtype} {tuple(x.shape)}")
    if offset_dev is not None and (offset_dev.numel() != 1 or offset_dev.dtype not in (torch.int64, torch.uint64)):
        _refuse(call, "offset_dev has to be one 64-bit integer")
    if not (0 <= seed < 1 << 64 and 0 <= offset < 1 << 64):
        _refuse(call, "seed and offset are unsigned 64-bit numbers")
    a, y = _rows(call, "x", x), _rows(call, "out", out)
    r = None if residual is None else _rows(call, "residual", residual)
    _call(call, device, stream, a.data_ptr(), _pitch(a, 0), _ptr(r), 0 if r is None else _pitch(r, 0), y.data_ptr(), _pitch(y, 0), dtype,
          a.shape[0], a.shape[1], p, seed, offset, _ptr(offset_dev))
    return out
