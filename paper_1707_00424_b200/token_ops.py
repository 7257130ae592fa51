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
_FLOAT, _INT, _INTS, _LONGS = torch.float32, torch.int32, (torch.int32,), (torch.int64, torch.uint64)


def _refuse(call: str, why: str):
    raise ParleError(_EINVAL, f"{call}: {why}")


def _device_of(call: str, t) -> int:
    """Index of the tensor's CUDA device."""
    index = t.get_device()
    if index < 0:
        _refuse(call, f"a tensor is on {t.device}: a CUDA device is needed")
    return index


def _dtype(call: str, name: str, t) -> int:
    d = _DTYPES.get(t.dtype)
    if d is None:
        _refuse(call, f"{name} has type {t.dtype}: fp32, bf16 and fp16 are supported")
    return d


def _dense(call: str, name: str, t, shape, dtype, index: int) -> int:
    """Address of a contiguous tensor of this shape and type on this device."""
    if t.shape != shape or t.dtype is not dtype or not t.is_contiguous():
        _refuse(call, f"{name} has to be a contiguous {dtype} tensor of shape {tuple(shape)}, not {t.dtype} {tuple(t.shape)} with strides {t.stride()}")
    if t.get_device() != index:
        _refuse(call, f"{name} is on {t.device}, the other tensors on cuda:{index}")
    return t.data_ptr()


def _word(call: str, name: str, t, dtypes, index: int) -> int:
    """Address of a tensor of one element, 0 for None."""
    if t is None:
        return 0
    if t.numel() != 1 or t.dtype not in dtypes or t.get_device() != index:
        _refuse(call, f"{name} has to be one element of {' or '.join(map(str, dtypes))} on cuda:{index}")
    return t.data_ptr()


def _rows(call: str, name: str, t, index: int):
    """t [..., cols] as (address, rows, cols, pitch); its last dimension has to be dense."""
    if t.dim() != 2:
        if t.dim() == 0:
            _refuse(call, f"{name} has no dimension")
        try:
            t = t.view(t.numel() // t.shape[-1] if t.shape[-1] else 0, t.shape[-1])
        except RuntimeError:
            _refuse(call, f"{name} of shape {tuple(t.shape)} and strides {t.stride()} is no array of rows without a copy")
    if t.get_device() != index:
        _refuse(call, f"{name} is on {t.device}, the other tensors on cuda:{index}")
    (rows, cols), (pitch, step) = t.shape, t.stride()
    if step != 1 and cols > 1:
        _refuse(call, f"the last dimension of {name} is not dense (strides {t.stride()})")
    return t.data_ptr(), rows, cols, pitch if rows > 1 else cols


def _groups(call: str, name: str, t, n: int, rows: int, cols: int, index: int):
    """t as [n, rows, cols], without a copy: (address, group pitch, row pitch)."""
    if t.dim() != 3 or t.shape[1] != rows:
        try:
            t = t.view(n, rows, cols)
        except RuntimeError:
            _refuse(call, f"{name} of shape {tuple(t.shape)} and strides {t.stride()} is no {(n, rows, cols)} without a copy")
    if t.get_device() != index:
        _refuse(call, f"{name} is on {t.device}, the other tensors on cuda:{index}")
    group, pitch, step = t.stride()
    if step != 1 and cols > 1:
        _refuse(call, f"the last dimension of {name} is not dense (strides {t.stride()})")
    if rows <= 1:                                        # the pitch of a dimension of one element has no meaning
        pitch = cols
    return t.data_ptr(), group if n > 1 else max(1, rows) * cols, pitch


def _call(call: str, index: int, stream, *args):
    """lib().<call>(*args, stream) with device `index` current."""
    fn = getattr(_LIB or _load(), call)
    if stream is None:
        raw = _current_raw_stream(index)
    else:
        if stream.device.index != index:
            _refuse(call, f"the stream is on {stream.device}, the tensors on cuda:{index}")
        raw = stream.cuda_stream
    if _current_device() == index:
        rc = fn(*args, raw)
    else:
        with torch.cuda.device(index):
            rc = fn(*args, raw)
    if rc != 0:
        raise ParleError(rc, call)


# (torch.cuda.current_stream() and current_device() make objects on the way: 2.2 us instead of 0.2 us a call)
_current_raw_stream, _current_device = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice
_LIB = None


def _load():
    global _LIB
    _LIB = lib()
    return _LIB


def _new(index: int, stream, shape, dtype):
    """Memory for a result: of the stream that the call runs on."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=index)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=index)


def token_logprobs(logits, tokens=None, k: int = 0, scale: float = 1.0, *, logprob=None, entropy=None, top_token=None,
                   top_logprob=None, flags=None, stream=None):
    """(logprob, entropy, top_token, top_logprob) of logits [..., vocab] at the inverse temperature `scale`
    (parle_token_logprobs): log probability of tokens [...] (int32, NO_TOKEN where there is none; logprob is None without
    tokens), entropy, and the k <= TOP_MAX most probable tokens with their log probabilities, [..., k]."""
    call = "parle_token_logprobs"
    index, dtype = _device_of(call, logits), _dtype(call, "logits", logits)
    x, rows, vocab, pitch = _rows(call, "logits", logits, index)
    lead = logits.shape[:-1]
    if not 0 <= k <= TOP_MAX:
        _refuse(call, f"k = {k} is not in [0, {TOP_MAX}]")
    if tokens is None:
        if logprob is not None:
            _refuse(call, "logprob needs tokens")
        tokens_at = logprob_at = 0
    else:
        tokens_at = _dense(call, "tokens", tokens, lead, _INT, index)
        if logprob is None:
            logprob = _new(index, stream, lead, _FLOAT)
        logprob_at = _dense(call, "logprob", logprob, lead, _FLOAT, index)
    if entropy is None:
        entropy = _new(index, stream, lead, _FLOAT)
    entropy_at = _dense(call, "entropy", entropy, lead, _FLOAT, index)
    best = (*lead, k)
    if top_token is None:
        top_token = _new(index, stream, best, _INT)
    if top_logprob is None:
        top_logprob = _new(index, stream, best, _FLOAT)
    top_token_at, top_logprob_at = _dense(call, "top_token", top_token, best, _INT, index), _dense(call, "top_logprob", top_logprob, best, _FLOAT, index)
    if not k:
        top_token_at = top_logprob_at = 0
    _call(call, index, stream, x, dtype, rows, vocab, pitch, tokens_at, scale, k, logprob_at, entropy_at, top_token_at, top_logprob_at,
          _word(call, "flags", flags, _INTS, index))
    return logprob, entropy, top_token, top_logprob


def token_logprobs_grad(logits, tokens=None, d_logprob=None, d_entropy=None, scale: float = 1.0, *, dlogits=None, logprob=None,
                        entropy=None, flags=None, stream=None):
    """dlogits of sum(d_logprob * logprob + d_entropy * entropy) (parle_token_logprobs_grad); dlogits may be logits itself.
    logprob and entropy are formed in the same pass when given."""
    call = "parle_token_logprobs_grad"
    index, dtype = _device_of(call, logits), _dtype(call, "logits", logits)
    x, rows, vocab, pitch = _rows(call, "logits", logits, index)
    lead = logits.shape[:-1]
    given = [0 if t is None else _dense(call, name, t, lead, kind, index)
             for name, t, kind in (("tokens", tokens, _INT), ("d_logprob", d_logprob, _FLOAT), ("d_entropy", d_entropy, _FLOAT),
                                   ("logprob", logprob, _FLOAT), ("entropy", entropy, _FLOAT))]
    if dlogits is None:
        dlogits = _new(index, stream, logits.shape, logits.dtype)
    elif dlogits.shape != logits.shape or dlogits.dtype is not logits.dtype:
        _refuse(call, f"dlogits is {dlogits.dtype} {tuple(dlogits.shape)}, logits {logits.dtype} {tuple(logits.shape)}")
    d, _, _, d_pitch = _rows(call, "dlogits", dlogits, index)
    _call(call, index, stream, x, dtype, rows, vocab, pitch, given[0], scale, given[1], given[2], given[3], given[4], d, d_pitch,
          _word(call, "flags", flags, _INTS, index))
    return dlogits


def embedding(table, tokens, scale: float = 1.0, *, out=None, dtype=None, flags=None, stream=None):
    """out[..., :] = scale * table[tokens[...], :] (parle_embedding): table [vocab, dim] with tokens of any shape, or one table per
    replica, [n, vocab, dim], with tokens [n, ...].  out: tokens' shape + [dim], of type `dtype` (the table's)."""
    call = "parle_embedding"
    index, table_dtype = _device_of(call, table), _dtype(call, "table", table)
    if table.dim() == 3:
        n, vocab, dim = table.shape
        if tokens.dim() == 0 or tokens.shape[0] != n:
            _refuse(call, f"{n} tables and tokens of shape {tuple(tokens.shape)}")
        table_at, table_gs, ld_table = _groups(call, "table", table, n, vocab, dim, index)
    elif table.dim() == 2:
        n = 1
        table_at, vocab, dim, ld_table = _rows(call, "table", table, index)
        table_gs = vocab * dim
    else:
        _refuse(call, f"table has {table.dim()} dimensions, not [vocab, dim] or [n, vocab, dim]")
    shape = tokens.shape
    tokens_at = _dense(call, "tokens", tokens, shape, _INT, index)
    if out is None:
        out = _new(index, stream, (*shape, dim), dtype or table.dtype)
    elif out.shape != (*shape, dim) or (dtype is not None and out.dtype is not dtype):
        _refuse(call, f"out is {out.dtype} {tuple(out.shape)}, not {dtype or out.dtype} {(*shape, dim)}")
    length = tokens.numel() // n if n else 0
    out_at, out_gs, ld_out = _groups(call, "out", out, n, length, dim, index)
    _call(call, index, stream, table_at, table_dtype, table_gs, ld_table, n, vocab, dim, tokens_at, length, scale, out_at,
          _dtype(call, "out", out), out_gs, ld_out, _word(call, "flags", flags, _INTS, index))
    return out


def embedding_grad_workspace_bytes(n: int, length: int, vocab: int, dim: int) -> int:
    """Bytes of scratch that embedding_grad() needs for n tables and `length` positions each."""
    return lib().parle_embedding_grad_workspace_bytes(n, length, vocab, dim)


def embedding_grad(dout, tokens, vocab: int, scale: float = 1.0, *, n=None, dtable=None, accumulate: bool = False, workspace=None,
                   flags=None, stream=None):
    """dtable[v, :] = scale * sum of the rows of dout [..., dim] whose token is v (parle_embedding_grad): fp32 [vocab, dim], or
    [n, vocab, dim] when dtable has three dimensions or n is given (tokens and dout then begin with n).  accumulate adds to
    dtable.  workspace: scratch of embedding_grad_workspace_bytes(), allocated when not given."""
    call = "parle_embedding_grad"
    index, dtype = _device_of(call, dout), _dtype(call, "dout", dout)
    shape = tokens.shape
    tokens_at = _dense(call, "tokens", tokens, shape, _INT, index)
    dim = dout.shape[-1] if dout.dim() else 0
    if dout.shape != (*shape, dim):
        _refuse(call, f"dout of shape {tuple(dout.shape)} and tokens of shape {tuple(shape)}")
    if dtable is None:
        if accumulate:
            _refuse(call, "accumulate needs a dtable")
        dtable = _new(index, stream, (vocab, dim) if n is None else (n, vocab, dim), _FLOAT)
    if dtable.dim() == 3:
        groups = dtable.shape[0]
        fits = dtable.shape == (groups, vocab, dim) and n in (None, groups) and tokens.dim() > 0 and shape[0] == groups
    else:
        groups, fits = 1, dtable.shape == (vocab, dim) and n is None
    if not fits or dtable.dtype is not _FLOAT:
        _refuse(call, f"dtable is {dtable.dtype} {tuple(dtable.shape)}: fp32 [{vocab}, {dim}], or [n, {vocab}, {dim}] for tokens [n, ...], is needed")
    length = tokens.numel() // groups if groups else 0
    dout_at, dout_gs, ld_dout = _groups(call, "dout", dout, groups, length, dim, index)
    dtable_at, dtable_gs, ld_dtable = _groups(call, "dtable", dtable, groups, vocab, dim, index)
    if workspace is None:
        nbytes = (_LIB or _load()).parle_embedding_grad_workspace_bytes(groups, length, vocab, dim)
        workspace_at = 0
        if nbytes:
            workspace = _new(index, stream, nbytes, torch.uint8)
            workspace_at = workspace.data_ptr()
    else:
        if not workspace.is_contiguous() or workspace.get_device() != index:
            _refuse(call, f"workspace has to be contiguous and on cuda:{index}")
        workspace_at, nbytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    _call(call, index, stream, dout_at, dtype, dout_gs, ld_dout, tokens_at, groups, length, vocab, dim, scale, dtable_at, dtable_gs, ld_dtable,
          1 if accumulate else 0, workspace_at, nbytes, _word(call, "flags", flags, _INTS, index))
    return dtable


def dropout(x, p: float, seed: int, offset: int = 0, *, residual=None, out=None, offset_dev=None, stream=None):
    """residual + dropout(x), the mask a function of (seed, offset + *offset_dev, element number) (parle_dropout).  out may be x or
    residual.  The gradient of x is dropout(gradient of the output, p, seed, offset)."""
    call = "parle_dropout"
    index, dtype = _device_of(call, x), _dtype(call, "x", x)
    x_at, rows, cols, ld_x = _rows(call, "x", x, index)
    residual_at = ld_r = 0
    if residual is not None:
        if residual.shape != x.shape or residual.dtype is not x.dtype:
            _refuse(call, f"residual is {residual.dtype} {tuple(residual.shape)}, x {x.dtype} {tuple(x.shape)}")
        residual_at, _, _, ld_r = _rows(call, "residual", residual, index)
    if out is None:
        out = _new(index, stream, x.shape, x.dtype)
    elif out.shape != x.shape or out.dtype is not x.dtype:
        _refuse(call, f"out is {out.dtype} {tuple(out.shape)}, x {x.dtype} {tuple(x.shape)}")
    out_at, _, _, ld_y = _rows(call, "out", out, index)
    if not (0 <= seed < 1 << 64 and 0 <= offset < 1 << 64):
        _refuse(call, "seed and offset are unsigned 64-bit numbers")
    _call(call, index, stream, x_at, ld_x, residual_at, ld_r, out_at, ld_y, dtype, rows, cols, p, seed, offset,
          _word(call, "offset_dev", offset_dev, _LONGS, index))
    return out
