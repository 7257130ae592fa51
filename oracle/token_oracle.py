"""fp64 oracle of the token operators, written from their definitions (numpy, one row or one token at a time): log probabilities
of given tokens with entropy, top alternatives and gradient; embedding lookup and its gradient; dropout from Philox 4x32-10."""
from __future__ import annotations

import math

import numpy as np

NO_TOKEN = -1


def log_softmax(x, scale: float):
    """log p of one row.  -inf logits have probability 0; a row of -inf alone gives -inf, NaN or +inf gives NaN."""
    x = np.asarray(x, np.float64)
    if np.isnan(x).any() or np.isposinf(x).any():
        return np.full(x.shape, np.nan)
    m = x.max()
    if m == -np.inf:
        return np.full(x.shape, -np.inf)
    d = scale * (x - m)
    return d - math.log(np.exp(d).sum())


def entropy(logp) -> float:
    if np.isnan(logp).any():
        return math.nan
    real = logp[logp > -np.inf]
    return float(-(np.exp(real) * real).sum())


def top(x, logp, k: int):
    """The k largest logits: (tokens, log probabilities); equal logits by token; -inf is no alternative."""
    if np.isnan(logp).any():
        return [NO_TOKEN] * k, [math.nan] * k
    order = sorted(range(len(x)), key=lambda j: (-float(x[j]), j))
    order = [j for j in order if x[j] > -np.inf][:k]
    rest = k - len(order)
    return order + [NO_TOKEN] * rest, [float(logp[j]) for j in order] + [-math.inf] * rest


def token_logprobs(x, tokens, scale: float = 1.0, k: int = 0):
    """x [rows, vocab] -> logprob [rows], entropy [rows], top tokens [rows, k], their log probabilities [rows, k]."""
    rows, vocab = x.shape
    out = np.zeros(rows), np.zeros(rows), np.zeros((rows, k), np.int64), np.zeros((rows, k))
    for r in range(rows):
        logp = log_softmax(x[r], scale)
        out[0][r] = logp[tokens[r]] if 0 <= tokens[r] < vocab else 0.0
        out[1][r] = entropy(logp)
        if k:
            out[2][r], out[3][r] = top(x[r], logp, k)
    return out


def token_logprobs_grad(x, tokens, d_logprob, d_entropy, scale: float = 1.0):
    """d/dx of sum_rows d_logprob log p_token + d_entropy H; None stands for zeros."""
    rows, vocab = x.shape
    grad = np.zeros((rows, vocab))
    for r in range(rows):
        real = 0 <= tokens[r] < vocab
        g = float(d_logprob[r]) if d_logprob is not None and real else 0.0
        h = float(d_entropy[r]) if d_entropy is not None else 0.0
        logp = log_softmax(x[r], scale)
        if g == 0 and h == 0 or np.isneginf(logp).all():
            continue
        p = np.exp(logp)
        one = np.zeros(vocab)
        if real:
            one[tokens[r]] = 1.0
        plogp = np.where(p > 0, p * np.where(p > 0, logp, 0.0), 0.0) if not np.isnan(p).any() else p
        grad[r] = scale * (g * (one - p) - h * (plogp + p * entropy(logp)))
    return grad


def embedding(table, tokens, scale: float = 1.0):
    """table [n, vocab, dim], tokens [n, length] -> [n, length, dim]; a place without a token gives zeros."""
    n, length = tokens.shape
    out = np.zeros((n, length, table.shape[2]))
    for g in range(n):
        for t in range(length):
            if 0 <= tokens[g, t] < table.shape[1]:
                out[g, t] = scale * np.asarray(table[g, tokens[g, t]], np.float64)
    return out


def embedding_grad(dout, tokens, vocab: int, scale: float = 1.0):
    """dout [n, length, dim], tokens [n, length] -> (sums [n, vocab, dim], the same sums of absolute values, terms [n, vocab])."""
    n, length, dim = dout.shape
    total, size, count = np.zeros((n, vocab, dim)), np.zeros((n, vocab, dim)), np.zeros((n, vocab), np.int64)
    for g in range(n):
        for t in range(length):
            v = tokens[g, t]
            if 0 <= v < vocab:
                row = np.asarray(dout[g, t], np.float64)
                total[g, v] += row
                size[g, v] += np.abs(row)
                count[g, v] += 1
    return scale * total, abs(scale) * size, count


def philox4x32_10(counter, key):
    """Philox 4x32 with ten rounds (Salmon, Moraes, Dror, Shaw, SC 2011): four 32-bit words of a counter and a two-word key."""
    c, k, low = list(counter), list(key), 0xFFFFFFFF
    for _ in range(10):
        a, b = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(b >> 32) ^ c[1] ^ k[0], b & low, (a >> 32) ^ c[3] ^ k[1], a & low]
        k = [(k[0] + 0x9E3779B9) & low, (k[1] + 0xBB67AE85) & low]
    return c


def dropout_fields(elements: int, seed: int, offset: int, first: int = 0):
    """The 16-bit fields of elements first .. first + elements - 1."""
    low, out = 0xFFFFFFFF, []
    offset %= 1 << 64
    for group in range(first // 8, (first + elements + 7) // 8):
        for w in philox4x32_10((group & low, group >> 32, offset & low, offset >> 32), (seed & low, seed >> 32)):
            out += [w & 0xFFFF, w >> 16]
    skip = first % 8
    return np.array(out[skip:skip + elements], np.int64)


def dropout(x, p: float, seed: int, offset: int, residual=None):
    """x [rows, cols] of any float type -> fp64."""
    threshold = math.floor(p * 65536 + 0.5)
    keep = dropout_fields(x.size, seed, offset).reshape(x.shape) >= threshold
    y = np.zeros(x.shape)
    y[keep] = np.asarray(x, np.float64)[keep] * 65536 / (65536 - threshold) if threshold < 65536 else 0
    return y if residual is None else y + np.asarray(residual, np.float64)


def sample(x, u: float, scale: float = 1.0, top_k: int = 0, top_p: float = 1.0, min_p: float = 0.0):
    """One row: (token, log probability among the kept, number kept, how near a comparison of sums was, relative to the sums).  Parameters as
    fp32 numbers; a row or parameters without an answer give NO_TOKEN, NaN or -inf, 0, 1."""
    x = np.asarray(x, np.float64)
    u, scale, top_p, min_p = (float(np.float32(v)) for v in (u, scale, top_p, min_p))
    bad = not (float(np.float32(1e-6)) <= scale <= 1e6 and 0 <= u < 1) or math.isnan(top_p) or math.isnan(min_p)
    if bad or np.isnan(x).any() or np.isposinf(x).any():
        return NO_TOKEN, math.nan, 0, 1.0
    best = x.max()
    if best == -np.inf:
        return NO_TOKEN, -math.inf, 0, 1.0
    order = np.lexsort((np.arange(len(x)), -x))
    order = order[x[order] > -np.inf]
    if top_k > 0:
        order = order[:top_k]
    near = 1.0
    w = np.exp(scale * (x[order] - best))
    kept = len(order)
    if top_p < 1:
        sums = np.cumsum(w)
        kept = int((sums < top_p * sums[-1]).sum()) + 1
        near = np.abs(sums - top_p * sums[-1]).min() / sums[-1]
    if min_p > 0:
        kept = min(kept, int((x[order] >= best + math.log(min(min_p, 1.0)) / scale).sum()))
    tokens = np.sort(order[:kept])
    w = np.exp(scale * (x[tokens] - best))
    sums = np.cumsum(w)
    at = int((sums <= u * sums[-1]).sum())
    at = min(at, int(np.flatnonzero(w).max()))             # (u below 1 by less than the sums' rounding)
    near = min(near, np.abs(sums[:-1] - u * sums[-1]).min() / sums[-1] if kept > 1 else 1.0)
    return int(tokens[at]), float(scale * (x[tokens[at]] - best) - math.log(sums[-1])), kept, float(near)
