"""Cases of the token operators: log probabilities of given tokens (with entropy, top alternatives and their gradient),
embedding lookup (with the gradient of its table) and counter-based dropout.

`listed()` and `draw()` give the cases, `prepare()` a case's inputs on the GPU, `run()` one pass through the operator: in elementary
torch operations, or, where `own` is true, through the library's entry points.  `exact()` has the definitions in 64 bits."""
import math

import numpy as np
import torch

own = False
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
BYTES = {"fp32": 4, "bf16": 2, "fp16": 2}
LOG2_COST = math.log(2048 * 131072)             # the largest listed logits: no drawn case has more


def listed():
    return [
        # one sequence's next token, sampled from a large vocabulary, reported with twenty alternatives
        dict(name="logprobs next token", op="logprobs", rows=1, vocab=131072, pad=0, dtype="bf16", k=20, scale=1.0, masked=0.0),
        # a sampled batch: 64 rows at temperature 0.7, some tokens banned (-inf), odd vocabulary, fp32 logits
        dict(name="logprobs sampled batch", op="logprobs", rows=64, vocab=50021, pad=0, dtype="fp32", k=5, scale=1 / 0.7, masked=0.05),
        # scoring prompts: every position's token, entropy and the best eight
        dict(name="logprobs scoring", op="logprobs", rows=2048, vocab=131072, pad=0, dtype="bf16", k=8, scale=1.0, masked=0.0),
        # a training step's loss and its gradient at a large vocabulary
        dict(name="logprobs step large", op="logprobs_step", rows=2048, vocab=131072, pad=0, dtype="bf16", scale=1.0, entropy=True),
        # the same for sixteen replicas' minibatches of 256 rows over 1000 classes, fp32 logits
        dict(name="logprobs step replicas", op="logprobs_step", rows=4096, vocab=1000, pad=0, dtype="fp32", scale=1.0, entropy=False),
        # a prompt's rows from a bf16 table, scaled by sqrt(D)
        dict(name="embedding prompt", op="embedding", n=1, length=16384, vocab=131072, dim=4096, table="bf16", dtype="bf16", scale=64.0),
        # eight sequences' single tokens
        dict(name="embedding next tokens", op="embedding", n=1, length=8, vocab=131072, dim=4096, table="bf16", dtype="bf16", scale=64.0),
        # the table's gradient for a batch of 16384 tokens of a skewed distribution
        dict(name="embedding gradient", op="embedding_grad", n=1, length=16384, vocab=50021, dim=2048, dtype="bf16", scale=1.0),
        # eight replicas with a table each, contexts of five tokens for minibatches of 128, an odd width
        dict(name="embedding gradient replicas", op="embedding_grad", n=8, length=640, vocab=1000, dim=101, dtype="fp32", scale=1.0),
        # a hidden state with its residual
        dict(name="dropout hidden", op="dropout", rows=16384, cols=4096, pad=0, dtype="bf16", p=0.1, residual=True),
        # sixteen replicas' minibatch inputs (256 rows of 4096)
        dict(name="dropout inputs", op="dropout", rows=4096, cols=4096, pad=0, dtype="fp32", p=0.2, residual=False),
        # a ragged slice of a wider array
        dict(name="dropout ragged", op="dropout", rows=77, cols=1001, pad=22, dtype="fp16", p=0.5, residual=False),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    op = rng.choice(("logprobs", "logprobs_step", "embedding", "embedding_grad", "dropout"))
    dtype = rng.choice(tuple(TYPES))
    if op in ("logprobs", "logprobs_step"):
        rows = _log_int(rng, 1, 8192)
        most = int(math.exp(LOG2_COST) / rows / (BYTES[dtype] / 2))
        vocab = _log_int(rng, 50, max(51, min(131072, most)))
        case = dict(op=op, rows=rows, vocab=vocab, pad=rng.choice((0, 0, 3, 64)), dtype=dtype, scale=rng.choice((1.0, 1 / 0.7, 0.5)))
        if op == "logprobs":
            return dict(case, k=min(vocab, rng.randint(0, 32)), masked=rng.choice((0.0, 0.3)))
        return dict(case, entropy=rng.random() < 0.5)
    if op == "embedding":
        return dict(op=op, n=rng.choice((1, 1, 3)), length=_log_int(rng, 1, 5000), vocab=_log_int(rng, 100, 40000), dim=_log_int(rng, 33, 4096),
                    table=rng.choice(tuple(TYPES)), dtype=dtype, scale=rng.choice((1.0, 11.5)))
    if op == "embedding_grad":
        return dict(op=op, n=rng.choice((1, 1, 3)), length=_log_int(rng, 1, 16384), vocab=_log_int(rng, 100, 16000), dim=_log_int(rng, 33, 2048),
                    dtype=dtype, scale=rng.choice((1.0, 11.5)))
    return dict(op=op, rows=_log_int(rng, 1, 8192), cols=_log_int(rng, 33, 4096), pad=rng.choice((0, 0, 5, 32)), dtype=dtype,
                p=rng.choice((0.1, 0.25, 0.5)), residual=rng.random() < 0.5)


def _tokens(shape, vocab, gen):
    """Token numbers whose frequency falls as 1 / (rank + 1)."""
    u = torch.rand(shape, generator=gen, device="cuda", dtype=torch.float64)
    return (torch.exp(u * math.log(vocab + 1)) - 1).long().clamp_(0, vocab - 1).int()


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *shape, dtype=torch.float32: torch.randn(*shape, generator=gen, device="cuda", dtype=dtype)  # noqa: E731
    op, dtype = case["op"], TYPES[case["dtype"]]
    s = dict(case)
    if op in ("logprobs", "logprobs_step"):
        rows, vocab = case["rows"], case["vocab"]
        s["logits"] = normal(rows, vocab + case["pad"], dtype=dtype).mul_(2.5)[:, :vocab]
        s["tokens"] = _tokens((rows,), vocab, gen)
        if rows > 1:                              # a tenth of a batch's rows are padding: they have no token
            s["tokens"].masked_fill_(torch.rand(rows, generator=gen, device="cuda") < 0.1, -1)
        new = lambda *shape, dtype=torch.float32: torch.empty(*shape, device="cuda", dtype=dtype)  # noqa: E731
        s["logprob"], s["entropy_out"] = new(rows), new(rows)
        if op == "logprobs":
            if case["masked"]:
                s["logits"].masked_fill_(torch.rand(rows, vocab, generator=gen, device="cuda") < case["masked"], -math.inf)
            s["top_token"], s["top_logprob"] = new(rows, case["k"], dtype=torch.int32), new(rows, case["k"])
        else:
            s["d_logprob"] = -torch.rand(rows, generator=gen, device="cuda")          # a weighted sum of losses
            s["d_entropy"] = torch.full((rows,), -0.01, device="cuda") if case["entropy"] else None
            s["dlogits"] = new(rows, vocab, dtype=dtype)
    elif op == "embedding":
        n, T, V, D = (case[x] for x in ("n", "length", "vocab", "dim"))
        s["table_data"] = normal(n, V, D, dtype=TYPES[case["table"]]).mul_(0.02)
        s["tokens"] = _tokens((n, T), V, gen)
        s["out"] = torch.empty(n, T, D, device="cuda", dtype=dtype)
    elif op == "embedding_grad":
        n, T, V, D = (case[x] for x in ("n", "length", "vocab", "dim"))
        s["dout"] = normal(n, T, D, dtype=dtype)
        s["tokens"] = _tokens((n, T), V, gen)
        if T > 1:
            s["tokens"].masked_fill_(torch.rand(n, T, generator=gen, device="cuda") < 0.1, -1)
        s["dtable"] = torch.empty(n, V, D, device="cuda")
    else:
        rows, cols, pad = case["rows"], case["cols"], case["pad"]
        s["x"] = normal(rows, cols + pad, dtype=dtype)[:, :cols]
        s["residual_data"] = normal(rows, cols, dtype=dtype) if case["residual"] else None
        s["out"] = torch.empty(rows, cols, device="cuda", dtype=dtype)
        s["seed"], s["offset"] = 0x9E3779B97F4A7C15 ^ (seed * 0x10001), 7 + seed % 1000
    return s


# ---- the plain forms -----------------------------------------------------------------------------------------------------

def _log_softmax(s):
    """Shifted scaled logits d, their exponentials, the sums of those, log p; all in 32 bits."""
    x = s["logits"].float()
    d = (x - x.amax(1, keepdim=True)) * s["scale"]
    e = torch.exp(d)
    total = e.sum(1, keepdim=True)
    return x, e / total, d - torch.log(total)


def _entropy(p, logp):
    return -(p * torch.where(p > 0, logp, 0)).sum(1)


def _given(logp, tokens):
    has = tokens >= 0
    return torch.where(has, logp.gather(1, tokens.clamp(min=0).long()[:, None])[:, 0], 0), has


def plain_logprobs(s):
    x, p, logp = _log_softmax(s)
    given, _ = _given(logp, s["tokens"])
    # one 64-bit key orders the logits and, among equal ones, the lower token first
    bits = (x + 0.0).view(torch.int32).long()
    order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits)
    key = (order << 32) - torch.arange(x.shape[1], device=x.device)
    top = torch.topk(key, s["k"], dim=1).indices
    real = x.gather(1, top) > -math.inf
    return given, _entropy(p, logp), torch.where(real, top, -1).int(), torch.where(real, logp.gather(1, top), -math.inf)


def plain_logprobs_step(s):
    _, p, logp = _log_softmax(s)
    given, has = _given(logp, s["tokens"])
    entropy = _entropy(p, logp)
    g = torch.where(has, s["d_logprob"], 0)[:, None]
    d = -g * p
    d.scatter_add_(1, s["tokens"].clamp(min=0).long()[:, None], g)
    if s["d_entropy"] is not None:
        d -= s["d_entropy"][:, None] * p * (torch.where(p > 0, logp, 0) + entropy[:, None])
    return given, entropy, (d * s["scale"]).to(s["logits"].dtype)


def plain_embedding(s):
    n, T = s["tokens"].shape
    rows = s["table_data"][torch.arange(n, device="cuda")[:, None], s["tokens"].long()]
    return (rows.float() * s["scale"]).to(s["out"].dtype)


def plain_embedding_grad(s):
    n, T, D = s["dout"].shape
    V = s["vocab"]
    has = (s["tokens"] >= 0)[:, :, None]
    at = torch.arange(n, device="cuda")[:, None] * V + s["tokens"].clamp(min=0).long()
    sums = torch.zeros(n * V, D, device="cuda")
    sums.index_add_(0, at.flatten(), torch.where(has, s["dout"].float(), 0).flatten(0, 1))
    return (sums * s["scale"]).view(n, V, D)


def _philox_fields(groups, seed, offset):
    """Philox 4x32-10 (Salmon et al., "Parallel random numbers: as easy as 1, 2, 3", 2011) in 64-bit integers: the counter of a
    group of eight elements is (group, offset), the key is the seed; its four words give eight 16-bit fields."""
    low = 0xFFFFFFFF
    group = torch.arange(groups, device="cuda")
    c = [group & low, group >> 32, torch.full_like(group, offset & low), torch.full_like(group, offset >> 32)]
    k0, k1 = seed & low, seed >> 32
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [((b >> 32) & low) ^ c[1] ^ k0, b & low, ((a >> 32) & low) ^ c[3] ^ k1, a & low]
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    words = torch.stack(c, 1)
    return torch.stack((words & 0xFFFF, words >> 16), 2).flatten()


def plain_dropout(s):
    rows, cols = s["x"].shape
    threshold = math.floor(s["p"] * 65536 + 0.5)
    fields = _philox_fields(-(-rows * cols // 8), s["seed"], s["offset"])[:rows * cols].view(rows, cols)
    y = torch.where(fields >= threshold, s["x"].float() * (65536 / (65536 - threshold)), 0)
    if s["residual_data"] is not None:
        y = y + s["residual_data"].float()
    return y.to(s["x"].dtype)


def run(state):
    s = state
    if own:
        import paper_1707_00424_b200 as pb
        if s["op"] == "logprobs":
            return pb.token_logprobs(s["logits"], s["tokens"], k=s["k"], scale=s["scale"], logprob=s["logprob"], entropy=s["entropy_out"],
                                     top_token=s["top_token"], top_logprob=s["top_logprob"])
        if s["op"] == "logprobs_step":
            dlogits = pb.token_logprobs_grad(s["logits"], s["tokens"], s["d_logprob"], s["d_entropy"], scale=s["scale"], dlogits=s["dlogits"],
                                             logprob=s["logprob"], entropy=s["entropy_out"])
            return s["logprob"], s["entropy_out"], dlogits
        if s["op"] == "embedding":
            return pb.embedding(s["table_data"], s["tokens"], scale=s["scale"], out=s["out"])
        if s["op"] == "embedding_grad":
            return pb.embedding_grad(s["dout"], s["tokens"], s["vocab"], scale=s["scale"], dtable=s["dtable"])
        return pb.dropout(s["x"], s["p"], s["seed"], s["offset"], residual=s["residual_data"], out=s["out"])
    return {"logprobs": plain_logprobs, "logprobs_step": plain_logprobs_step, "embedding": plain_embedding,
            "embedding_grad": plain_embedding_grad, "dropout": plain_dropout}[s["op"]](s)


# ---- what a pass cannot do without ------------------------------------------------------------------------------------------

def _distinct(tokens, vocab):
    """Expected number of different tokens among `tokens` drawn as _tokens() draws them."""
    p = np.log1p(1 / np.arange(1, vocab + 1)) / math.log(vocab + 1)
    return float(np.sum(-np.expm1(tokens * np.log1p(-p))))


def work(case):
    op, size = case["op"], BYTES[case["dtype"]]
    if op in ("logprobs", "logprobs_step"):
        rows, elements = case["rows"], case["rows"] * case["vocab"]
        if op == "logprobs":
            return {"bytes": elements * size + rows * (12 + 8 * case["k"]), "flops": 5 * elements}
        return {"bytes": 2 * elements * size + rows * (20 if case["entropy"] else 16), "flops": 8 * elements}
    if op == "dropout":
        elements = case["rows"] * case["cols"]
        return {"bytes": elements * size * (3 if case["residual"] else 2), "flops": 2 * elements}
    n, T, V, D = (case[x] for x in ("n", "length", "vocab", "dim"))
    if op == "embedding":
        return {"bytes": n * (T * 4 + T * D * size + _distinct(T, V) * D * BYTES[case["table"]]), "flops": n * T * D}
    return {"bytes": n * (T * 4 + T * D * size + V * D * 4), "flops": n * (T + V) * D}


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------------------

def _exact_rows(z, tokens, k, d_logprob, d_entropy, scale):
    """Some rows of the log probabilities: z are scaled logits in 64 bits."""
    logp = z - torch.logsumexp(z, 1, keepdim=True)
    p = logp.exp()
    plogp = torch.special.xlogy(p, p)
    entropy = -plogp.sum(1)
    one = torch.zeros_like(p)
    real = torch.nonzero(tokens >= 0)[:, 0]
    one[real, tokens[real].long()] = 1
    given = torch.zeros_like(entropy)
    given[real] = logp[real, tokens[real].long()]
    if d_logprob is None:
        ranked = torch.sort(z, dim=1, descending=True, stable=True)
        top, values = ranked.indices[:, :k].int(), logp.gather(1, ranked.indices[:, :k])
        return given, entropy, top.masked_fill(values == -math.inf, -1), values
    g = d_logprob.double() * (tokens >= 0)
    grad = g[:, None] * (one - p)
    if d_entropy is not None:
        grad -= d_entropy.double()[:, None] * (plogp + p * entropy[:, None])
    return given, entropy, grad * scale


def _exact_fields(groups, seed, offset):
    """The generator once more, in unsigned 64-bit numpy integers on the host."""
    u, low = np.uint64, np.uint64(0xFFFFFFFF)
    i = np.arange(groups, dtype=u)
    x0, x1, x2, x3 = i & low, i >> u(32), np.full(groups, offset % 2**32, u), np.full(groups, offset // 2**32, u)
    for r in range(10):
        k0, k1 = u((seed % 2**32 + r * 0x9E3779B9) % 2**32), u((seed // 2**32 + r * 0xBB67AE85) % 2**32)
        m0, m1 = u(0xD2511F53) * x0, u(0xCD9E8D57) * x2
        x0, x1, x2, x3 = (m1 >> u(32)) ^ x1 ^ k0, m1 & low, (m0 >> u(32)) ^ x3 ^ k1, m0 & low
    return np.stack((x0, x1, x2, x3), 1).astype(np.uint32).view(np.uint16).reshape(-1)


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op in ("logprobs", "logprobs_step"):
        step = max(1, (1 << 26) // case["vocab"])
        parts = []
        for at in range(0, case["rows"], step):
            cut = slice(at, at + step)
            g, h = s.get("d_logprob"), s.get("d_entropy")
            parts.append(_exact_rows(s["logits"][cut].double() * case["scale"], s["tokens"][cut], case.get("k"),
                                     None if g is None else g[cut], None if h is None else h[cut], case["scale"]))
        return tuple(torch.cat(x) for x in zip(*parts))
    if op == "embedding":
        return torch.stack([t[i.long()].double() * case["scale"] for t, i in zip(s["table_data"], s["tokens"])])
    if op == "embedding_grad":
        n, T, V, D = (case[x] for x in ("n", "length", "vocab", "dim"))
        total = torch.zeros(n, V + 1, D, device="cuda", dtype=torch.float64)      # row V takes the positions without a token
        for t, i, d in zip(total, s["tokens"], s["dout"]):
            i = torch.where(i >= 0, i, V).long()
            order = torch.sort(i, stable=True).indices
            t.index_put_((i[order],), d.double()[order], accumulate=True)
        return total[:, :V] * case["scale"]
    rows, cols = s["x"].shape
    threshold = int(round(case["p"] * 65536))
    kept = _exact_fields(-(-rows * cols // 8), s["seed"], s["offset"])[:rows * cols] >= threshold
    keep = torch.from_numpy(kept).cuda().view(rows, cols)
    y = s["x"].double().masked_fill(~keep, 0) * 65536 / (65536 - threshold)
    return y + s["residual_data"].double() if case["residual"] else y
