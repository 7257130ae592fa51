"""Cases of the operators that end a training step and a decoding step: AdamW over many tensors (moments in 32 or in 8 bits), the
norm of a list of gradients, and sampling of tokens with temperature, top-k, top-p and min-p.

`listed()` and `draw()` give the cases, `prepare()` a case's inputs on the GPU, `run()` one pass through the operator: in elementary
torch operations, or, where `own` is true, through the library's entry points.  `exact()` has the definitions in 64 bits."""
import math
import random

import numpy as np
import torch

own = False
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
BYTES = {"fp32": 4, "bf16": 2, "fp16": 2}
BLOCK = 256                                      # elements that share a scale where moments have 8 bits
LARGEST = 448.0                                  # of the 8-bit type (e4m3)
SMALLEST = 2.0 ** -9
NOTHING = 2.0 ** -100                            # a block whose values all lie below this holds zeros
WEYL_I, WEYL_T, WEYL = 12664745, 9560335, 1 << 24          # the threshold of element i at step t: (i WEYL_I + t WEYL_T) mod 2^24
BETA1, BETA2, EPS, DECAY, RATE = 0.9, 0.999, 1e-8, 0.1, 1e-3
MOST_LOGITS = 512 * 131072                       # no drawn case has more

WIDE = "4096-8192-8192-8192-8192-1000"


def listed():
    return [
        # the smallest model, three replicas' layers as tensors of their own: latency alone
        dict(name="adamw small model", op="adamw", layers="64-32-10", n=3, align=32, param="fp32", grad="fp32", copy="", bits=32, clip=False),
        # one replica of the widest model in fp32
        dict(name="adamw wide model", op="adamw", layers=WIDE, n=1, align=32, param="fp32", grad="fp32", copy="", bits=32, clip=False),
        # many tensors of all sizes, back to back in memory; gradients of 16 bits, clipped by their norm; a 16-bit copy of each weight
        dict(name="adamw many tensors", op="adamw", count=300, low=1, high=60000, align=1, param="fp32", grad="bf16", copy="bf16", bits=32, clip=True),
        # a table of tokens in 16 bits with moments in 8
        dict(name="adamw 8 bits table", op="adamw", count=1, low=50021 * 2048, high=50021 * 2048, align=256, param="bf16", grad="bf16", copy="", bits=8, clip=False),
        # eight replicas of a model of middling width, fp32 weights with moments in 8 bits, clipped
        dict(name="adamw 8 bits replicas", op="adamw", layers="784-1024-1024-10", n=8, align=256, param="fp32", grad="fp32", copy="", bits=8, clip=True),
        # the norm of one replica's gradient of the widest model
        dict(name="norm wide model", op="norm", layers=WIDE, n=1, align=32, grad="fp32"),
        # the norm of many tensors of all sizes, back to back
        dict(name="norm many tensors", op="norm", count=300, low=1, high=60000, align=1, grad="bf16"),
        # one sequence's next token
        dict(name="sample next token", op="sample", rows=1, vocab=131072, pad=0, dtype="bf16", scale=1 / 0.7, k=50, p=0.9, min_p=0.0, peaked=True, masked=0.0, per_row=False),
        # a batch of requests, each with parameters of its own, some tokens banned, odd vocabulary
        dict(name="sample requests", op="sample", rows=64, vocab=50021, pad=0, dtype="fp32", scale=1.0, k=40, p=0.95, min_p=0.05, peaked=True, masked=0.05, per_row=True),
        # many continuations of one prompt from the whole vocabulary
        dict(name="sample whole vocabulary", op="sample", rows=256, vocab=131072, pad=0, dtype="bf16", scale=1.0, k=0, p=1.0, min_p=0.0, peaked=True, masked=0.0, per_row=False),
        # the same from the tokens that make up 95% of an undecided model's distribution (thousands of them)
        dict(name="sample undecided", op="sample", rows=256, vocab=131072, pad=0, dtype="bf16", scale=1.0, k=0, p=0.95, min_p=0.0, peaked=False, masked=0.0, per_row=False),
        # a large batch with top-k, top-p and min-p together
        dict(name="sample large batch", op="sample", rows=512, vocab=131072, pad=0, dtype="bf16", scale=1 / 0.8, k=200, p=0.95, min_p=0.02, peaked=True, masked=0.0, per_row=False),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    op = rng.choice(("adamw", "adamw", "norm", "sample", "sample"))
    types = tuple(TYPES)
    if op == "sample":
        rows, dtype = _log_int(rng, 1, 4096), rng.choice(types)
        vocab = _log_int(rng, 50, max(51, min(131072, MOST_LOGITS // rows * 2 // BYTES[dtype])))
        return dict(op=op, rows=rows, vocab=vocab, pad=rng.choice((0, 0, 3, 64)), dtype=dtype, scale=rng.choice((1.0, 1 / 0.7, 0.5)),
                    k=rng.choice((0, 0, 1, _log_int(rng, 2, vocab))), p=rng.choice((1.0, 0.5, 0.9, 0.99)), min_p=rng.choice((0.0, 0.0, 0.01, 0.1)),
                    peaked=rng.random() < 0.5, masked=rng.choice((0.0, 0.3)), per_row=rng.random() < 0.3)
    many = rng.random() < 0.5
    count = _log_int(rng, 20, 600) if many else rng.randint(1, 4)
    high = _log_int(rng, 50, 100000) if many else _log_int(rng, 300, 20_000_000)
    case = dict(op=op, count=count, low=1 if many else max(1, high // 3), high=high, align=rng.choice((1, 32)), grad=rng.choice(types))
    if op == "norm":
        return case
    bits, param = rng.choice((32, 8)), rng.choice(types)
    return dict(case, align=256 if bits == 8 else case["align"], param=param, copy=rng.choice(("", "bf16", "fp16")) if param == "fp32" else "",
                bits=bits, clip=rng.random() < 0.5)


def _sizes(case):
    """Elements of each tensor."""
    if "layers" in case:
        dims = [int(d) for d in case["layers"].split("-")]
        return [x for a, b in zip(dims, dims[1:]) for x in (a * b, b)] * case["n"]
    r = random.Random(case["count"] * 1000003 + case["high"])
    return [_log_int(r, case["low"], case["high"]) for _ in range(case["count"])]


def _places(case):
    """Where each tensor begins in a vector that holds them all, and that vector's length."""
    at, total, a = [], 0, case["align"]
    for n in _sizes(case):
        at.append(total)
        total += -(-n // a) * a
    return at, total


def _quantise(x, threshold, root):
    """x [blocks, BLOCK] in 8 bits: codes and the scale of each block.  A value between two codes goes to the upper one where the rest is at
    least 1 - threshold / 2^24, a threshold that runs through all numbers from step to step: a moment that moves by less than half of
    a code's spacing a step moves all the same.  Of a root, what is above zero stays above zero."""
    top = x.abs().amax(1, keepdim=True)
    none = top < NOTHING
    y = (x * torch.where(none, 0, LARGEST / top)).clamp(-LARGEST, LARGEST).double()
    spacing = torch.exp2(torch.frexp(y.abs().clamp(min=2.0 ** -6)).exponent.double() - 4)
    code = torch.floor(y.abs() / spacing + threshold / WEYL) * spacing * torch.sign(y)
    if root:
        code = torch.where((x > 0) & ~none, code.clamp(min=SMALLEST), 0)
    return code.to(torch.float8_e4m3fn), torch.where(none, 0, top / LARGEST)[:, 0]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *shape, dtype=torch.float32: torch.randn(*shape, generator=gen, device="cuda", dtype=dtype)  # noqa: E731
    uniform = lambda *shape: torch.rand(*shape, generator=gen, device="cuda")  # noqa: E731
    s = dict(case)
    if case["op"] == "sample":
        rows, vocab = case["rows"], case["vocab"]
        logits = normal(rows, vocab + case["pad"], dtype=TYPES[case["dtype"]]).mul_(2.5)[:, :vocab]
        if case["peaked"]:                        # a few tokens stand out, as after most prompts
            part = vocab // 32
            liked = torch.randint(part, (rows, 32), generator=gen, device="cuda") + part * torch.arange(32, device="cuda")
            logits.scatter_(1, liked, (8 + 8 * uniform(rows, 32)).to(logits.dtype))
        if case["masked"]:
            logits.masked_fill_(uniform(rows, vocab) < case["masked"], -math.inf)
        s["logits"], s["u"] = logits, uniform(rows)
        if case["per_row"]:                       # each row has its own parameters, some of them none
            some = lambda v, none: torch.where(uniform(rows) < 0.3, torch.full((rows,), none, device="cuda"), v)  # noqa: E731
            s["scale"] = case["scale"] * (0.8 + uniform(rows))
            s["k"] = some((1 + uniform(rows) * 2 * case["k"]).floor(), 0.0).int()
            s["p"] = some(case["p"] * uniform(rows).sqrt(), 1.0)
            s["min_p"] = some(case["min_p"] * 2 * uniform(rows), 0.0)
        s["token"], s["logprob"], s["kept"] = (torch.empty(rows, device="cuda", dtype=t) for t in (torch.int32, torch.float32, torch.int32))
        return s
    at, total = _places(case)
    sizes = _sizes(case)
    within = torch.zeros(total, dtype=torch.bool, device="cuda")
    inner = lambda v: [v[a:a + n] for a, n in zip(at, sizes)]  # noqa: E731
    torch._foreach_add_(inner(within.view(torch.uint8)), 1)
    s["norm"] = torch.empty((), device="cuda")
    s["grad_data"] = normal(total, dtype=TYPES[case["grad"]]).mul_(0.01).mul_(within)
    s["grads"] = inner(s["grad_data"])
    if case["op"] == "norm":
        return s
    s["step"] = 3 + seed % 1000
    s["max_norm"] = 0.5 * 0.01 * math.sqrt(sum(sizes))       # about half of the norm
    s["param_data"] = normal(total, dtype=TYPES[case["param"]]).mul_(0.05).mul_(within)
    s["params"] = inner(s["param_data"])
    s["copy_data"] = torch.zeros(total, device="cuda", dtype=TYPES[case["copy"]]) if case["copy"] else None
    s["copies"] = inner(s["copy_data"]) if case["copy"] else None
    m, r = normal(total).mul_(0.003).mul_(within), uniform(total).mul_(0.01).add_(0.002).mul_(within)
    if case["bits"] == 32:
        s["exp_avg_data"], s["exp_avg_sq_data"] = m, r.square_()
        s["exp_avg_scales"] = s["exp_avg_sq_scales"] = None
    else:
        # the number that each block's first element has within its tensor
        s["first"] = torch.cat([torch.arange(0, n, BLOCK) for n in sizes]).cuda()[:, None]
        for key, x, root in (("exp_avg", m, False), ("exp_avg_sq", r, True)):
            codes, scales = _quantise(x.view(-1, BLOCK), WEYL / 2, root)
            s[key + "_data"], s[key + "_scale_data"] = codes.view(-1), scales
            s[key + "_scales"] = [scales[a // BLOCK:(a + n + BLOCK - 1) // BLOCK] for a, n in zip(at, sizes)]
    s["exp_avg"], s["exp_avg_sq"] = inner(s["exp_avg_data"]), inner(s["exp_avg_sq_data"])
    return s


# ---- the plain forms -----------------------------------------------------------------------------------------------------

def plain_norm(s):
    return s["grad_data"].double().square().sum().sqrt().float()


def plain_adamw(s):
    """The elements between the tensors are zeros, which stay zeros: one pass over the vectors is one over all tensors."""
    g = s["grad_data"].float()
    if s["clip"]:
        s["norm"].copy_(plain_norm(s))
        g = g * (s["max_norm"] / s["norm"]).clamp(max=1.0)
    if s["bits"] == 32:
        m, v = s["exp_avg_data"], s["exp_avg_sq_data"]
    else:
        m = s["exp_avg_data"].float().view(-1, BLOCK) * s["exp_avg_scale_data"][:, None]
        v = (s["exp_avg_sq_data"].float().view(-1, BLOCK) * s["exp_avg_sq_scale_data"][:, None]).square()
        m, v = m.flatten(), v.flatten()
    m = m * BETA1 + g * (1 - BETA1)
    v = v * BETA2 + g * g * (1 - BETA2)
    r = torch.sqrt(v)
    p = s["param_data"].float()
    p = p * (1 - RATE * DECAY) - RATE / (1 - BETA1 ** s["step"]) * m / (r / math.sqrt(1 - BETA2 ** s["step"]) + EPS)
    s["param_data"].copy_(p)
    if s["copy_data"] is not None:
        s["copy_data"].copy_(p)
    if s["bits"] == 32:
        s["exp_avg_data"].copy_(m)
        s["exp_avg_sq_data"].copy_(v)
    else:
        threshold = ((s["first"] + torch.arange(BLOCK, device="cuda")) * WEYL_I + s["step"] * WEYL_T) % WEYL
        codes, scales = _quantise(m.view(-1, BLOCK), threshold, False)
        roots, root_scales = _quantise(r.view(-1, BLOCK), WEYL - 1 - threshold, True)
        s["exp_avg_data"].copy_(codes.view(-1))
        s["exp_avg_scale_data"].copy_(scales)
        s["exp_avg_sq_data"].copy_(roots.view(-1))
        s["exp_avg_sq_scale_data"].copy_(root_scales)
    return _updated(s)


def _updated(s):
    out = dict(param=s["param_data"], exp_avg=s["exp_avg_data"], exp_avg_sq=s["exp_avg_sq_data"])
    if s["copy_data"] is not None:
        out["copy"] = s["copy_data"]
    if s["clip"]:
        out["norm"] = s["norm"]
    if s["bits"] == 8:
        out["exp_avg_scale"], out["exp_avg_sq_scale"] = s["exp_avg_scale_data"], s["exp_avg_sq_scale_data"]
    return out


def _column(v, like):
    """A parameter as a column of 64-bit numbers, rounded to 32 bits first."""
    return torch.as_tensor(v, device=like.device, dtype=torch.float32).double().expand(like.shape[0])[:, None]


def plain_sample(s):
    """In 64 bits: a cumulative sum is compared with a number next to it."""
    x = s["logits"].double()
    scale, p, min_p = (_column(s[key], x) for key in ("scale", "p", "min_p"))
    k = torch.as_tensor(s["k"], device="cuda").long().expand(x.shape[0])[:, None]
    ranked, order = torch.sort(s["logits"], dim=1, descending=True, stable=True)
    ranked = ranked.double()
    best = ranked[:, :1]
    keep = (ranked > -math.inf) & ((k <= 0) | (torch.arange(x.shape[1], device="cuda") < k))
    sums = torch.cumsum(torch.exp((ranked - best) * scale) * keep, 1)
    before = torch.nn.functional.pad(sums[:, :-1], (1, 0))
    keep &= ((p >= 1) | (before < p * sums[:, -1:])) & (ranked >= best + torch.log(min_p) / scale)
    kept = torch.zeros_like(keep).scatter_(1, order, keep)
    w = torch.exp((x - best) * scale) * kept
    sums = torch.cumsum(w, 1)
    token = (sums > s["u"].double()[:, None] * sums[:, -1:]).int().argmax(1, keepdim=True)
    logprob = torch.log(w.gather(1, token) / sums[:, -1:])
    return token[:, 0].int(), logprob[:, 0].float(), kept.sum(1).int()


def run(state):
    s = state
    if own:
        import paper_1707_00424_b200 as pb
        if s["op"] == "sample":
            return pb.sample_tokens(s["logits"], s["u"], scale=s["scale"], top_k=s["k"], top_p=s["p"], min_p=s["min_p"], token=s["token"],
                                    logprob=s["logprob"], kept=s["kept"])
        if s["op"] == "norm":
            return pb.grad_norm(s["grads"], out=s["norm"])
        if s["clip"]:
            pb.grad_norm(s["grads"], out=s["norm"])
        pb.adamw(s["params"], s["grads"], s["exp_avg"], s["exp_avg_sq"], step=s["step"], lr=RATE, betas=(BETA1, BETA2), eps=EPS, weight_decay=DECAY,
                 exp_avg_scales=s["exp_avg_scales"], exp_avg_sq_scales=s["exp_avg_sq_scales"], copies=s["copies"],
                 norm=s["norm"] if s["clip"] else None, max_norm=s["max_norm"] if s["clip"] else None)
        return _updated(s)
    return {"sample": plain_sample, "norm": plain_norm, "adamw": plain_adamw}[s["op"]](s)


# ---- what a pass cannot do without ------------------------------------------------------------------------------------------

def work(case):
    if case["op"] == "sample":
        elements = case["rows"] * case["vocab"]
        return {"bytes": elements * BYTES[case["dtype"]] + case["rows"] * (32 if case["per_row"] else 16), "flops": 4 * elements}
    elements = sum(_sizes(case))
    size = BYTES[case["grad"]]
    if case["op"] == "norm":
        return {"bytes": elements * size + 4, "flops": 2 * elements}
    size += 2 * BYTES[case["param"]] + (BYTES[case["copy"]] if case["copy"] else 0)
    size += 16 if case["bits"] == 32 else 4 + 16 / BLOCK
    return {"bytes": elements * size, "flops": (15 if case["bits"] == 32 else 25) * elements}


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------------------

def _exact_block_codes(x, part, root):
    """Of the 8-bit type's two numbers around each value (2^(e - 3) apart from 2^e to 2^(e + 1), 2^-9 below 2^-6) the upper one where the value
    and `part` of their distance reach it."""
    top = x.abs().max(dim=1, keepdim=True).values
    y = x.abs() / torch.where(top < NOTHING, math.inf, top) * LARGEST
    apart = 2.0 ** torch.floor(torch.log2(torch.maximum(y, torch.full_like(y, 2.0 ** -6)))) / 8
    lower = torch.floor(y / apart) * apart
    code = lower + apart * (y - lower + part * apart >= apart)
    if root:
        code = torch.where((y > 0) & (code == 0), SMALLEST, code)
    return code * torch.sign(x), torch.where(top < NOTHING, 0, top)[:, 0] / LARGEST


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "sample":
        rows, vocab = case["rows"], case["vocab"]
        if rows * (2e-4 + vocab * 2.5e-7) > 18:
            return None
        col = lambda key: np.broadcast_to(np.asarray(torch.as_tensor(s[key]).cpu(), np.float64), (rows,))  # noqa: E731
        f32 = lambda v: float(np.float32(v))  # noqa: E731
        logits, u = s["logits"].float().cpu().numpy(), s["u"].cpu().numpy().astype(np.float64)
        found, logprobs, counts = [], [], []
        for x, z, scale, k, p, low in zip(logits, u, col("scale"), col("k"), col("p"), col("min_p")):
            scale, p, low = f32(scale), f32(p), f32(low)
            x = x.astype(np.float64)
            rank = np.argsort(-x, kind="stable")[:int(np.sum(x > -np.inf))]
            rank = rank[:int(k)] if k > 0 else rank
            w = np.exp(scale * (x[rank] - x[rank[0]]))
            if p < 1:
                some = 1 + int(np.searchsorted(np.cumsum(w), p * np.sum(w), side="left"))
                some = min(some, len(rank))
            else:
                some = len(rank)
            if low > 0:
                some = min(some, int(np.sum(scale * (x[rank] - x[rank[0]]) >= math.log(low))))
            chosen = np.sort(rank[:some])
            w = np.exp(scale * (x[chosen] - x[rank[0]]))
            c = np.cumsum(w)
            i = min(int(np.searchsorted(c, z * c[-1], side="right")), some - 1)
            found.append(chosen[i])
            logprobs.append(scale * (x[chosen[i]] - x[rank[0]]) - math.log(c[-1]))
            counts.append(some)
        return torch.tensor(found, dtype=torch.int32), torch.tensor(logprobs, dtype=torch.float64), torch.tensor(counts, dtype=torch.int32)
    g = s["grad_data"].double()
    norm = torch.linalg.vector_norm(g)
    if case["op"] == "norm":
        return norm
    if case["clip"]:
        g = g * min(1.0, s["max_norm"] / float(norm))
    m, v = s["exp_avg_data"].double(), s["exp_avg_sq_data"].double()
    if case["bits"] == 8:
        m = m * s["exp_avg_scale_data"].double().repeat_interleave(BLOCK)
        v = (v * s["exp_avg_sq_scale_data"].double().repeat_interleave(BLOCK)) ** 2
    m, v = torch.lerp(g, m, BETA1), torch.lerp(g * g, v, BETA2)
    t = s["step"]
    p = s["param_data"].double()
    p = p - RATE * (DECAY * p + m / -math.expm1(t * math.log(BETA1)) / (torch.sqrt(v / -math.expm1(t * math.log(BETA2))) + EPS))
    out = dict(param=p, exp_avg=m, exp_avg_sq=v)
    if case["copy"]:
        out["copy"] = p
    if case["clip"]:
        out["norm"] = norm
    if case["bits"] == 8:
        number = torch.cat([torch.arange(-(-n // BLOCK) * BLOCK) for n in _sizes(case)]).cuda().view(-1, BLOCK)
        part = (number * WEYL_I + t * WEYL_T).remainder(WEYL)
        m, out["exp_avg_scale"] = _exact_block_codes(m.view(-1, BLOCK), part.double() / WEYL, False)
        r, out["exp_avg_sq_scale"] = _exact_block_codes(v.sqrt().view(-1, BLOCK), (WEYL - 1 - part).double() / WEYL, True)
        out["exp_avg"], out["exp_avg_sq"] = m.view(-1), r.view(-1)
    return out
