"""What the operators over lists and the sampling of tokens refuse, on the CPU: every call here returns before it touches the device."""
import ctypes as C
import math

import pytest
import torch

import paper_1707_00424_b200 as pb
from paper_1707_00424_b200.binding import AdamwStep, AdamwTensor, GradTensor, Sampling

EINVAL, EALIGN, EWORKSPACE, ETOOBIG = -1, -3, -6, -8
P = 1 << 20                                               # an aligned address that is never read
F32, BF16, F16, NO_COPY = 0, 1, 2, -1


def norm(tensors=((P, 100),), count=None, dtype=F32, out=2 * P, workspace=3 * P, nbytes=1 << 20):
    arr = (GradTensor * max(1, len(tensors)))(*tensors)
    return pb.lib().parle_grad_norm(arr if tensors else None, len(tensors) if count is None else count, dtype, out, workspace, nbytes, None)


def adamw(size=100, second=None, count=None, param_dtype=F32, grad_dtype=F32, copy_dtype=NO_COPY, bits=32, flags=None, no_step=False, **kw):
    arrays = dict(param=P, grad=2 * P, exp_avg=3 * P, exp_avg_sq=4 * P, exp_avg_scale=5 * P, exp_avg_sq_scale=6 * P, copy=7 * P)
    h = dict(lr=0.1, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.1, grad_scale=1.0, max_norm=math.inf, step=1, norm=None, lr_dev=None, step_dev=None)
    for k, v in kw.items():
        (arrays if k in arrays else h)[k] = v
    tensors = [AdamwTensor(size=size, **arrays)]
    if second is not None:
        tensors.append(AdamwTensor(size=10, **{**{k: v + (P >> 1) for k, v in arrays.items()}, **second}))
    arr = (AdamwTensor * len(tensors))(*tensors)
    step = AdamwStep(**h)
    return pb.lib().parle_adamw(arr, len(tensors) if count is None else count, param_dtype, grad_dtype, copy_dtype, bits, None if no_step else C.byref(step), flags, None)


def sample(logits=P, dtype=F32, rows=2, vocab=8, ld=8, u=2 * P, token=3 * P, logprob=None, kept=None, flags=None, no_sampling=False, **kw):
    h = Sampling(**{**dict(scale=1.0, top_p=1.0, min_p=0.0, top_k=0, scales=None, top_ps=None, min_ps=None, top_ks=None), **kw})
    return pb.lib().parle_sample_tokens(logits, dtype, rows, vocab, ld, u, None if no_sampling else C.byref(h), token, logprob, kept, flags, None)


@pytest.mark.parametrize("call, kw, code", [
    (norm, dict(count=-1), EINVAL), (norm, dict(tensors=(), count=1), EINVAL), (norm, dict(dtype=3), EINVAL), (norm, dict(out=None), EINVAL),
    (norm, dict(tensors=((P, -1),)), EINVAL), (norm, dict(tensors=((None, 5),)), EINVAL), (norm, dict(tensors=((P, 5), (P + 2, 5))), EALIGN),
    (norm, dict(tensors=((P + 1, 5),), dtype=BF16), EALIGN), (norm, dict(out=P + 2), EALIGN), (norm, dict(workspace=None), EINVAL),
    (norm, dict(workspace=P + 64), EALIGN), (norm, dict(nbytes=7), EWORKSPACE), (norm, dict(tensors=((P, 1 << 30),), nbytes=8 * 65535), EWORKSPACE),
    (norm, dict(tensors=((P, (1 << 40) + 1),)), ETOOBIG),
    (adamw, dict(count=-1), EINVAL), (adamw, dict(no_step=True), EINVAL), (adamw, dict(param_dtype=3), EINVAL), (adamw, dict(grad_dtype=-1), EINVAL),
    (adamw, dict(bits=16), EINVAL), (adamw, dict(copy_dtype=F32), EINVAL), (adamw, dict(copy_dtype=BF16, param_dtype=BF16), EINVAL), (adamw, dict(copy_dtype=7), EINVAL),
    (adamw, dict(size=-1), EINVAL), (adamw, dict(size=(1 << 40) + 1), ETOOBIG),
    *((adamw, {k: None}, EINVAL) for k in ("param", "grad", "exp_avg", "exp_avg_sq")), (adamw, dict(copy=None, copy_dtype=F16), EINVAL),
    (adamw, dict(exp_avg_scale=None, bits=8), EINVAL), (adamw, dict(exp_avg_sq_scale=None, bits=8), EINVAL),
    *((adamw, {k: P + 9 * P + 2}, EALIGN) for k in ("param", "grad", "exp_avg", "exp_avg_sq")), (adamw, dict(copy=P + 1, copy_dtype=F16), EALIGN),
    (adamw, dict(exp_avg_scale=5 * P + 2, bits=8), EALIGN), (adamw, dict(param=P + 1, param_dtype=BF16), EALIGN), (adamw, dict(flags=P + 2), EALIGN),
    (adamw, dict(lr=-0.1), EINVAL), (adamw, dict(lr=math.nan), EINVAL), (adamw, dict(lr=math.inf), EINVAL), (adamw, dict(lr=1e39), EINVAL),
    (adamw, dict(beta1=1.0), EINVAL), (adamw, dict(beta1=-0.1), EINVAL), (adamw, dict(beta2=1.0), EINVAL), (adamw, dict(beta2=math.nan), EINVAL),
    (adamw, dict(eps=0.0), EINVAL), (adamw, dict(eps=1.1), EINVAL), (adamw, dict(eps=math.nan), EINVAL), (adamw, dict(weight_decay=-0.1), EINVAL),
    (adamw, dict(weight_decay=math.inf), EINVAL), (adamw, dict(grad_scale=0.0), EINVAL), (adamw, dict(grad_scale=math.inf), EINVAL), (adamw, dict(grad_scale=1e-60), EINVAL),
    (adamw, dict(max_norm=0.0, norm=P), EINVAL), (adamw, dict(max_norm=math.nan, norm=P), EINVAL), (adamw, dict(max_norm=1e-60, norm=P), EINVAL), (adamw, dict(max_norm=1.0), EINVAL),
    (adamw, dict(step=0), EINVAL), (adamw, dict(step=-1, step_dev=P), EINVAL), (adamw, dict(norm=P + 1), EALIGN), (adamw, dict(lr_dev=P + 2), EALIGN), (adamw, dict(step_dev=P + 4), EALIGN),
    (adamw, dict(second=dict(param=P)), EINVAL), (adamw, dict(second=dict(exp_avg=3 * P)), EINVAL), (adamw, dict(second=dict(exp_avg_sq=P)), EINVAL), (adamw, dict(exp_avg_sq=3 * P), EINVAL),
    (adamw, dict(second=dict(copy=7 * P), copy_dtype=BF16), EINVAL), (adamw, dict(second=dict(exp_avg_scale=5 * P), bits=8), EINVAL), (adamw, dict(exp_avg_sq_scale=5 * P, bits=8), EINVAL),
    (sample, dict(logits=None), EINVAL), (sample, dict(dtype=3), EINVAL), (sample, dict(rows=-1), EINVAL), (sample, dict(vocab=0), EINVAL), (sample, dict(ld=-1), EINVAL),
    (sample, dict(u=None), EINVAL), (sample, dict(token=None), EINVAL), (sample, dict(no_sampling=True), EINVAL), (sample, dict(scale=0.0), EINVAL), (sample, dict(scale=9e-7), EINVAL),
    (sample, dict(scale=1.1e6), EINVAL), (sample, dict(scale=math.nan), EINVAL), (sample, dict(top_k=-1), EINVAL), (sample, dict(top_p=-0.1), EINVAL), (sample, dict(top_p=1.01), EINVAL),
    (sample, dict(top_p=math.nan), EINVAL), (sample, dict(min_p=-0.1), EINVAL), (sample, dict(min_p=1.01), EINVAL), (sample, dict(min_p=math.nan), EINVAL),
    (sample, dict(rows=(1 << 27) + 1), ETOOBIG), (sample, dict(vocab=(1 << 30) + 1), ETOOBIG), (sample, dict(logits=P + 2), EALIGN), (sample, dict(logits=P + 1, dtype=F16), EALIGN),
    *((sample, {k: P + 2}, EALIGN) for k in ("u", "token", "logprob", "kept", "flags", "scales", "top_ps", "min_ps", "top_ks")),
])
def test_the_c_entry_points_refuse(call, kw, code):
    assert call(**kw) == code


def test_nothing_to_do_is_no_error():
    assert adamw(size=0) == 0 and adamw(size=0, param=None, grad=None, exp_avg=None, exp_avg_sq=None) == 0 and adamw(count=0) == 0
    assert sample(rows=0) == 0 and sample(rows=0, logits=None, u=None, token=None) == 0


def test_workspace_of_the_norm():
    size = lambda *n: pb.lib().parle_grad_norm_workspace_bytes((GradTensor * len(n))(*((P, k) for k in n)), len(n))      # noqa: E731
    assert size(0) == 0 and size(5, -1) == 0 and size((1 << 40) + 1) == 0 and pb.lib().parle_grad_norm_workspace_bytes(None, 3) == 0
    assert size(1) == 128 and size(1 << 30) >= 8 * 65536 and size(*[1] * 1000) >= 8000 and size(1000) % 128 == 0


def test_a_long_list_with_the_same_array_at_both_ends_is_refused():
    n = 50000
    arr = (AdamwTensor * n)(*(AdamwTensor(*((k * n + i + 1) * 64 for k in range(7)), 1) for i in range(n)))
    arr[n - 1].exp_avg_sq = arr[0].param
    step = AdamwStep(0.1, 0.9, 0.99, 1e-8, 0.1, 1.0, math.inf, 1, None, None, None)
    assert pb.lib().parle_adamw(arr, n, F32, F32, NO_COPY, 32, C.byref(step), None, None) == EINVAL


def test_the_functions_refuse_tensors_that_are_not_on_a_gpu():
    x = torch.zeros(2, 8)
    for call in (lambda: pb.grad_norm([x]), lambda: pb.adamw([x], [x], [x], [x], step=1, lr=0.1), lambda: pb.sample_tokens(x, torch.zeros(2))):
        with pytest.raises(pb.ParleError) as e:
            call()
        assert e.value.code == EINVAL and "CUDA device" in str(e.value)
    with pytest.raises(ValueError):
        pb.adamw_state([x], 16)


def test_zero_states():
    p = [torch.zeros(3, 100), torch.zeros(256), torch.zeros(())]
    m, v, ms, vs = pb.adamw_state(p, 8)
    assert [t.shape for t in m] == [t.shape for t in p] == [t.shape for t in v] and m[0].dtype == torch.float8_e4m3fn
    assert [t.numel() for t in ms] == [2, 1, 1] == [t.numel() for t in vs]
    assert pb.adamw_state(p)[2:] == (None, None) and pb.adamw_state(p)[0][0].dtype == torch.float32
