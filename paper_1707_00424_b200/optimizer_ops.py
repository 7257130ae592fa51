"""Operators of libparle.so over lists of tensors: the norm of gradients, and AdamW with moments in 32 or in 8 bits.

As the token operators (token_ops.py): tensors are checked and one call of the C ABI is made in the module _token_ops, on `stream` or the
current stream of the first tensor's device; outside autograd; tensors written count as modified in place (a parameter that requires a
gradient is stepped all the same).  Lists are lists or tuples; their tensors are contiguous, of one type a list, on one device."""
from __future__ import annotations

from . import token_ops

BLOCK = 256


def grad_norm(grads, *, out=None, workspace=None, stream=None):
    """The norm of all elements of the tensors in `grads`, a tensor of one fp32 number (parle_grad_norm).  workspace: scratch, allocated
    when not given; 8 bytes for each begun 16376 elements of each tensor, and 128 bytes more, are enough wherever the tensors begin."""
    return (token_ops._MODULE or token_ops.load()).grad_norm(grads, out, workspace, stream)


def adamw_state(params, bits: int = 32):
    """(exp_avg, exp_avg_sq, exp_avg_scales, exp_avg_sq_scales) of no steps for adamw(): lists of zeros like params.  bits 32: fp32
    moments, the last two are None.  bits 8: codes of type float8_e4m3fn, and an fp32 scale for each 256 elements."""
    import torch
    if bits not in (8, 32):
        raise ValueError("moments have 8 or 32 bits")
    kind = torch.float32 if bits == 32 else torch.float8_e4m3fn
    moments = [[torch.zeros(p.shape, dtype=kind, device=p.device) for p in params] for _ in range(2)]
    if bits == 32:
        return (*moments, None, None)
    return (*moments, *([torch.zeros(-(-p.numel() // BLOCK), dtype=torch.float32, device=p.device) for p in params] for _ in range(2)))


def adamw(params, grads, exp_avg, exp_avg_sq, *, step: int, lr: float, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay: float = 0.01,
          exp_avg_scales=None, exp_avg_sq_scales=None, copies=None, grad_scale: float = 1.0, norm=None, max_norm=None, step_dev=None, lr_dev=None,
          flags=None, stream=None) -> None:
    """One AdamW step of all params from grads, in place (parle_adamw has the definition).  exp_avg, exp_avg_sq: the moments, all fp32, or
    all float8_e4m3fn with the scales of their blocks, as adamw_state() makes them.  step: 1 in the first step.  copies: tensors of bf16 or
    fp16 that receive the new fp32 params.  norm: grad_norm(grads), on the device; gradients are then clipped to max_norm, and a norm that
    is no finite number skips the step (parameters, moments and copies keep their values).  step_dev (int64) and lr_dev (fp32), tensors of
    one element, are added to step and multiplied with lr when the kernel runs.  flags (int32, one element): FLAG_NONFINITE is set where a
    step was skipped or gave a parameter that is no finite number."""
    (token_ops._MODULE or token_ops.load()).adamw(params, grads, exp_avg, exp_avg_sq, exp_avg_scales, exp_avg_sq_scales, copies, step, lr, *betas, eps,
                                                  weight_decay, grad_scale, norm, max_norm, step_dev, lr_dev, flags, stream)
