"""Arrays of an AdamW step that are read and written at once, refused on the CPU: every call here returns before it touches the device."""
import ctypes as C
import math

import pytest

import paper_1707_00424_b200 as pb
from paper_1707_00424_b200.binding import AdamwStep, AdamwTensor

EINVAL, EALIGN = -1, -3
P = 1 << 20                                               # an aligned address that is never read
NAMES = ("param", "grad", "exp_avg", "exp_avg_sq", "exp_avg_scale", "exp_avg_sq_scale", "copy")


def adamw(n=3, bits=8, sizes=None, change=None, flags=None, **numbers):
    """n tensors with arrays of their own; change: (tensor, array) -> (tensor, array) whose address it gets."""
    arr = (AdamwTensor * n)(*(AdamwTensor(*((k * n + i + 1) * P for k in range(7)), size=sizes[i] if sizes else 100) for i in range(n)))
    for (i, name), (j, other) in (change or {}).items():
        setattr(arr[i], name, getattr(arr[j], other))
    h = dict(lr=0.1, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.1, grad_scale=1.0, max_norm=math.inf, step=1, norm=None, lr_dev=None, step_dev=None)
    step = AdamwStep(**{**h, **{k: getattr(arr[v[0]], v[1]) for k, v in numbers.items()}})
    return pb.lib().parle_adamw(arr, n, 0, 0, 2, bits, C.byref(step), getattr(arr[flags[0]], flags[1]) if flags else None, None)


@pytest.mark.parametrize("written", [name for name in NAMES if name != "grad"])
@pytest.mark.parametrize("reader, writer", [(0, 0), (0, 2), (2, 0)])
def test_a_gradient_that_is_a_written_array(written, reader, writer):
    assert adamw(change={(reader, "grad"): (writer, written)}) == EINVAL
    if "scale" not in written:
        assert adamw(bits=32, change={(reader, "grad"): (writer, written)}) == EINVAL


def test_the_last_of_many_gradients():
    assert adamw(n=3000, change={(2999, "grad"): (0, "exp_avg_sq_scale")}) == EINVAL
    assert adamw(n=3000, change={(0, "grad"): (2999, "copy")}) == EINVAL


@pytest.mark.parametrize("number", ["norm", "lr_dev", "step_dev"])
def test_a_number_on_the_device_that_is_a_written_array(number):
    for written in ("param", "exp_avg", "exp_avg_sq_scale"):
        assert adamw(**{number: (1, written)}) == EINVAL
    assert adamw(flags=(2, "param")) == EINVAL


def test_arrays_of_empty_tensors_are_not_looked_at():
    assert adamw(sizes=[0, 0, 0], change={(0, "grad"): (1, "param"), (2, "param"): (1, "param")}) == 0
