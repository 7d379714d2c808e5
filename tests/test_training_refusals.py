"""What the calls between the gradients and the next weights refuse, through the C entry points: every case is turned down on the host
before anything is launched, so that none of it needs a GPU (the addresses are made up)."""
import ctypes
import math

import pytest

from paper_2607_08782_b200 import binding
from paper_2607_08782_b200.binding import BF16, FP32, DirectorAdamW, DirectorParam, DirectorTensor

A = 1 << 40                     # a page of its own for every array
PAGE = 1 << 24
NORM, WORK, STEPS, STATUS, LR = (A + (100 + i) * PAGE for i in range(5))
INVALID, UNSUPPORTED = 1, 5


def _tensors(*items):
    a = (DirectorTensor * max(1, len(items)))()
    for t, (data, numel, kind) in zip(a, items):
        t.data, t.numel, t.type = data, numel, kind
    return len(items), a


def _norm(n, a, norm=NORM, work=WORK):
    return binding.load_library().director_grad_norm(n, a, norm, work, None)


def _clip(n, a, out, max_norm=1.0, norm=NORM, work=WORK):
    return binding.load_library().director_clip_grads(n, a, out, max_norm, norm, work, None)


BAD_TENSORS = [
    (None, 5, FP32), (A, -1, FP32), (A, 5, 2), (A, 5, -1), (A + 1, 5, BF16), (A + 2, 5, FP32),
]


@pytest.mark.parametrize("bad", BAD_TENSORS)
def test_tensors_of_the_wrong_kind(bad):
    n, a = _tensors((A + PAGE, 3, FP32), bad)
    assert _norm(n, a) == INVALID
    assert _clip(n, a, None) == INVALID
    good = _tensors((A + PAGE, 3, FP32), (A + 3 * PAGE, 5, FP32))[1]
    assert _clip(n, good, a) == INVALID


def test_a_tensor_that_is_too_long():
    n, a = _tensors((A, (1 << 40) + 1, BF16))
    assert _norm(n, a) == UNSUPPORTED and _clip(n, a, None) == UNSUPPORTED
    assert _norm((1 << 24) + 1, a) == UNSUPPORTED
    assert _step(_tensors((None, 0, BF16))[1], (DirectorParam * 1)(_param(numel=(1 << 40) + 1))) == UNSUPPORTED


def test_missing_and_misaligned_buffers():
    n, a = _tensors((A, (1 << 20) + 1, FP32))                # one element more than what needs no workspace
    for bad in (None, NORM + 1):
        assert _norm(n, a, norm=bad) == INVALID and _clip(n, a, None, norm=bad) == INVALID
    for bad in (None, WORK + 8):
        assert _norm(n, a, work=bad) == INVALID and _clip(n, a, None, work=bad) == INVALID
    assert _norm(1, None) == INVALID and _norm(-1, a) == INVALID
    assert _norm(n, a, norm=A + 400) == INVALID and _norm(n, a, work=A + 1600) == INVALID       # inside the gradient
    assert _norm(n, a, norm=WORK + 16) == INVALID


@pytest.mark.parametrize("max_norm", [0.0, -1.0, -math.inf, math.nan])
def test_max_norm_has_to_be_positive(max_norm):
    n, a = _tensors((A, 5, FP32))
    assert _clip(n, a, None, max_norm) == INVALID


def test_clip_refuses_overlaps_and_other_lengths():
    n, a = _tensors((A, 100, FP32), (A + 396, 100, FP32))            # in place, the last element is the next one's first
    assert _clip(n, a, None) == INVALID
    n, a = _tensors((A, 100, FP32), (A, 100, FP32))                  # the same tensor twice
    assert _clip(n, a, None) == INVALID
    n, a = _tensors((A, 100, BF16))
    assert _clip(n, a, _tensors((A, 100, FP32))[1]) == INVALID       # the same address, another type
    assert _clip(n, a, _tensors((A + 2, 100, BF16))[1]) == INVALID   # shifted by an element
    assert _clip(n, a, _tensors((A + PAGE, 99, BF16))[1]) == INVALID
    assert _clip(n, a, None, norm=A + 100) == INVALID                # the result inside a gradient
    assert _clip(n, a, None, work=A) == INVALID


def _step(grads, params, h=None, lr=None, steps=STEPS, norm=NORM, status=STATUS, work=WORK, n=None):
    h = DirectorAdamW(1e-3, 0.9, 0.99, 1e-8, 0.0, 1.0) if h is None else h
    return binding.load_library().director_adamw_step(len(params) if n is None else n, grads, params, ctypes.byref(h) if h else None, lr, steps,
                                                      norm, status, work, None)


def _param(base=A, numel=100, kind=BF16, **over):
    fields = dict(weight=base, master=base + PAGE if kind == BF16 else None, exp_avg=base + 2 * PAGE, exp_avg_sq=base + 3 * PAGE,
                  numel=numel, type=kind)
    fields.update(over)
    return DirectorParam(*(fields[k] for k in ("weight", "master", "exp_avg", "exp_avg_sq", "numel", "type")), 0)


def _grad(numel=100, at=A + 50 * PAGE):
    return _tensors((at, numel, BF16))[1]


@pytest.mark.parametrize("over", [
    dict(weight=None), dict(master=None), dict(exp_avg=None), dict(exp_avg_sq=None), dict(weight=A + 1), dict(master=A + PAGE + 2),
    dict(exp_avg=A + 1), dict(numel=99), dict(numel=-1), dict(type=7), dict(exp_avg=A + 3 * PAGE), dict(exp_avg=A), dict(master=A + 100),
    dict(exp_avg=A + 50 * PAGE)])
def test_step_refuses_bad_weights_and_states(over):
    assert _step(_grad(), (DirectorParam * 1)(_param(**over))) == INVALID


def test_step_refuses_a_master_of_an_fp32_weight_and_weights_given_twice():
    assert _step(_grad(), (DirectorParam * 1)(_param(kind=FP32, master=A + PAGE))) == INVALID
    twice = (DirectorParam * 2)(_param(), _param())
    grads = _tensors((A + 50 * PAGE, 100, BF16), (A + 60 * PAGE, 100, BF16))[1]
    assert _step(grads, twice) == INVALID


def test_step_refuses_missing_and_misaligned_buffers():
    p = (DirectorParam * 1)(_param())
    for over in (dict(steps=None), dict(steps=STEPS + 4), dict(norm=NORM + 2), dict(status=STATUS + 1), dict(work=None), dict(work=WORK + 8),
                 dict(lr=LR + 2), dict(lr=A), dict(norm=STEPS), dict(h=False), dict(n=-1)):
        assert _step(_grad(), p, **over) == INVALID, over
    assert _step(_grad(), None, n=1) == INVALID


@pytest.mark.parametrize("field, value", [
    ("beta1", 1.0), ("beta1", -0.1), ("beta1", math.nan), ("beta2", 1.0), ("beta2", math.nan), ("eps", -1e-8), ("eps", math.inf),
    ("eps", math.nan), ("max_norm", 0.0), ("max_norm", math.nan), ("lr", math.inf), ("lr", math.nan), ("weight_decay", math.inf)])
def test_step_refuses_bad_numbers(field, value):
    h = DirectorAdamW(1e-3, 0.9, 0.99, 1e-8, 0.0, 1.0)
    setattr(h, field, value)
    assert _step(_grad(), (DirectorParam * 1)(_param()), h=h) == INVALID


def test_python_refusals_that_need_no_gpu():
    import torch
    from paper_2607_08782_b200 import training
    with pytest.raises(ValueError):
        training.TensorList([torch.zeros(4)])
    with pytest.raises(TypeError):
        training.TensorList([torch.zeros(4, dtype=torch.float16)])
    from paper_2607_08782_b200.finetune import train
    with pytest.raises(ValueError):
        train(optimizer="sgd")


def test_the_header_and_the_binding_agree_on_the_small_norm():
    import os
    import re
    text = open(os.path.join(os.path.dirname(__file__), "..", "include", "director.h")).read()
    assert int(re.search(r"DIRECTOR_SMALL_TENSORS (\d+)", text)[1]) == binding.SMALL_TENSORS
    assert eval(re.search(r"DIRECTOR_SMALL_BYTES \((.*?)\)", text)[1]) == binding.SMALL_BYTES
    assert ctypes.sizeof(DirectorTensor) == 24 and ctypes.sizeof(DirectorParam) == 48 and ctypes.sizeof(DirectorAdamW) == 48
