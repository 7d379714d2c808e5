"""The reference that the GPU tests of AdamW hold the kernels to, itself held to the definitions in fp64 and to torch's AdamW."""
import types

import numpy as np
import pytest
import torch

import test_gpu_training
from oracle import director_training_oracle as tro


class _Exact(test_gpu_training._Reference):
    """The reference with a tolerance of fp64's rounding in place of the kernels'."""

    @staticmethod
    def check(got, want, tol):
        assert (got.detach().double() - want).abs().max() <= 1e-12 * want.abs().max() + 1e-300


def _optimizer(n, t, seed=0, masters=False):
    g = torch.Generator().manual_seed(seed)
    w, m, v = torch.randn(n, generator=g).double(), torch.randn(n, generator=g).double() * 1e-2, torch.rand(n, generator=g).double() * 1e-3
    if t == 0:
        m.zero_(), v.zero_()
    return types.SimpleNamespace(weights=[w.to(torch.bfloat16) if masters else w], masters=[w.clone() if masters else None], exp_avg=[m], exp_avg_sq=[v],
                                 steps=torch.tensor([t]), betas=(0.9, 0.95), eps=1e-8, weight_decay=0.1)


def _advance(opt, w, m, v):
    """New tensors: in fp64 the reference holds the old ones themselves."""
    w, opt.exp_avg[0], opt.exp_avg_sq[0] = (torch.as_tensor(t).clone() for t in (w, m, v))
    if opt.masters[0] is not None:
        opt.masters[0], opt.weights[0] = w, w.to(torch.bfloat16)
    else:
        opt.weights[0] = w
    opt.steps = opt.steps + 1


@pytest.mark.parametrize("masters", [False, True])
@pytest.mark.parametrize("t", [0, 1, 1000])
@pytest.mark.parametrize("fraction", [0.3, 1.5, float("inf")])
def test_the_reference_is_the_oracle(fraction, t, masters):
    opt = _optimizer(500, t, t, masters)
    for k in range(3):
        grad = torch.randn(500, generator=torch.Generator().manual_seed(50 + k)).double()
        norm = tro.grad_norm([grad.numpy()])
        limit = fraction * norm
        factor = tro.clip_factor(norm, limit)
        assert factor == (0.3 if fraction == 0.3 else 1.0) or abs(factor - fraction) < 1e-15
        ref = _Exact(opt)
        state = [(opt.masters[0] if masters else opt.weights[0]).numpy().copy(), opt.exp_avg[0].numpy().copy(), opt.exp_avg_sq[0].numpy().copy()]
        _advance(opt, *tro.adamw(*state, int(opt.steps) + 1, factor * grad.numpy(), 3e-3, opt.betas, opt.eps, opt.weight_decay))
        assert abs(ref.step([grad], 3e-3, limit) - norm) <= 1e-12 * norm


@pytest.mark.parametrize("decay", [0.0, 0.1])
def test_the_reference_is_torchs_adamw(decay):
    opt = _optimizer(300, 0)
    opt.weight_decay = decay
    w = torch.nn.Parameter(opt.weights[0].clone())
    theirs = torch.optim.AdamW([w], lr=3e-3, betas=opt.betas, eps=opt.eps, weight_decay=decay)
    for k in range(5):
        grad = torch.randn(300, generator=torch.Generator().manual_seed(70 + k)).double() * 10.0 ** -k
        w.grad = grad.clone()
        ref = _Exact(opt)
        theirs.step()
        state = theirs.state[w]
        _advance(opt, w.detach(), state["exp_avg"], state["exp_avg_sq"])
        ref.step([grad], 3e-3, float("inf"))


@pytest.mark.parametrize("mistake", ["no decay", "no correction", "eps under the root", "unclipped", "beta1 for beta2", "step not counted", "coupled decay"])
def test_the_reference_with_the_kernels_tolerance_sees_mistakes(mistake):
    opt = _optimizer(500, 3)
    grad = torch.randn(500, generator=torch.Generator().manual_seed(1)).double() * 1e-3
    norm = tro.grad_norm([grad.numpy()])
    g, t, lr, (b1, b2), eps, decay = 0.5 * grad.numpy(), 4, 3e-3, opt.betas, opt.eps, opt.weight_decay
    w, m, v = opt.weights[0].numpy().copy(), opt.exp_avg[0].numpy().copy() * 1e-2, opt.exp_avg_sq[0].numpy().copy() * 1e-6
    opt.exp_avg[0], opt.exp_avg_sq[0] = torch.as_tensor(m.copy()), torch.as_tensor(v.copy())
    ref = test_gpu_training._Reference(opt)
    if mistake == "no decay":
        decay = 0.0
    elif mistake == "unclipped":
        g = 2.0 * g
    elif mistake == "beta1 for beta2":
        b2 = b1
    elif mistake == "coupled decay":
        g, decay = g + decay * w, 0.0
    m, v = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g ** 2
    m_hat, v_hat = (m, v) if mistake == "no correction" else (m / (1 - b1 ** t), v / (1 - b2 ** t))
    den = np.sqrt(v_hat + eps) if mistake == "eps under the root" else np.sqrt(v_hat) + eps
    _advance(opt, w - lr * decay * w - lr * m_hat / den, m, v)
    if mistake == "step not counted":
        opt.steps = opt.steps - 1
    with pytest.raises(AssertionError):
        ref.step([grad], lr, 0.5 * norm)


def test_the_reference_with_the_kernels_tolerance_takes_the_right_result():
    opt = _optimizer(500, 3)
    grad = torch.randn(500, generator=torch.Generator().manual_seed(1)).double() * 1e-3
    norm = tro.grad_norm([grad.numpy()])
    ref = test_gpu_training._Reference(opt)
    state = [opt.weights[0].numpy().copy(), opt.exp_avg[0].numpy().copy(), opt.exp_avg_sq[0].numpy().copy()]
    _advance(opt, *tro.adamw(*state, 4, 0.5 * grad.numpy(), 3e-3, opt.betas, opt.eps, opt.weight_decay))
    ref.step([grad], 3e-3, 0.5 * norm)
