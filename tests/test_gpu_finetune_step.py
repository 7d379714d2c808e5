"""What the fine-tuning example does to its weights, step by step."""
import numpy as np
import pytest

from oracle import director_training_oracle as tro

pytestmark = pytest.mark.gpu

DIMS = dict(tokens=128, hidden=256, width=256, experts=8, topk=2, shared=1)


@pytest.mark.parametrize("max_norm, balance", [(0.0, 0.0), (1e-3, 0.0), (1e-3, 0.01), (1e9, 0.01)])
def test_every_update_of_the_example_is_adamws(monkeypatch, max_norm, balance):
    """The steps that train() takes with AdamW, on the gradients of the layer, against the definition in fp64."""
    import math

    import torch
    from paper_2607_08782_b200 import finetune
    from test_gpu_training import _Reference
    seen = []

    class Checked(finetune.AdamW):
        def step(self, grads=None, lr=None):
            grads = list(grads)
            ref, before = _Reference(self), [w.detach().clone() for w in self.weights]
            norm = super().step(grads, lr)
            ref.step(grads, self.lr, self.max_norm)
            assert all(not torch.equal(a, b.detach()) for a, b in zip(before, self.weights)), "every weight learns"
            seen.append((self.max_norm, len(grads)))
            return norm
    monkeypatch.setattr(finetune, "AdamW", Checked)
    losses = finetune.train(steps=4, lr=1e-2, optimizer="adamw", max_norm=max_norm, balance=balance, **DIMS)
    assert seen == [(max_norm or math.inf, 7)] * 4 and np.isfinite(losses).all()


def test_what_the_other_optimizer_gets_is_clipped(monkeypatch):
    import torch
    from paper_2607_08782_b200 import finetune
    seen = []

    def checked(grads, max_norm, out=None):
        norm = clip(grads, max_norm, out=out)
        want = tro.grad_norm([g.double().cpu().numpy() for g in grads])
        factor = tro.clip_factor(want, max_norm)
        assert factor < 1.0 and abs(norm.item() - want) <= 2.0 ** -19 * want
        for o, g in zip(out, grads):                          # the norm's error, the factor's and the product's rounding
            assert o.dtype is torch.float32 and ((o.double() - factor * g.double()).abs() <= 2.0 ** -19 * g.double().abs() * factor + 1e-45).all()
        seen.append(norm)
        return norm
    clip = finetune.clip_grads
    monkeypatch.setattr(finetune, "clip_grads", checked)
    losses = finetune.train(steps=3, optimizer="torch", max_norm=1e-3, balance=0.01, **DIMS)
    assert len(seen) == 3 and np.isfinite(losses).all()


@pytest.mark.parametrize("balance", [0.0, 0.5])
def test_the_gradient_that_the_example_takes(balance):
    """The logits' gradient of loss + balance * term is the layer's gradient and the oracle's for the term."""
    import torch
    from paper_2607_08782_b200.finetune import moe_layer
    from test_gpu_training import _batch, _layer
    layer = _layer()
    logits, x, dy = _batch(6)
    logits.requires_grad_()
    y = moe_layer(layer, x, logits)
    plain, = torch.autograd.grad((y.float() * dy.float()).sum(), [logits])
    y, even = moe_layer(layer, x, logits, balance=True)
    idx = layer.topk_idx[:96].cpu().numpy()
    both, = torch.autograd.grad((y.float() * dy.float()).sum() + balance * even.sum(), [logits])
    want = tro.balance_backward(logits.detach().double().cpu().numpy(), idx, None, 2, balance)
    # the term's own error: scores to 2^-20 of their size, and E/N f is at most E/N; then one rounding of the sum
    bound = balance * 8 / 96 * 2.0 ** -19 + 2.0 ** -24 * both.double().abs().cpu().numpy()
    assert (np.abs((both.double() - plain.double()).cpu().numpy() - want) <= bound).all()
    assert abs(even.item() - tro.balance(logits.detach().double().cpu().numpy(), idx, None, 2)[0]) <= 2.0 ** -18
