"""The oracle of the training step's operators: against central differences, worked examples and torch's own AdamW in fp64 (CPU)."""
import numpy as np
import pytest

from oracle import director_oracle as orc
from oracle import director_training_oracle as tro


def _case(T, E, K, seed, masked):
    rng = np.random.default_rng(seed)
    logits = rng.standard_normal((T, E)) + rng.standard_normal(E)
    idx = orc.route(logits.astype(np.float32), K)[0]
    return logits, idx, (rng.random(T) < 0.6) if masked else None


@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("T, E, K", [(1, 3, 1), (7, 5, 2), (9, 4, 4)])
def test_balance_gradient_is_the_difference_of_losses(T, E, K, masked):
    logits, idx, mask = _case(T, E, K, T, masked)
    got = tro.balance_backward(logits, idx, mask, K, 0.7)
    h = 1e-5
    for t in range(T):
        for e in range(E):
            up, down = logits.copy(), logits.copy()
            up[t, e] += h
            down[t, e] -= h
            diff = 0.7 * (tro.balance(up, idx, mask, K)[0] - tro.balance(down, idx, mask, K)[0]) / (2 * h)
            assert abs(got[t, e] - diff) < 1e-9                  # h^2 / 6 of a third derivative below E


def test_balance_by_hand():
    # two tokens, two experts, top-1: scores (3/4, 1/4) and (1/4, 3/4); both choose expert 0
    logits = np.log(np.array([[3.0, 1.0], [1.0, 3.0]]))
    loss, counts, p, _, _ = tro.balance(logits, np.array([[0], [0]]), None, 1)
    assert np.allclose(p, [[0.75, 0.25], [0.25, 0.75]]) and list(counts) == [2, 0, 2]
    assert abs(loss - 2 * (1.0 * 0.5 + 0.0 * 0.5)) < 1e-15
    loss, counts, *_ = tro.balance(logits, np.array([[0], [0]]), np.array([1, 0]), 1)
    assert list(counts) == [1, 0, 1] and abs(loss - 1.5) < 1e-15
    even = tro.balance(np.zeros((4, 4)), np.arange(4).reshape(4, 1), None, 1)
    assert even[0] == 1.0 and not even[3].any()
    nothing = tro.balance(logits, np.array([[0], [0]]), np.zeros(2), 1)
    assert nothing[0] == 0.0 and not nothing[1].any()


def test_norm_and_factor():
    assert tro.grad_norm([np.array([3.0]), np.array([[0.0, -4.0]])]) == 5.0 and tro.grad_norm([]) == 0.0
    assert tro.clip_factor(5.0, 1.0) == 0.2 and tro.clip_factor(0.5, 1.0) == 1.0
    assert tro.clip_factor(np.inf, 1.0) == 1.0 and tro.clip_factor(np.nan, 1.0) == 1.0


@pytest.mark.parametrize("decay", [0.0, 0.1])
def test_adamw_is_torchs(decay):
    import torch
    rng = np.random.default_rng(1)
    w = rng.standard_normal(50)
    p = torch.nn.Parameter(torch.tensor(w))
    opt = torch.optim.AdamW([p], lr=3e-3, betas=(0.8, 0.97), eps=1e-6, weight_decay=decay)
    m, v = np.zeros(50), np.zeros(50)
    for t in range(1, 6):
        g = rng.standard_normal(50) * 10.0 ** -t
        p.grad = torch.tensor(g)
        opt.step()
        w, m, v = tro.adamw(w, m, v, t, g, 3e-3, (0.8, 0.97), 1e-6, decay)
        assert np.abs(p.detach().numpy() - w).max() < 1e-13
