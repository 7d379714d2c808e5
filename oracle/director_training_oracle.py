"""What a training step needs besides the gradients, in fp64: the router's balance term and its gradient, the global norm of
gradients, clipping by it, and AdamW.  Test infrastructure: shares no code with the GPU path."""
import numpy as np


def balance(logits, idx, mask, K):
    """(loss, counts [E+1], p [T,E], diff [T,E], f): diff = f_e - sum_j f_j p_tj; p and diff are zero for tokens without scores (masked,
    or a row that is not finite), f less its mean."""
    T, E = logits.shape
    valid = np.ones(T, bool) if mask is None else mask.astype(bool)
    x = np.where(valid[:, None], logits.astype(np.float64), 0.0)
    with np.errstate(invalid="ignore"):
        z = np.exp(x - x.max(1, keepdims=True))
        p = z / z.sum(1, keepdims=True)
    good = valid & np.isfinite(p).all(1)
    p = np.where(good[:, None], p, 0.0)
    chosen = idx[valid].reshape(-1)
    counts = np.bincount(chosen[(chosen >= 0) & (chosen < E)], minlength=E)
    N = int(valid.sum())
    loss = E * float(counts / (K * max(N, 1)) @ p.sum(0)) / max(N, 1)
    f = (E * counts - counts.sum()) / (E * K * max(N, 1))
    return loss, np.append(counts, N), p, np.where(good[:, None], f - (p @ f)[:, None], 0.0), f


def balance_backward(logits, idx, mask, K, dloss, added=None):
    """dlogits of the loss with the counts held fixed."""
    _, counts, p, diff, _ = balance(logits, idx, mask, K)
    d = dloss * logits.shape[1] / max(int(counts[-1]), 1) * p * diff
    return d if added is None else d + added


def grad_norm(grads):
    return float(np.sqrt(sum(float((np.asarray(g, np.float64) ** 2).sum()) for g in grads)))


def clip_factor(norm, max_norm):
    """What the gradients are multiplied by; one where the norm is not finite."""
    return max_norm / norm if np.isfinite(norm) and norm > max_norm else 1.0


def adamw(w, m, v, t, g, lr, betas, eps, weight_decay):
    """(w, m, v) after step number t."""
    m = betas[0] * m + (1 - betas[0]) * g
    v = betas[1] * v + (1 - betas[1]) * g ** 2
    w = w - lr * weight_decay * w - lr * (m / (1 - betas[0] ** t)) / (np.sqrt(v / (1 - betas[1] ** t)) + eps)
    return w, m, v
