"""The fp64 definitions of the backward pass against central differences of the forward's, and by hand (CPU)."""
import numpy as np
import pytest

from oracle import director_grad_oracle as gro
from oracle import director_oracle as orc


def _difference(f, x, d, eps=1e-6):
    """Directional derivative of the scalar f at x along d."""
    return (f(x + eps * d) - f(x - eps * d)) / (2 * eps)


def _rng(seed):
    return np.random.default_rng(seed)


def test_combine_and_dispatch_gradients_are_the_derivatives():
    rng = _rng(1)
    T, K, H = 7, 3, 5
    inv = rng.permutation(T * K).reshape(T, K).astype(np.int32)
    yp, w, dy = rng.normal(size=(T * K, H)), rng.random((T, K)), rng.normal(size=(T, H))
    dyp, dw = gro.combine_backward(dy, yp, inv, w)
    d = rng.normal(size=yp.shape)
    assert np.isclose(_difference(lambda v: np.sum(dy * orc.combine(v, inv, w)), yp, d), np.sum(dyp * d), rtol=1e-7)
    d = rng.normal(size=w.shape)
    assert np.isclose(_difference(lambda v: np.sum(dy * orc.combine(yp, inv, v)), w, d), np.sum(dw * d), rtol=1e-7)
    dxp, x = rng.normal(size=(T * K, H)), rng.normal(size=(T, H))
    dx = gro.dispatch_backward(dxp, inv)

    def moved(v):
        xp = np.zeros((T * K, H))
        for s in range(K):
            xp[inv[:, s]] = v
        return np.sum(dxp * xp)
    d = rng.normal(size=x.shape)
    assert np.isclose(_difference(moved, x, d), np.sum(dx * d), rtol=1e-7)
    assert np.allclose(gro.dispatch_backward(dxp, inv, x), dx + x)


def test_a_skipped_assignment_takes_no_part():
    rng = _rng(2)
    inv = np.array([[0, -1], [1, 2]], dtype=np.int32)
    dy, yp, w = rng.normal(size=(2, 4)), rng.normal(size=(4, 4)), np.ones((2, 2))
    dyp, dw = gro.combine_backward(dy, yp, inv, w)
    assert dw[0, 1] == 0 and not dyp[3].any()
    assert np.array_equal(gro.dispatch_backward(yp, inv)[0], yp[0])


def test_gate_gradient_is_the_derivative():
    rng = _rng(3)
    T, E, K = 6, 9, 4
    logits, dw = rng.normal(size=(T, E)), rng.normal(size=(T, K))
    idx = np.argsort(-logits, axis=1)[:, :K]

    def f(l):
        z = np.take_along_axis(l, idx, axis=1)
        p = np.exp(z - z.max(1, keepdims=True))
        return np.sum(dw * p / p.sum(1, keepdims=True))
    z = np.take_along_axis(logits, idx, axis=1)
    w = np.exp(z) / np.exp(z).sum(1, keepdims=True)
    dl = gro.route_backward(idx, w, dw, E)
    d = rng.normal(size=logits.shape)
    assert np.isclose(_difference(f, logits, d), np.sum(dl * d), rtol=1e-7)
    assert np.allclose(dl.sum(1), 0, atol=1e-14)                  # a softmax is blind to a common shift
    assert np.allclose(gro.route_backward(idx[:, :1], np.ones((T, 1)), dw[:, :1], E), 0)


@pytest.mark.parametrize("which", ["x", "wg", "wu", "wd"])
def test_ffn_gradient_is_the_derivative(which):
    rng = _rng(4)
    n, H, F = 5, 6, 7
    a = dict(x=rng.normal(size=(n, H)), wg=rng.normal(size=(F, H)), wu=rng.normal(size=(F, H)), wd=rng.normal(size=(H, F)))
    dy = rng.normal(size=(n, H))
    _, g, u = gro.swiglu_ffn(**a)
    grads = dict(zip(("x", "wg", "wu", "wd"), gro.swiglu_ffn_backward(a["x"], dy, g, u, a["wg"], a["wu"], a["wd"])))
    d = rng.normal(size=a[which].shape)
    got = _difference(lambda v: np.sum(dy * gro.swiglu_ffn(**{**a, which: v})[0]), a[which], d)
    assert np.isclose(got, np.sum(grads[which] * d), rtol=1e-6)


def test_grouped_gradient_sums_over_replicas():
    rng = _rng(5)
    H, F, E = 4, 3, 2
    xp, dyp = rng.normal(size=(9, H)), rng.normal(size=(9, H))
    w = [rng.normal(size=s) for s in ((E, F, H), (E, F, H), (E, H, F))]
    seg, slot = np.array([0, 4, 4, 7, 9]), np.array([0, -1, 1, 0])      # expert 0 on two slots, one slot unused
    g, u = np.zeros((9, F)), np.zeros((9, F))
    for lo, hi, e in ((0, 4, 0), (4, 7, 1), (7, 9, 0)):
        _, g[lo:hi], u[lo:hi] = gro.swiglu_ffn(xp[lo:hi], w[0][e], w[1][e], w[2][e])
    dxp, dwg, dwu, dwd = gro.expert_ffn_backward(xp, dyp, seg, slot, g, u, *w)
    rows = np.r_[0:4, 7:9]
    one = gro.swiglu_ffn_backward(xp[rows], dyp[rows], g[rows], u[rows], w[0][0], w[1][0], w[2][0])
    assert np.allclose(dxp[rows], one[0]) and np.allclose(dwg[0], one[1]) and np.allclose(dwu[0], one[2]) and np.allclose(dwd[0], one[3])


def test_checkpoint_by_hand_and_its_error():
    v = np.zeros((4, 32))
    v[0, :3] = [1.0, -0.5, 0.25]            # largest 1.0 = 2^0: step 2^-6, codes 64, -32, 16
    v[1, :2] = [1.999, -3.0]                # largest 3: step 2^-5
    v[2, 20] = np.inf
    v[3, 16:18] = [127.9, 1e-3]             # 127.9 / 2^0 is held at 127
    codes, exps = gro.checkpoint_encode(v)
    assert list(codes[0, :4]) == [64, -32, 16, 0] and exps[0, 0] == 121
    assert codes[1, 1] == -96 and codes[1, 0] == 64 and exps[0, 1] == 122
    assert exps[1, 2] == 255 and exps[0, 2] == 1
    assert codes[3, 16] == 127 and codes[3, 17] == 0 and exps[1, 3] == 127
    back = gro.checkpoint_decode(codes, exps)
    assert np.isnan(back[2, 16:]).all() and not back[2, :16].any()
    rng = _rng(6)
    v = rng.normal(size=(64, 64)) * 10.0 ** rng.integers(-6, 6, size=(64, 1))
    back = gro.checkpoint_decode(*gro.checkpoint_encode(v))
    big = np.repeat(np.abs(v).reshape(64, 4, 16).max(-1), 16, axis=1)
    assert (np.abs(back - v) <= 2.0 ** -7 * 1.01 * big).all()


def test_training_on_the_checkpoint_is_near_the_exact_gradient():
    """What the eight bits cost: gradients from the kept gate and up values against those from the exact ones."""
    rng = _rng(7)
    n, H, F = 96, 64, 128
    x, dy = rng.normal(size=(n, H)), rng.normal(size=(n, H))
    w = [rng.normal(size=s) * H ** -0.5 for s in ((F, H), (F, H), (H, F))]
    _, g, u = gro.swiglu_ffn(x, *w)
    kept = [gro.checkpoint_decode(*gro.checkpoint_encode(v)) for v in (g, u)]
    a = gro.swiglu_ffn_backward(x, dy, g, u, *w)
    b = gro.swiglu_ffn_backward(x, dy, *kept, *w)
    for p, q in zip(a[:4], b[:4]):
        assert np.linalg.norm(p - q) < 0.02 * np.linalg.norm(p)
