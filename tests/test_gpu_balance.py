"""The router's balance term: loss, counts and gradient against the definition in fp64."""
import numpy as np
import pytest

from oracle import director_training_oracle as tro

pytestmark = pytest.mark.gpu


def _director(T, E, K):
    from paper_2607_08782_b200.binding import Director
    return Director(T, 256, 128, E, K, 0, 16, 16)


def _inputs(T, E, K, masked, seed, spread=1.0):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    logits = (torch.randn((T, E), generator=g, device="cuda") + torch.randn((E,), generator=g, device="cuda")) * spread
    idx = logits.topk(K, dim=1).indices.int().contiguous()
    mask = (torch.rand((T,), generator=g, device="cuda") < 0.7).to(torch.uint8) if masked else None
    added = torch.randn((T, E), generator=g, device="cuda") * 1e-3
    return logits, idx, mask, added


def _p_tolerance(logits):
    """Relative error of a score.  The exponential: its argument, d log2(e) with d = x - max, is rounded once (2^-24 |d| log2(e), so
    2^-24 |d| of the score; twice that allowed), 2 ulp of the power of two; the sum over E <= 256 terms: 16 in a lane, one after another,
    and 4 shuffles; the division."""
    x = logits.double()
    x = x[x.isfinite().all(1)]
    d = float((x.amax(1) - x.amin(1)).max()) if x.numel() else 0.0
    return 2 * (2 * min(d, 90.0) + 4 + 20 + 2) * 2.0 ** -24


def _check(d, T, E, K, logits, idx, mask, added, dloss=0.37):
    import torch
    loss = torch.full((1,), 7.0, device="cuda")
    counts = torch.full((E + 1,), -7, dtype=torch.int64, device="cuda")
    d.balance_loss(T, logits, idx, mask, loss, counts)
    want, want_counts, p, diff, f = tro.balance(logits.cpu().numpy(), idx.cpu().numpy(), None if mask is None else mask.cpu().numpy(), K)
    f_max, N = np.abs(f).max(), max(int(want_counts[-1]), 1)
    assert np.array_equal(counts.cpu().numpy(), want_counts)
    tol = _p_tolerance(logits if mask is None else logits[mask.bool()])
    # the sum over tokens: up to 64 of a lane one after another, 5 shuffles; all terms positive
    assert abs(loss.item() - want) <= (tol + 2.0 ** -24 * (64 + 5 + 2)) * want + 1e-30
    scale = np.float32(dloss).astype(np.float64) * E / N
    dl = torch.tensor([dloss], device="cuda")
    for base in (None, added):
        out = torch.full((T, E), 7.0, device="cuda")
        d.balance_loss_backward(T, logits, counts, mask, dl, base, out)
        ref = scale * p * diff + (0.0 if base is None else base.double().cpu().numpy())
        # relative errors of p and scale, and of the difference: the mean carries p's error and 24 roundings
        bound = scale * p * (2 * tol + 2.0 ** -21) * (np.abs(diff) + f_max) + 2.0 ** -24 * np.abs(ref) + 1e-37
        assert (np.abs(out.double().cpu().numpy() - ref) <= bound).all()
        if base is not None:
            again = base.clone()                              # added in place
            d.balance_loss_backward(T, logits, counts, mask, dl, again, again)
            assert torch.equal(again, out)
    return loss, counts


@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("E, K", [(1, 1), (2, 1), (3, 3), (8, 2), (13, 5), (16, 1), (17, 4), (32, 8), (60, 4), (64, 6), (100, 7), (128, 8),
                                  (129, 2), (251, 8), (256, 8)])
@pytest.mark.parametrize("T", [1, 2, 31, 257, 4099])
def test_matches_the_definition(T, E, K, masked):
    d = _director(T, E, K)
    _check(d, T, E, K, *_inputs(T, E, K, masked, T * 1000 + E))
    assert d.last_status() == 0


@pytest.mark.parametrize("E, K", [(8, 2), (60, 4), (256, 8)])
def test_a_long_batch_and_the_same_bits_again(E, K):
    import torch
    T = 70001
    d = _director(T, E, K)
    logits, idx, mask, added = _inputs(T, E, K, True, 5)
    loss, counts = _check(d, T, E, K, logits, idx, mask, added)
    for _ in range(3):
        l2, c2 = torch.empty_like(loss), torch.empty_like(counts)
        d.balance_loss(T, logits, idx, mask, l2, c2)
        assert torch.equal(l2, loss) and torch.equal(c2, counts)
    d.balance_loss(17, logits, idx, mask, l2, c2)            # a shorter batch after a long one
    assert int(c2[E]) == int(mask[:17].sum())
    assert d.last_status() == 0


def test_offsets_past_31_bits():
    """More logits than 31 bits count: the loss in pieces, the gradient of the first and the last tokens."""
    import torch
    T, E, K = 8_400_011, 256, 1
    if torch.cuda.mem_get_info()[0] < 100 << 30:
        pytest.skip("needs 100 GB")
    d = _director(T, E, K)
    g = torch.Generator(device="cuda").manual_seed(3)
    logits = torch.randn((T, E), generator=g, device="cuda")
    idx = torch.randint(0, E // 2, (T, K), generator=g, device="cuda").int()
    mask = (torch.arange(T, device="cuda") % 7 != 0)
    loss, counts = torch.empty(1, device="cuda"), torch.empty(E + 1, dtype=torch.int64, device="cuda")
    d.balance_loss(T, logits, idx, mask, loss, counts)
    N = int(mask.sum())
    want = torch.bincount(idx[mask].view(-1).long(), minlength=E)
    assert torch.equal(counts[:E], want) and int(counts[E]) == N
    P = torch.zeros(E, dtype=torch.float64, device="cuda")
    for lo in range(0, T, 400_000):
        p = logits[lo:lo + 400_000].double().softmax(1)
        P += p[mask[lo:lo + 400_000]].sum(0)
    f = want.double() / N
    ref = E * float(f @ P) / N
    tol = _p_tolerance(logits[:100_000])
    assert abs(loss.item() - ref) <= (tol + 2.0 ** -24 * (64 + 5 + 2)) * ref
    out = torch.full((T, E), 7.0, device="cuda")
    d.balance_loss_backward(T, logits, counts, mask, torch.ones(1, device="cuda"), None, out)
    f = (E * want - want.sum()).double() / (E * N)
    for rows in (slice(0, 3000), slice((1 << 31) // E - 1500, (1 << 31) // E + 1500), slice(T - 3000, T)):
        p = logits[rows].double().softmax(1) * mask[rows].unsqueeze(1)
        diff = f - (p @ f).unsqueeze(1)
        bound = E / N * p * (2 * tol + 2.0 ** -21) * (diff.abs() + f.abs().max()) + 1e-37
        assert ((out[rows].double() - E / N * p * diff).abs() <= bound).all()
    assert d.last_status() == 0


def test_every_expert_chosen_by_every_token_has_no_gradient():
    import torch
    d = _director(500, 8, 8)
    logits, idx, _, _ = _inputs(500, 8, 8, False, 1)
    loss, counts = _check(d, 500, 8, 8, logits, idx, None, torch.zeros((500, 8), device="cuda"))
    out = torch.full((500, 8), 7.0, device="cuda")
    d.balance_loss_backward(500, logits, counts, None, torch.ones(1, device="cuda"), None, out)
    assert not out.any() and abs(loss.item() - 1.0) < 1e-5


def test_nothing_valid():
    import torch
    d = _director(40, 60, 4)
    logits, idx, _, added = _inputs(40, 60, 4, False, 2)
    logits.fill_(float("nan"))
    idx.fill_(1 << 30)
    loss, counts = _check(d, 40, 60, 4, logits, idx, torch.zeros(40, dtype=torch.bool, device="cuda"), added)
    assert loss.item() == 0.0 and not counts.any() and d.last_status() == 0


@pytest.mark.parametrize("E, K", [(8, 2), (61, 4), (256, 8)])
def test_masked_rows_are_not_looked_at(E, K):
    """Whatever padding holds: NaN, infinities, indices of no expert."""
    T = 999
    d = _director(T, E, K)
    logits, idx, mask, added = _inputs(T, E, K, True, 3)
    import torch
    rows = (mask == 0).nonzero().view(-1)
    logits[rows[0::3]] = float("nan")
    logits[rows[1::3]] = float("inf")
    logits[rows[2::3]] = -float("inf")
    idx[rows] = -5
    _check(d, T, E, K, logits, idx, mask, added)
    _check(d, T, E, K, logits, idx, mask.bool(), added)
    assert d.last_status() == 0
    assert torch.isfinite(added).all()


@pytest.mark.parametrize("E", [8, 61, 256])
def test_rows_that_are_not_finite_and_scores_of_zero(E):
    import torch
    T, K = 300, 2
    d = _director(T, E, K)
    logits, idx, _, added = _inputs(T, E, K, False, 4)
    logits[5, 0] = -float("inf")                              # an expert that is ruled out: score 0, no error
    logits[6, 1:] = -float("inf")                             # one expert left: score 1
    logits[7] = torch.finfo(torch.float32).min                # the type's lowest value everywhere: an even row
    logits[8, 1] = torch.finfo(torch.float32).min
    logits[9] = torch.finfo(torch.float32).max
    logits[10] = 0.0
    _check(d, T, E, K, logits, idx, None, added)
    assert d.last_status() == 0
    for value, row in ((float("nan"), 11), (float("inf"), 12)):
        bad = logits.clone()
        bad[row, E - 1] = value
        _check(d, T, E, K, bad, idx, None, added)
        assert d.last_status() == 8 and d.last_status() == 0
    bad = logits.clone()
    bad[13] = -float("inf")
    _check(d, T, E, K, bad, idx, None, added)
    assert d.last_status() == 8


def test_large_logits_do_not_overflow():
    T, E, K = 200, 60, 4
    d = _director(T, E, K)
    _check(d, T, E, K, *_inputs(T, E, K, False, 6, spread=1e4))
    _check(d, T, E, K, *_inputs(T, E, K, False, 7, spread=1e-6))


@pytest.mark.parametrize("E", [8, 61, 256])
@pytest.mark.parametrize("at", [1e3, 9e5, 2e6, 1e9, 1e12, 1e30, 1e37, 3e38])
def test_logits_far_from_zero(E, at):
    """Rows around `at` and -`at`, one step of fp32 or a few units apart."""
    import torch
    T, K = 64, 2
    d = _director(T, E, K)
    logits, idx, _, added = _inputs(T, E, K, False, 12)
    logits[:32] = at + logits[:32]
    logits[32:] = -at + logits[32:]
    logits[5, 1] = torch.nextafter(logits[5, 1], torch.tensor(0.0, device="cuda"))
    logits[40, 2] = logits[40].max() - 3.0
    assert torch.isfinite(logits).all()
    _check(d, T, E, K, logits, idx, None, added)
    assert d.last_status() == 0


def test_indices_of_no_expert_are_skipped_and_reported():
    T, E, K = 120, 60, 4
    d = _director(T, E, K)
    logits, idx, _, added = _inputs(T, E, K, False, 8)
    idx[3, 1], idx[100, 0], idx[7, 3] = E, -1, 1 << 30
    _check(d, T, E, K, logits, idx, None, added)
    assert d.last_status() == 7 and d.last_status() == 0


def test_the_gradient_is_the_difference_of_losses():
    """Central differences of the fp64 loss with the counts held fixed: h^2/6 of the third derivative, far below the tolerance."""
    import torch
    T, E, K = 6, 5, 2
    d = _director(T, E, K)
    logits, idx, _, _ = _inputs(T, E, K, False, 9)
    loss, counts = torch.empty(1, device="cuda"), torch.empty(E + 1, dtype=torch.int64, device="cuda")
    d.balance_loss(T, logits, idx, None, loss, counts)
    out = torch.empty((T, E), device="cuda")
    d.balance_loss_backward(T, logits, counts, None, torch.ones(1, device="cuda"), None, out)
    x, f = logits.double().cpu().numpy(), counts.cpu().numpy()[:E] / (K * T)

    def value(x):
        z = np.exp(x - x.max(1, keepdims=True))
        return E * float(f @ (z / z.sum(1, keepdims=True)).mean(0))
    h, diff = 1e-4, np.zeros((T, E))
    for t in range(T):
        for e in range(E):
            up, down = x.copy(), x.copy()
            up[t, e] += h
            down[t, e] -= h
            diff[t, e] = (value(up) - value(down)) / (2 * h)
    assert np.abs(out.cpu().numpy() - diff).max() < 1e-6


def test_counts_of_several_batches_give_the_gradient_of_their_loss():
    import torch
    T, E, K = 500, 60, 4
    d = _director(T, E, K)
    logits, idx, _, _ = _inputs(T, E, K, False, 10)
    whole, parts, part = (torch.empty(E + 1, dtype=torch.int64, device="cuda") for _ in range(3))
    loss, one = torch.empty(1, device="cuda"), torch.ones(1, device="cuda")
    d.balance_loss(T, logits, idx, None, loss, whole)
    parts.zero_()
    for lo, hi in ((0, 200), (200, 500)):
        d.balance_loss(hi - lo, logits[lo:hi], idx[lo:hi], None, loss, part)
        parts += part
    assert torch.equal(whole, parts)
    a, b = torch.empty((T, E), device="cuda"), torch.empty((T, E), device="cuda")
    d.balance_loss_backward(T, logits, whole, None, one, None, a)
    for lo, hi in ((0, 200), (200, 500)):
        d.balance_loss_backward(hi - lo, logits[lo:hi], parts, None, one, None, b[lo:hi])
    assert torch.equal(a, b)


def test_refusals():
    import torch
    from paper_2607_08782_b200.binding import DirectorError
    T, E, K = 16, 8, 2
    d = _director(T, E, K)
    logits, idx, _, added = _inputs(T, E, K, False, 11)
    loss, counts, out = torch.empty(1, device="cuda"), torch.empty(E + 1, dtype=torch.int64, device="cuda"), torch.empty((T, E), device="cuda")
    for bad, error in ((dict(logits=logits.double()), TypeError), (dict(logits=logits.t()), ValueError), (dict(logits=logits[:T - 1]), ValueError),
                       (dict(topk_idx=idx.long()), TypeError), (dict(topk_idx=idx[:, :1]), ValueError), (dict(loss=loss.double()), TypeError),
                       (dict(counts=counts[:E]), ValueError), (dict(counts=counts.int()), TypeError),
                       (dict(token_mask=torch.ones(T, device="cuda")), TypeError), (dict(token_mask=torch.ones(T - 1, dtype=torch.bool, device="cuda")), ValueError),
                       (dict(token_mask=torch.ones(T, dtype=torch.bool)), ValueError), (dict(T=T + 1), ValueError), (dict(T=0), DirectorError)):
        args = dict(dict(T=T, logits=logits, topk_idx=idx, token_mask=None, loss=loss, counts=counts), **bad)
        with pytest.raises(error):
            d.balance_loss(**args)
    one = torch.ones(1, device="cuda")
    room = torch.empty((2 * T, E), device="cuda")
    for bad, error in ((dict(dloss=one.double()), TypeError), (dict(added=added[:3]), ValueError), (dict(added=added.bfloat16()), TypeError),
                       (dict(dlogits=out[:3]), ValueError), (dict(dlogits=logits), DirectorError), (dict(T=0), DirectorError),
                       (dict(added=room[4:4 + T], dlogits=room[:T]), DirectorError), (dict(logits=room[8:8 + T], dlogits=room[:T]), DirectorError)):
        args = dict(dict(T=T, logits=logits, counts=counts, token_mask=None, dloss=one, added=None, dlogits=out), **bad)
        with pytest.raises(error):
            d.balance_loss_backward(**args)
