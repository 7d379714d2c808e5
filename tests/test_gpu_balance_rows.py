"""The balance term's gradient on rows that have none."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("E", [8, 61, 101, 256])              # rows read in 16-byte words and value by value, one lane to a row and many
@pytest.mark.parametrize("dloss", [float("inf"), -float("inf"), float("nan"), 3e38])
def test_rows_without_scores_get_what_is_added_whatever_the_losss_gradient(E, dloss):
    """A loss scale that overflowed: masked rows, and rows that are not finite, hold `added` and nothing else (3e38: dloss E/N leaves
    the range where N < E)."""
    import torch
    from paper_2607_08782_b200.binding import Director
    T, K = 7, 2
    d = Director(T, 256, 128, E, K, 0, 16, 16)
    g = torch.Generator(device="cuda").manual_seed(E)
    logits = torch.randn((T, E), generator=g, device="cuda")
    idx = logits.topk(K, dim=1).indices.int().contiguous()
    added = torch.randn((T, E), generator=g, device="cuda")
    mask = torch.tensor([1, 0, 1, 1, 0, 1, 0], dtype=torch.uint8, device="cuda")
    logits[3, 1], logits[5] = float("nan"), -float("inf")
    rows = [1, 3, 4, 5, 6]
    loss, counts = torch.empty(1, device="cuda"), torch.empty(E + 1, dtype=torch.int64, device="cuda")
    d.balance_loss(T, logits, idx, mask, loss, counts)
    dl = torch.tensor([dloss], device="cuda")
    for base in (added, None):
        out = torch.full((T, E), 7.0, device="cuda")
        d.balance_loss_backward(T, logits, counts, mask, dl, base, out)
        want = added[rows] if base is not None else torch.zeros((len(rows), E), device="cuda")
        assert torch.equal(out[rows], want)
    again = added.clone()                                     # added in place
    d.balance_loss_backward(T, logits, counts, mask, dl, again, again)
    assert torch.equal(again[rows], added[rows])
    none = torch.zeros((T,), dtype=torch.bool, device="cuda")  # no valid token at all
    d.balance_loss(T, logits, idx, none, loss, counts)
    d.balance_loss_backward(T, logits, counts, none, dl, added, out)
    assert torch.equal(out, added)
    assert d.last_status() == 8                               # the two rows that are not finite
