"""The balance term through the layer: which batch's choices it counts."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def _layer(T_max=96):
    from paper_2607_08782_b200.finetune import make_layer
    X = np.zeros((8, 4), dtype=np.uint8)
    X[np.arange(8), np.arange(8) // 2] = 1
    return make_layer(T_max, 256, 256, 8, 2, 0, 4, 3, X, 5)


def _batch(T, seed):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn((T, 8), generator=g, device="cuda"), torch.randn((T, 256), generator=g, device="cuda").bfloat16()


def _counts(logits):
    import torch
    return torch.bincount(logits.topk(2, dim=1).indices.view(-1), minlength=8)


@pytest.mark.parametrize("how", ["route", "forward", "forward without costs", "graph"])
def test_a_batch_is_not_larger_than_what_was_routed(how):
    import torch
    layer = _layer()
    (large, x), (small, xs) = _batch(96, 1), _batch(40, 2)
    with pytest.raises(RuntimeError):                        # nothing routed yet
        layer.balance_loss(1, large)
    graph = layer.capture(40, small, xs) if how == "graph" else None
    layer.route(96, large)
    assert torch.equal(layer.balance_loss(96, large)[1][:8], _counts(large))
    if how == "route":
        layer.route(40, small)
    elif how == "graph":
        graph.replay()
    else:
        layer.forward(40, small, xs, with_cost=how == "forward")
    for T in (41, 96):                                       # the choices from place 40 on are the batch's before
        with pytest.raises(RuntimeError):
            layer.balance_loss(T, large)
    assert torch.equal(layer.balance_loss(40, small)[1][:8], _counts(small))
    assert torch.equal(layer.balance_loss(17, small)[1][:8], _counts(small[:17]))       # its first tokens
    layer.forward_train(96, large, x)
    assert torch.equal(layer.balance_loss(96, large)[1][:8], _counts(large))
    layer.d.check_device_status()


@pytest.mark.parametrize("end", ["backward", "backward without the term", "route", "forward", "forward_train", "graph", "nothing to keep"])
def test_the_batch_is_let_go_with_its_pass(end):
    """Logits and mask are held for the backward pass and not beyond it."""
    import gc
    import weakref

    import torch
    layer = _layer()
    (other, xo), (logits, x) = _batch(40, 3), _batch(96, 4)
    dy, weight = torch.randn((96, 256), device="cuda").bfloat16(), torch.full((1,), 0.1, device="cuda")
    graph = layer.capture(40, other, xo) if end == "graph" else None
    mask = torch.ones(96, dtype=torch.uint8, device="cuda")
    if end == "nothing to keep":
        layer.route(96, logits)
    else:
        layer.forward_train(96, logits, x)
    layer.balance_loss(96, logits, mask)
    held = weakref.ref(mask)
    del mask
    gc.collect()
    assert (held() is not None) == (end != "nothing to keep"), "the backward pass reads it"
    if end.startswith("backward"):
        layer.backward(96, dy, weight if end == "backward" else None)
    elif end == "route":
        layer.route(40, other)
    elif end == "forward":
        layer.forward(40, other, xo)
    elif end == "forward_train":
        layer.forward_train(40, other, xo)
    elif end == "graph":
        graph.replay()
    gc.collect()
    assert held() is None and layer.balanced is None
    layer.d.check_device_status()
