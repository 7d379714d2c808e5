"""The backward pass as a user has it: MoELayer.forward_train / backward and the autograd function of finetune.py."""
import numpy as np
import pytest

from oracle import director_grad_oracle as gro
from oracle import director_oracle as orc
from paper_2607_08782_b200 import synth

pytestmark = pytest.mark.gpu

DIMS = dict(T=300, H=256, F=256, E=8, K=2, S=1, R=4, C=3)




def _layer(seed=3, **over):
    from paper_2607_08782_b200.finetune import make_layer
    d = {**DIMS, **over}
    X = np.zeros((d["E"], d["R"]), dtype=np.uint8)
    X[np.arange(d["E"]), np.arange(d["E"]) * d["R"] // d["E"]] = 1
    X[0, d["R"] - 1] = 1
    return make_layer(d["T"], d["H"], d["F"], d["E"], d["K"], d["S"], d["R"], d["C"], X, seed), X


def _np(t):
    return t.detach().double().cpu().numpy()


def _reference(layer, X, C, logits, x, dy):
    """The whole layer's gradients in fp64, from exact gate and up values."""
    idx, _, w = orc.route(logits.detach().cpu().numpy(), layer.dims["K"])
    disp = orc.dispatch(idx, X, C)
    inv, seg, slot = disp["inv_row"], disp["seg_offsets"], disp["slot_expert"]
    x64, dy64 = _np(x), _np(dy)
    wg, wu, wd = (_np(t) for t in layer.w)
    xp = x64[disp["row_token"]]
    yp, g, u = np.zeros_like(xp), np.zeros((len(xp), wg.shape[1])), np.zeros((len(xp), wg.shape[1]))
    for k, e in enumerate(slot):
        s = slice(int(seg[k]), int(seg[k + 1]))
        if e >= 0:
            yp[s], g[s], u[s] = gro.swiglu_ffn(xp[s], wg[e], wu[e], wd[e])
    dyp, dw = gro.combine_backward(dy64, yp, inv, w)
    dxp, *dweights = gro.expert_ffn_backward(xp, dyp, seg, slot, g, u, wg, wu, wd)
    out = dict(zip(("w_gate", "w_up", "w_down"), dweights))
    dx_shared = None
    if layer.dims["S"]:
        ws = [_np(t) for t in layer.ws]
        _, gs, us = gro.swiglu_ffn(x64, *ws)
        dx_shared, out["ws_gate"], out["ws_up"], out["ws_down"], *_ = gro.swiglu_ffn_backward(x64, dy64, gs, us, *ws)
    out["x"] = gro.dispatch_backward(dxp, inv, dx_shared)
    out["logits"] = gro.route_backward(idx, w, dw, logits.shape[1])
    return out


# What separates the layer from exact arithmetic: the 8-bit values (0.7 % of a value rms, see the checkpoint's tests) in every
# gradient, four roundings to bf16 (0.2 % rms each) on the way to x and the weights, yp's rounding in the logits'.  sqrt of the
# squares is 0.9 %; 2 % leaves a factor of two.
TOL = 0.02


@pytest.mark.parametrize("S", [0, 2])
@pytest.mark.parametrize("T", [1, 5, 300])
def test_layer_gradients_match_the_definition(T, S):
    import torch
    layer, X = _layer(S=S)
    g = torch.Generator(device="cuda").manual_seed(T)
    x = torch.randn((T, 256), generator=g, device="cuda").bfloat16()
    logits = torch.randn((T, 8), generator=g, device="cuda")
    dy = torch.randn((T, 256), generator=g, device="cuda").bfloat16()
    y = layer.forward_train(T, logits, x).clone()
    layer.d.set_ffn_variant(6)
    assert torch.equal(y, layer.forward(T, logits, x, with_cost=False)), "the training forward's outputs are the inference forward's"
    layer.forward_train(T, logits, x)
    got = layer.backward(T, dy)
    layer.d.check_device_status()
    want = _reference(layer, X, DIMS["C"], logits, x, dy)
    assert sorted(got) == sorted(want)
    for name, ref in want.items():
        val = _np(got[name]).reshape(ref.shape)
        assert np.linalg.norm(val - ref) <= TOL * np.linalg.norm(ref) + 1e-30, name


def test_autograd_gives_the_same_gradients_and_accumulates():
    import torch
    from paper_2607_08782_b200.finetune import moe_layer
    layer, _ = _layer(S=1)
    T = 64
    x = torch.randn((T, 256), device="cuda").bfloat16().requires_grad_()
    logits = torch.randn((T, 8), device="cuda").requires_grad_()
    for w in layer.w + layer.ws:
        w.requires_grad_()
    dy = torch.randn((T, 256), device="cuda").bfloat16()
    moe_layer(layer, x, logits).backward(dy)
    first = [t.grad.clone() for t in (x, logits, *layer.w, *layer.ws)]
    layer.forward_train(T, logits.detach(), x.detach())
    direct = layer.backward(T, dy)
    for a, n in zip(first, ("x", "logits", "w_gate", "w_up", "w_down", "ws_gate", "ws_up", "ws_down")):
        assert torch.equal(a, direct[n]), n
    moe_layer(layer, x, logits).backward(dy)
    assert torch.equal(layer.w[0].grad, first[2] + first[2])


def test_only_what_needs_a_gradient_gets_one_and_order_is_checked():
    import torch
    from paper_2607_08782_b200.finetune import moe_layer
    layer, _ = _layer(S=0)
    x = torch.randn((8, 256), device="cuda").bfloat16()
    logits = torch.randn((8, 8), device="cuda").requires_grad_()
    y1 = moe_layer(layer, x, logits)
    y2 = moe_layer(layer, x, logits)
    y2.float().sum().backward()
    assert logits.grad is not None and layer.w[0].grad is None
    with pytest.raises(RuntimeError):
        y1.float().sum().backward()
    with pytest.raises(RuntimeError):
        layer.backward(8, x)
    layer.forward_train(8, logits.detach(), x)
    with pytest.raises(RuntimeError):
        layer.backward(7, x[:7])
    layer.forward(8, logits.detach(), x)                  # a serving pass in between has taken the buffers
    with pytest.raises(RuntimeError):
        layer.backward(8, x)
    with pytest.raises(TypeError):
        moe_layer(layer, x.float(), logits)
    with pytest.raises(ValueError):
        moe_layer(layer, x, logits[:, :7])


def test_backward_on_another_stream_and_in_a_graph():
    import torch
    layer, _ = _layer(S=1)
    T = 96
    x = torch.randn((T, 256), device="cuda").bfloat16()
    logits = torch.randn((T, 8), device="cuda")
    dy = torch.randn((T, 256), device="cuda").bfloat16()
    layer.forward_train(T, logits, x)
    want = {n: t.clone() for n, t in layer.backward(T, dy).items()}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer.forward_train(T, logits, x)
        got = {n: t.clone() for n, t in layer.backward(T, dy).items()}
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(want[n], got[n]) for n in want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.forward_train(T, logits, x)
        views = layer.backward(T, dy)
    for _ in range(3):
        for v in views.values():
            v.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(want[n], views[n]) for n in want)
    layer.d.check_device_status()


@pytest.mark.parametrize("shared", [0, 1])
def test_the_example_learns(shared):
    from paper_2607_08782_b200.finetune import train
    losses = train(steps=40, tokens=256, shared=shared)
    assert np.mean(losses[-5:]) < 0.7 * np.mean(losses[:3]), losses
