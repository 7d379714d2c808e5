"""Fine-tuning with the layer: its forward and backward pass as one torch.autograd function, and a small example that trains.

    python -m paper_2607_08782_b200.finetune [--steps 60] [--tokens 512] [--hidden 256] [--width 256] [--experts 8] [--topk 2]

The example takes a layer and its router, disturbs their weights, and trains the disturbed ones back to the originals' outputs,
under a placement with replicas: the gradients of a replicated expert are sums over its replicas, and the placement plays no
part in what is learnt."""
from __future__ import annotations

import argparse

import numpy as np
import torch
from torch.autograd.function import once_differentiable

from .layer import MoELayer

_WEIGHTS = ("w_gate", "w_up", "w_down", "ws_gate", "ws_up", "ws_down")


class _Layer(torch.autograd.Function):
    @staticmethod
    def forward(ctx, layer, token_src_rank, x, logits, *weights):
        T = x.shape[0]
        y = layer.forward_train(T, logits.contiguous(), x.contiguous(), token_src_rank).clone()
        ctx.layer = layer
        # What the backward pass reads of the caller's: autograd then notices where it was changed in place (x itself is read by
        # the shared experts alone, the routed experts' rows are copies).  The pass's number goes the same way, so that under
        # activation checkpointing it comes back as that of the pass that was run again.
        ctx.save_for_backward(torch.tensor(layer.passes, device="cpu"), *weights, *((x,) if layer.dims["S"] > 0 else ()))
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        kept, layer = int(ctx.saved_tensors[0]), ctx.layer         # the first access raises if a tensor was changed
        if layer.trained is None or layer.trained[3] != kept:
            raise RuntimeError("the layer keeps one forward pass: run its backward before the layer's next pass")
        g = layer.backward(dy.shape[0], dy.contiguous())
        weights = [g[n] for n in _WEIGHTS if n in g]
        return (None, None, *(t.clone() if need else None for t, need in zip([g["x"], g["logits"], *weights], ctx.needs_input_grad[2:])))


def moe_layer(layer: MoELayer, x: torch.Tensor, logits: torch.Tensor, token_src_rank: torch.Tensor | None = None) -> torch.Tensor:
    """y [T,H] of the layer for x [T,H] (bf16) and the router's logits [T,E] (fp32), differentiable in both and in the layer's
    weights (those that require a gradient).  Between the passes the experts' gate and up values are kept in 8 bits, which moves the
    gradients by under 1 %; the weights' come out in bf16.  The layer's placement has to be set.  One forward pass at a time is kept: the
    backward pass of a call has to run before the layer's next call (torch.utils.checkpoint lifts this: it runs the call again
    when its backward pass comes), and before the weights (with shared experts, x too) are changed
    in place.  token_src_rank (int32 [T]): the tokens' home ranks, for the locality-first choice of replicas (see MoELayer.dispatch)."""
    if x.dtype != torch.bfloat16 or logits.dtype != torch.float32:
        raise TypeError(f"x has to be bf16 and logits fp32, got {x.dtype} and {logits.dtype}")
    T, d = x.shape[0], layer.dims
    if x.shape != (T, d["H"]) or logits.shape != (T, d["E"]) or not 1 <= T <= d["T_max"]:
        raise ValueError(f"x {tuple(x.shape)} and logits {tuple(logits.shape)} do not fit the layer {d}")
    weights = layer.w + (layer.ws if d["S"] > 0 else ())
    return _Layer.apply(layer, token_src_rank, x, logits, *weights)


def make_layer(T, H, F, E, K, S, R, C, X, seed, scale=0.05) -> MoELayer:
    """A layer with random weights under the placement X."""
    g = torch.Generator(device="cuda").manual_seed(seed)

    def w(*shape):
        return (torch.randn(shape, generator=g, device="cuda") * scale).bfloat16()
    shared = (w(S * F, H), w(S * F, H), w(H, S * F)) if S > 0 else (None, None, None)
    layer = MoELayer(T, H, F, E, K, S, R, C, w(E, F, H), w(E, F, H), w(E, H, F), *shared)
    layer.set_placement(X)
    return layer


def train(steps=60, tokens=512, hidden=256, width=256, experts=8, topk=2, shared=0, lr=1e-3, seed=1, report=None):
    """Trains a disturbed copy of a layer back to it, with Adam on fp32 copies of the weights; returns the relative squared error
    of every step."""
    ranks = min(experts, max(4, -(-experts // 14)))              # a rank holds at most 16 experts
    C = -(-experts // ranks) + 2
    X = np.zeros((experts, ranks), dtype=np.uint8)
    X[np.arange(experts), np.arange(experts) * ranks // experts] = 1
    for e in range(min(2, experts)):
        X[e, ranks - 1] = 1                                      # the first experts have a replica on the last rank
    dims = (tokens, hidden, width, experts, topk, shared, ranks, C)
    teacher, student, noise = (make_layer(*dims, X, s) for s in (seed, seed, seed + 1))
    for w, n in zip(student.w + (student.ws if shared else ()), noise.w + (noise.ws if shared else ())):
        w.add_(n, alpha=0.5)
    g = torch.Generator(device="cuda").manual_seed(seed + 2)
    router_t = torch.randn((experts, hidden), generator=g, device="cuda") * hidden ** -0.5
    router = router_t + 0.1 * torch.randn((experts, hidden), generator=g, device="cuda") * hidden ** -0.5
    router.requires_grad_()
    weights = [w.requires_grad_() for w in student.w + (student.ws if shared else ())]
    masters = [w.detach().float() for w in weights]
    opt = torch.optim.Adam([router, *masters], lr=lr)
    losses = []
    for step in range(steps):
        x = torch.randn((tokens, hidden), generator=g, device="cuda").bfloat16()
        with torch.no_grad():
            target = teacher.forward(tokens, (x.float() @ router_t.t()).contiguous(), x, with_cost=False).float()
        y = moe_layer(student, x, x.float() @ router.t())
        loss = (y.float() - target).square().mean() / target.square().mean()
        grads = torch.autograd.grad(loss, [router, *weights])
        router.grad = grads[0]
        for m, gr in zip(masters, grads[1:]):
            m.grad = gr.float()
        opt.step()
        with torch.no_grad():
            for w, m in zip(weights, masters):
                w.copy_(m)
        losses.append(loss.item())
        if report and (step % 10 == 0 or step == steps - 1):
            report(f"step {step:4d}  loss {losses[-1]:.4f}")
    student.d.check_device_status()
    return losses


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, default in (("steps", 60), ("tokens", 512), ("hidden", 256), ("width", 256), ("experts", 8), ("topk", 2), ("shared", 0)):
        ap.add_argument(f"--{name}", type=int, default=default)
    train(**vars(ap.parse_args()), report=print)


if __name__ == "__main__":
    main()
