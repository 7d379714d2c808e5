"""What the training calls have to notice: indexes out of range, buffers that are no longer a forward pass's own, arguments of
the wrong kind."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def _layer(S=1, F=256, seed=3):
    from paper_2607_08782_b200.finetune import make_layer
    return make_layer(64, 256, F, 8, 2, S, 4, 3, _placement(0), seed)


def _placement(which):
    """Eight experts on four ranks, expert `which` with a replica on another rank."""
    X = np.zeros((8, 4), dtype=np.uint8)
    X[np.arange(8), np.arange(8) // 2] = 1
    X[which, 3 - which // 2] = 1
    return X


def _inputs(seed=0, T=64):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn((T, 8), generator=g, device="cuda"), torch.randn((T, 256), generator=g, device="cuda").bfloat16(),
            torch.randn((T, 256), generator=g, device="cuda").bfloat16())


@pytest.mark.parametrize("K", [1, 2, 3, 6, 8])
@pytest.mark.parametrize("H", [256, 768])
def test_dispatch_backward_skips_and_reports_a_row_past_the_end(K, H):
    import torch
    from paper_2607_08782_b200.binding import Director
    T = 9
    A = T * K
    d = Director(T, H, 128, 8, K, 0, 2, 8)
    room = torch.full((A + 4, H), 100.0, dtype=torch.bfloat16, device="cuda")     # the rows behind the batch's are no part of it
    room[:A] = (torch.arange(A, device="cuda") % 16).to(torch.bfloat16).unsqueeze(1)
    inv = torch.randperm(A, generator=torch.Generator().manual_seed(K)).int().view(T, K).cuda()
    add = torch.full((T, H), 0.5, dtype=torch.bfloat16, device="cuda")
    for bad in (A, A + 3):
        table = inv.clone()
        table[4, K - 1] = bad
        for shared in (None, add):
            dx = torch.full((T, H), 7.0, dtype=torch.bfloat16, device="cuda")
            d.dispatch_backward(T, room, table, shared, dx)
            assert d.last_status() == 7 and d.last_status() == 0
            rows = room[:A].float()[table.clamp(max=A - 1).long()] * (table < A).unsqueeze(-1)
            assert torch.equal(dx.float(), rows.sum(1) + (0.5 if shared is not None else 0.0))    # small whole numbers: exact
    table[4, K - 1] = -1                                                          # nothing there is no error
    d.dispatch_backward(T, room, table, None, dx)
    assert d.last_status() == 0


# ---- the workspace -------------------------------------------------------------------------------------------------


def _freed_garbage():
    """Leaves small pieces of device memory behind that are not zero, for the next small allocations to find."""
    import ctypes
    import torch
    cuda = ctypes.CDLL("libcudart.so.12")
    pieces = []                                           # 4 MB of them: every hole in the small blocks is filled once
    for _ in range(8192):
        p = ctypes.c_void_p()
        assert cuda.cudaMalloc(ctypes.byref(p), ctypes.c_size_t(512)) == 0
        assert cuda.cudaMemset(p, 0x01, ctypes.c_size_t(512)) == 0
        pieces.append(p)
    torch.cuda.synchronize()
    for p in pieces:
        assert cuda.cudaFree(p) == 0


def _busy(stream, ms):
    """Ordinary work for about `ms` milliseconds."""
    import torch
    with torch.cuda.stream(stream):
        a = torch.zeros(1 << 28, device="cuda")            # 1 GB: about 0.3 ms a pass
        for _ in range(int(ms / 0.3)):
            a.add_(1.0)


def _train_once(layer, logits, x, dy):
    layer.forward_train(64, logits, x)
    return {n: t.clone() for n, t in layer.backward(64, dy).items()}


def test_the_first_training_step_runs_beside_a_busy_default_stream():
    """The training workspace is ready when the call that makes it returns, whatever the default stream still has to do: torch's
    side streams do not wait for it."""
    import torch
    logits, x, dy = _inputs()
    want = _train_once(_layer(F=4096), logits, x, dy)
    side = torch.cuda.Stream()
    for _ in range(3):
        layer = _layer(F=4096)                           # more work items than the GPU has SMs: the counters matter
        torch.cuda.synchronize()
        _freed_garbage()
        _busy(torch.cuda.default_stream(), 200)
        with torch.cuda.stream(side):
            got = _train_once(layer, logits, x, dy)
        side.synchronize()
        assert all(torch.equal(want[n], got[n]) for n in want)
        torch.cuda.synchronize()
        assert layer.d.last_status() == 0


def test_a_context_made_beside_a_busy_default_stream_is_ready():
    import torch
    from paper_2607_08782_b200.layer import MoELayer
    logits, x, dy = _inputs()
    quiet = _layer(F=4096)
    want = _train_once(quiet, logits, x, dy)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        _freed_garbage()
        _busy(torch.cuda.default_stream(), 200)
        with torch.cuda.stream(side):
            layer = MoELayer(64, 256, 4096, 8, 2, 1, 4, 3, *quiet.w, *quiet.ws)
            layer.set_placement(_placement(0))
            got = _train_once(layer, logits, x, dy)
            assert layer.d.last_status() == 0
        side.synchronize()
        assert all(torch.equal(want[n], got[n]) for n in want)
        torch.cuda.synchronize()


# ---- the layer's passes --------------------------------------------------------------------------------------------


def test_backward_notices_another_placement():
    import torch
    layer = _layer()
    logits, x, dy = _inputs()
    layer.forward_train(64, logits, x)
    want = {n: t.clone() for n, t in layer.backward(64, dy).items()}
    layer.forward_train(64, logits, x)
    layer.set_placement(_placement(5))
    with pytest.raises(RuntimeError, match="placement"):
        layer.backward(64, dy)
    layer.set_placement(_placement(0))                    # filled anew: not the tables that the forward pass ran with
    with pytest.raises(RuntimeError, match="placement"):
        layer.backward(64, dy)
    with pytest.raises(Exception):
        layer.set_placement(np.zeros((8, 4), dtype=np.uint8))       # refused: the placement stays
    layer.forward_train(64, logits, x)
    with pytest.raises(Exception):
        layer.set_placement(np.zeros((8, 4), dtype=np.uint8))
    got = layer.backward(64, dy)
    assert all(torch.equal(want[n], got[n]) for n in want)
    layer.d.check_device_status()


def test_backward_notices_another_placement_slot():
    import torch
    layer = _layer()
    logits, x, dy = _inputs()
    layer.d.reserve_placements(2)
    layer.forward_train(64, logits, x)
    want = {n: t.clone() for n, t in layer.backward(64, dy).items()}
    layer.d.select_placement(1)
    layer.set_placement(_placement(5))
    layer.d.select_placement(0)
    layer.forward_train(64, logits, x)
    layer.d.select_placement(1)
    with pytest.raises(RuntimeError, match="placement"):
        layer.backward(64, dy)
    layer.d.select_placement(0)                           # back at the forward pass's tables
    got = layer.backward(64, dy)
    assert all(torch.equal(want[n], got[n]) for n in want)
    layer.d.check_device_status()


def test_a_replayed_serving_pass_takes_the_buffers():
    import torch
    layer = _layer()
    logits, x, dy = _inputs()
    other = _inputs(seed=1)
    graph = layer.capture(64, other[0], other[1])
    layer.forward_train(64, logits, x)
    graph.replay()
    with pytest.raises(RuntimeError):
        layer.backward(64, dy)
    y = layer.y[:64].clone()
    assert torch.equal(y, layer.forward(64, other[0], other[1])), "the replay is the pass that was captured"
    layer.forward_train(64, logits, x)
    layer.backward(64, dy)
    layer.d.check_device_status()


def test_autograd_notices_a_training_pass_of_the_layer_itself():
    """The buffers then hold another pass's values, of the same size."""
    from paper_2607_08782_b200.finetune import moe_layer
    layer = _layer()
    logits, x, dy = _inputs()
    logits.requires_grad_()
    y = moe_layer(layer, x, logits)
    other = _inputs(seed=1)
    layer.forward_train(64, other[0], other[1])
    with pytest.raises(RuntimeError):
        y.float().sum().backward()
    layer.backward(64, dy)                                # which is still there for its own backward pass
    layer.d.check_device_status()


@pytest.mark.parametrize("what", ["x", "expert", "shared"])
def test_autograd_notices_what_was_changed_in_place(what):
    import torch
    from paper_2607_08782_b200.finetune import moe_layer
    layer = _layer(S=1)
    logits, x, _ = _inputs()
    logits.requires_grad_()
    for w in layer.w + layer.ws:
        w.requires_grad_()
    y = moe_layer(layer, x, logits)
    with torch.no_grad():
        {"x": x, "expert": layer.w[1], "shared": layer.ws[2]}[what].mul_(0.5)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.float().sum().backward()
    moe_layer(layer, x, logits).float().sum().backward()
    assert logits.grad is not None


def test_without_shared_experts_x_may_be_written_to():
    """The routed experts' rows are copies: a residual connection in place is as good as any other."""
    import torch
    from paper_2607_08782_b200.finetune import moe_layer
    layer = _layer(S=0)
    logits, x, dy = _inputs()
    for w in layer.w:
        w.requires_grad_()
    want = torch.autograd.grad(moe_layer(layer, x, logits), layer.w, dy)
    stream = x.clone()
    y = moe_layer(layer, stream, logits)
    stream += y.detach()
    assert all(torch.equal(a, b) for a, b in zip(want, torch.autograd.grad(y, layer.w, dy)))


def test_a_pass_without_a_backward_pass_keeps_no_graph_alive():
    import gc
    import weakref
    import torch
    from paper_2607_08782_b200.finetune import moe_layer

    class Probe(torch.autograd.Function):
        @staticmethod
        def forward(ctx, t):
            return t * 1

        @staticmethod
        def backward(ctx, g):
            return g
    layer = _layer()
    logits, leaf, _ = _inputs()
    x = Probe.apply(leaf.requires_grad_())
    node = weakref.ref(x.grad_fn)
    y = moe_layer(layer, x, logits)
    del x, y
    gc.collect()
    assert node() is None, "the layer holds on to the graph of its input"


def test_forward_train_refuses_what_it_would_misread():
    import torch
    from paper_2607_08782_b200.finetune import moe_layer
    layer = _layer()
    logits, x, dy = _inputs()
    for bad in (dict(logits=logits.double()), dict(x=x.float()), dict(x=x.half())):
        with pytest.raises(TypeError):
            layer.forward_train(64, **{"logits": logits, "x": x, **bad})
    for bad in (dict(logits=logits[:63]), dict(x=x[:63]), dict(logits=logits.t().contiguous().t()), dict(x=x.t().contiguous().t()),
                dict(logits=logits.cpu()), dict(x=x.cpu())):
        with pytest.raises(ValueError):
            layer.forward_train(64, **{"logits": logits, "x": x, **bad})
    with pytest.raises(ValueError):
        moe_layer(layer, x, logits.cpu())
    with pytest.raises(ValueError):
        moe_layer(layer, x.cpu(), logits)
    with pytest.raises(RuntimeError):                     # no pass has run
        layer.backward(64, dy)
    layer.forward_train(64, logits, x)
    layer.backward(64, dy)
    layer.d.check_device_status()


def test_training_under_locality_first_takes_the_tokens_home_ranks():
    """Which replica serves a token plays no part in what is learnt: a token's own gradients have the same bits, the weights' sums
    come in another order (two roundings to bf16 of fp32 sums)."""
    import torch
    from paper_2607_08782_b200.finetune import moe_layer
    layer = _layer()
    layer.set_replica_policy(1)
    logits, x, dy = _inputs()
    layer.forward_train(64, logits, x)
    seg = layer.seg_offsets.clone()
    want = {n: t.clone() for n, t in layer.backward(64, dy).items()}
    home = (3 - torch.arange(64, device="cuda") // 16).int()
    layer.forward_train(64, logits, x, token_src_rank=home)
    tables = [t.clone() for t in (layer.dest_rank, layer.inv_row, layer.seg_offsets)]
    got = {n: t.clone() for n, t in layer.backward(64, dy).items()}
    assert not torch.equal(seg, tables[2]), "the home ranks count"
    layer.dispatch(64, x, token_src_rank=home)
    assert all(torch.equal(a, b) for a, b in zip(tables, (layer.dest_rank, layer.inv_row, layer.seg_offsets)))
    for n in want:
        if n in ("x", "logits"):
            assert torch.equal(want[n], got[n]), n
        else:
            assert (got[n].double() - want[n].double()).norm() <= 2.0 ** -7 * want[n].double().norm(), n
    logits.requires_grad_()
    y = moe_layer(layer, x, logits, home)
    assert torch.equal(torch.autograd.grad(y, logits, dy)[0], got["logits"])
    with pytest.raises(TypeError):
        layer.forward_train(64, logits.detach(), x, token_src_rank=home.long())
    with pytest.raises(ValueError):
        layer.forward_train(64, logits.detach(), x, token_src_rank=home[:63])
    layer.d.check_device_status()


def test_under_activation_checkpointing_calls_may_overlap():
    """The forward pass runs again before the backward pass needs its buffers, inside a block of other operations or alone."""
    import torch
    from torch.utils.checkpoint import checkpoint
    from paper_2607_08782_b200.finetune import moe_layer
    layer = _layer()
    for w in layer.w + layer.ws:
        w.requires_grad_()

    def alone(x, logits):
        return moe_layer(layer, x, logits)

    def block(x, logits):
        return x + torch.tanh(moe_layer(layer, torch.sin(x), logits * 2))
    batches = [_inputs(seed=k) for k in range(3)]
    for fn in (alone, block):
        want, got = [], []
        for logits, x, dy in batches:
            leaves = [x.clone().requires_grad_(), logits.clone().requires_grad_()]
            want.append(torch.autograd.grad(fn(*leaves), [*leaves, *layer.w, *layer.ws], dy))
        for reentrant in (False, True):
            leaves = [[x.clone().requires_grad_(), logits.clone().requires_grad_()] for logits, x, _ in batches]
            ys = [checkpoint(fn, *lv, use_reentrant=reentrant) for lv in leaves]
            if reentrant:                                 # which hands gradients to .grad alone
                for (_, _, dy), y in zip(batches, ys):
                    y.backward(dy)
                assert all(torch.equal(a.grad, b) for lv, w in zip(leaves, want) for a, b in zip(lv, w))
            else:
                for (_, _, dy), y, lv, w in zip(batches, ys, leaves, want):
                    assert all(torch.equal(a, b) for a, b in zip(torch.autograd.grad(y, [*lv, *layer.w, *layer.ws], dy), w))
    layer.d.check_device_status()


def test_a_refused_dy_leaves_the_pass_as_it_is():
    import torch
    layer = _layer()
    logits, x, dy = _inputs()
    want = _train_once(layer, logits, x, dy)
    layer.forward_train(64, logits, x)
    for bad, error in ((dy.float(), TypeError), (dy[:63], ValueError), (dy.t(), ValueError), (dy.cpu(), ValueError)):
        with pytest.raises(error):
            layer.backward(64, bad)
    got = layer.backward(64, dy)
    assert all(torch.equal(want[n], got[n]) for n in want)
    layer.d.check_device_status()
