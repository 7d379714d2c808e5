"""bf16 weights that are written between the steps of an optimizer that holds their masters."""
import pytest

pytestmark = pytest.mark.gpu


def _made(seed=1, sizes=(3000, 5, 700), **kw):
    import torch
    from paper_2607_08782_b200.training import AdamW
    g = torch.Generator(device="cuda").manual_seed(seed)
    kinds = (torch.bfloat16, torch.float32, torch.bfloat16)
    w = [(torch.randn(n, generator=g, device="cuda") * 0.1).to(k) for n, k in zip(sizes, kinds)]
    return AdamW(w, lr=1e-2, **kw), lambda: [torch.randn(n, generator=g, device="cuda") for n in sizes]


def _kept(opt):
    return [t.clone() for t in (*opt.weights, *[m for m in opt.masters if m is not None], *opt.exp_avg, *opt.exp_avg_sq, opt.steps)]


@pytest.mark.parametrize("steps_before", [0, 2])
def test_loaded_weights_are_not_overwritten_from_the_masters_of_before(steps_before):
    import torch
    opt, grads = _made()
    for _ in range(steps_before):
        opt.step(grads())
    loaded = torch.randn(700, device="cuda").bfloat16()
    opt.weights[2].copy_(loaded)                              # as a module's load_state_dict does
    kept = _kept(opt)
    for _ in range(2):
        with pytest.raises(RuntimeError, match="weight 2"):
            opt.step(grads())
    assert all(torch.equal(a, b) for a, b in zip(_kept(opt), kept)), "nothing was done"
    opt.masters_from_weights()
    assert torch.equal(opt.masters[2], loaded.float()) and opt.masters[1] is None
    g = grads()
    opt.step(g)
    assert int(opt.steps) == steps_before + 1
    # from there it goes on as any weight: of its first three steps none is longer than 1.01 lr (Cauchy's inequality on the moments'
    # weights), and the result, shorter than |w| + 0.02, is rounded
    assert ((opt.weights[2].float() - loaded.float()).abs() <= 1.02e-2 + 2.0 ** -8 * (loaded.float().abs() + 0.02)).all()
    assert torch.equal(opt.weights[2], opt.masters[2].bfloat16())
    opt.step(grads())


def test_going_back_to_the_masters():
    import torch
    opt, grads = _made()
    opt.step(grads())
    before = opt.weights[0].clone()
    opt.weights[0].zero_()
    with pytest.raises(RuntimeError):
        opt.step(grads())
    opt.load_state_dict(opt.state_dict())
    assert torch.equal(opt.weights[0], before)
    opt.step(grads())


def test_weights_swapped_out_and_back_go_on():
    """Averaged weights for an evaluation: the steps go on as if nothing had been."""
    import torch
    (opt, grads), (twin, other) = _made(max_norm=1.0), _made(max_norm=1.0)
    for k in range(3):
        assert torch.equal(opt.step(grads()), twin.step(other()))
        saved = [w.clone() for w in opt.weights]
        for w in opt.weights:
            w.fill_(float("nan") if k == 1 else 3.0)
        for w, s in zip(opt.weights, saved):
            w.copy_(s)
    assert all(torch.equal(a, b) for a, b in zip(_kept(opt), _kept(twin)))


def test_fp32_weights_and_parts_of_a_buffer_are_taken_as_they_are():
    import torch
    from paper_2607_08782_b200.training import AdamW
    opt, grads = _made()
    opt.weights[1].fill_(2.0)                                 # it is its own master
    opt.step(grads())
    assert (opt.weights[1] - 2.0).abs().max() < 0.1
    room = torch.randn(1000, device="cuda").bfloat16()        # two optimizers, and something else, in one buffer
    a, b = AdamW([torch.nn.Parameter(room[:300])], lr=1e-2), AdamW([room[300:900]], lr=1e-2)
    for _ in range(3):
        a.step([torch.randn(300, device="cuda")])
        b.step([torch.randn(600, device="cuda")])
        room[900:].add_(1.0)
    assert int(a.steps) == int(b.steps) == 3


def test_masters_that_are_nan_and_inference_tensors():
    import torch
    from paper_2607_08782_b200.training import AdamW
    opt, grads = _made()
    bad = grads()
    bad[0][7] = float("nan")
    opt.step(bad)                                             # no limit: it reaches the weights
    assert opt.weights[0].isnan().sum() == 1
    opt.weights[2].add_(0.0)                                  # written, and the same
    opt.step(grads())
    with torch.inference_mode():
        w = torch.randn(64, device="cuda").bfloat16()
        inference = AdamW([w], lr=1e-2)
        inference.step([torch.randn(64, device="cuda")])
        inference.step([torch.randn(64, device="cuda")])


def test_captured_steps_and_eager_ones_in_turn():
    import torch
    opt, grads = _made()
    g = grads()
    opt.step(g)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        opt.step(g)
    for _ in range(3):
        graph.replay()
        opt.step(g)
    assert int(opt.steps) == 7
    opt.weights[0].mul_(2.0)
    graph = torch.cuda.CUDAGraph()
    with pytest.raises(RuntimeError, match="before this capture"):
        with torch.cuda.graph(graph):
            opt.step(g)
    opt.masters_from_weights()
    opt.step(g)
    assert int(opt.steps) == 8
