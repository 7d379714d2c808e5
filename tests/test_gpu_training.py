"""Gradient norm, clipping and AdamW against the definitions in fp64."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

# A thread adds up to 32 squares in fp32 (a square of a bf16 is exact, fma rounds once a term), all positive: 32 x 2^-24, halved by the
# square root, and the result's own rounding.
NORM_TOL = 2.0 ** -20 + 2.0 ** -24

SIZES = [1, 0, 7, 8, 9, 255, 2047, 2048, 2049, 8191, 8192, 8193, 100003, 3 * 256 * 257]


def _tensors(sizes, types, seed, scale=1.0, shift=0):
    """Tensors of normal values, `shift` elements behind an aligned address."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    out = []
    for i, n in enumerate(sizes):
        t = {"f": torch.float32, "b": torch.bfloat16}[types[i % len(types)]]
        room = (torch.randn((n + shift,), generator=g, device="cuda") * scale).to(t)
        out.append(room[shift:])
    return out


def _norm64(tensors):
    return math.sqrt(sum(float(t.double().square().sum()) for t in tensors if t is not None))


@pytest.mark.parametrize("shift", [0, 1, 3, 4])
@pytest.mark.parametrize("types", ["f", "b", "fb", "bbf"])
def test_norm(types, shift):
    from paper_2607_08782_b200.training import grad_norm
    for k in range(len(SIZES)):
        t = _tensors(SIZES[k:k + 1], types[-1], k, shift=shift)
        want = _norm64(t)
        assert abs(grad_norm(t).item() - want) <= NORM_TOL * want, SIZES[k]
    t = _tensors(SIZES, types, 50, shift=shift)
    want = _norm64(t)
    assert abs(grad_norm(t).item() - want) <= NORM_TOL * want


@pytest.mark.parametrize("count", [15, 63, 64, 65, 480, 481, 1000])
def test_norm_of_many_tensors_and_the_same_bits_again(count):
    import torch
    from paper_2607_08782_b200.training import TensorList, grad_norm
    t = TensorList(_tensors([(i * 37) % 3001 for i in range(count)], "fbb", count))
    got = grad_norm(t)
    want = _norm64(t)
    assert abs(got.item() - want) <= NORM_TOL * want and got.shape == ()
    assert all(torch.equal(grad_norm(t), got) for _ in range(5))


def test_norm_of_a_large_tensor():
    import torch
    from paper_2607_08782_b200.training import grad_norm
    n = (1 << 31) + 12345                                    # more elements than 31 bits count
    t = torch.ones((n,), dtype=torch.bfloat16, device="cuda")
    t[-1] = 3e4
    want = math.sqrt(n - 1 + float(t[-1].double()) ** 2)
    assert abs(grad_norm([t]).item() - want) <= NORM_TOL * want


@pytest.mark.parametrize("scale", [1e-38, 1e-30, 1e-19, 1e-12, 1e18, 1e25])
def test_squares_outside_fp32s_range(scale):
    import torch
    from paper_2607_08782_b200.training import grad_norm
    for types in ("f", "b"):
        t = _tensors([5000, 3], types, 1, scale=scale)
        want = _norm64(t)
        assert abs(grad_norm(t).item() - want) <= NORM_TOL * want
        t.append(torch.zeros(7000, device="cuda"))
        t.append(torch.full((1,), 1.0, device="cuda"))
        want = _norm64(t)
        assert abs(grad_norm(t).item() - want) <= NORM_TOL * want


def test_norm_of_nothing_and_of_values_that_are_not_finite():
    import torch
    from paper_2607_08782_b200.training import grad_norm
    assert grad_norm([]).item() == 0.0
    assert grad_norm([torch.empty(0, device="cuda"), torch.zeros(100, device="cuda")]).item() == 0.0
    for n in (1, 9000):
        t = torch.zeros(n, device="cuda")
        t[-1] = float("inf")
        assert grad_norm([t]).item() == math.inf
        t[0] = float("nan")
        assert math.isnan(grad_norm([t]).item())
    assert grad_norm([torch.full((10000,), 3e38, device="cuda")]).item() == math.inf          # the norm itself leaves the range


HALF = {"f": 2.0 ** -24, "b": 2.0 ** -8}


@pytest.mark.parametrize("shift", [0, 1, 4])
@pytest.mark.parametrize("src, dst", [("b", None), ("f", None), ("b", "f"), ("f", "f"), ("f", "b"), ("bf", "fb")])
@pytest.mark.parametrize("fraction", [0.3, 1.5])
def test_clip(src, dst, shift, fraction):
    import torch
    from paper_2607_08782_b200.training import clip_grads
    sizes = SIZES + [(i * 131) % 2500 for i in range(20)]
    for part in (sizes[:14], sizes):
        g = _tensors(part, src, 3, shift=shift)
        before = [t.clone() for t in g]
        out = None if dst is None else _tensors(part, dst, 4, shift=shift)
        want = _norm64(g)
        limit = fraction * want
        got = clip_grads(g, limit, out=out)
        assert abs(got.item() - want) <= NORM_TOL * want
        scale = min(1.0, limit / want)
        for i, (t, b) in enumerate(zip(g if out is None else out, before)):
            ref = b.double() * scale
            kind = (dst or src)[i % len(dst or src)]
            # the factor: the norm's error, its own rounding; the product's and the result's
            tol = HALF[kind] + 2.0 ** -24 + (NORM_TOL + 2.0 ** -23 if scale < 1 else 0.0)
            assert ((t.double() - ref).abs() <= tol * ref.abs() + 1e-40).all()
            if scale == 1.0 and dst is None:
                assert torch.equal(t, b)
        if out is not None:
            assert all(torch.equal(a, b) for a, b in zip(g, before))


@pytest.mark.parametrize("count", [64, 65, 361, 800])
def test_clip_of_many_tensors(count):
    import torch
    from paper_2607_08782_b200.training import clip_grads
    g = _tensors([(i * 61) % 2701 for i in range(count)], "fbb", count, shift=count % 3)
    want = _norm64(g)
    out = [torch.full_like(t, 7.0, dtype=torch.float32) for t in g]
    assert abs(clip_grads(g, 0.5 * want, out=out).item() - want) <= NORM_TOL * want
    for o, t in zip(out, g):
        ref = 0.5 * t.double()
        assert ((o.double() - ref).abs() <= (NORM_TOL + 4 * 2.0 ** -24) * ref.abs()).all()


def test_clip_in_place_into_itself_and_without_a_limit():
    import torch
    from paper_2607_08782_b200.training import TensorList, clip_grads
    g = _tensors([3000, 5], "bf", 5)
    before = [t.clone() for t in g]
    clip_grads(g, math.inf)
    assert all(torch.equal(a, b) for a, b in zip(g, before))
    both = TensorList(g)
    version = g[0]._version
    clip_grads(both, 1.0, out=both)
    assert g[0]._version > version, "autograd is told"
    assert abs(_norm64(g) - 1.0) < 2.0 ** -8
    assert clip_grads([], 1.0).item() == 0.0


@pytest.mark.parametrize("value", [float("inf"), float("nan")])
def test_clip_leaves_gradients_that_are_not_finite(value):
    import torch
    from paper_2607_08782_b200.training import clip_grads
    g = _tensors([3000, 500], "bf", 6)
    g[1][7] = value
    before = [t.clone() for t in g]
    got = clip_grads(g, 0.1)
    assert not math.isfinite(got.item())
    assert all(torch.equal(a.nan_to_num(1.0, 2.0, 3.0), b.nan_to_num(1.0, 2.0, 3.0)) for a, b in zip(g, before))


# ---- AdamW ---------------------------------------------------------------------------------------------------------


class _Reference:
    """AdamW in fp64, from the state that the optimizer is in; and how far fp32 arithmetic may be off it in one step."""

    def __init__(self, opt):
        self.w = [(m if m is not None else w.detach()).double() for w, m in zip(opt.weights, opt.masters)]
        self.m, self.v = [t.double() for t in opt.exp_avg], [t.double() for t in opt.exp_avg_sq]
        self.t, self.opt = int(opt.steps), opt

    def step(self, grads, lr, max_norm):
        o, (b1, b2) = self.opt, self.opt.betas
        norm = _norm64(grads)
        scale = min(1.0, max_norm / norm) if norm > 0 and math.isfinite(max_norm) else 1.0
        self.t += 1
        clip = NORM_TOL + 2.0 ** -23 if scale < 1 else 0.0
        eps = 2.0 ** -24
        for i, g in enumerate(grads):
            if g is None:
                continue
            x = g.double() * scale
            m, v, w = b1 * self.m[i] + (1 - b1) * x, b2 * self.v[i] + (1 - b2) * x * x, self.w[i]
            # m: the constants, two products, their sum, the factor.  v: one product more, the factor twice
            dm = 4 * eps * ((b1 * self.m[i]).abs() + ((1 - b1) * x).abs()) + clip * ((1 - b1) * x).abs()
            dv = 5 * eps * v + 2 * clip * (1 - b2) * x * x
            rate = lr / (1 - b1 ** self.t)
            den = (v / (1 - b2 ** self.t)).sqrt() + o.eps
            new = w - lr * o.weight_decay * w - rate * m / den
            # the quotient: m's error; of the root half of v's; six roundings (rate, product, root and its constant, eps, sum, quotient)
            rel_den = 0.5 * dv / v.clamp(min=1e-300)
            dw = rate * dm / den + (rate * m / den).abs() * (rel_den + 7 * eps) + 2 * eps * (w.abs() + new.abs()) + 2 * eps * lr * o.weight_decay * w.abs()
            self.check(o.exp_avg[i], m, dm)
            self.check(o.exp_avg_sq[i], v, dv)
            master = o.masters[i]
            if master is None:
                self.check(o.weights[i], new, dw)
            else:
                import torch
                self.check(master, new, dw)
                assert torch.equal(o.weights[i].detach(), master.to(torch.bfloat16)), "a bf16 weight is its master rounded"
        assert int(o.steps) == self.t
        return norm

    @staticmethod
    def check(got, want, tol):
        assert ((got.detach().double() - want).abs() <= tol + 1e-38).all()


def _optimizer(sizes, wtypes, gtypes, seed, shift=0, **kw):
    from paper_2607_08782_b200.training import AdamW
    opt = AdamW(_tensors(sizes, wtypes, seed, 0.05), **kw)
    return opt, lambda k: _tensors(sizes, gtypes, seed + 100 + k, 1e-2 * 10 ** (k % 3), shift=shift)


@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("wtypes, gtypes", [("b", "b"), ("f", "f"), ("b", "f"), ("f", "b"), ("bbf", "bbf")])
@pytest.mark.parametrize("decay, max_norm", [(0.0, math.inf), (0.1, 0.5), (0.01, 1e9)])
def test_steps(wtypes, gtypes, shift, decay, max_norm):
    opt, grads = _optimizer(SIZES, wtypes, gtypes, 1, shift, lr=3e-3, betas=(0.9, 0.95), eps=1e-8, weight_decay=decay, max_norm=max_norm)
    for k in range(4):
        ref, g = _Reference(opt), grads(k)
        norm = opt.step(g)
        want = ref.step(g, 3e-3, max_norm)
        assert norm is None if max_norm == math.inf else abs(norm.item() - want) <= NORM_TOL * want
    assert opt.last_status() == 0


@pytest.mark.parametrize("extra", [-2049, -1, 0, 1, 2049])
def test_sizes_where_one_launch_ends(extra):
    """A call is one launch up to two chunks (2048 weights of a step, 8192 gradients of clip_grads) for every SM."""
    import torch
    from paper_2607_08782_b200.training import clip_grads
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    for chunk in (2048, 8192):
        n = 2 * sms * chunk + extra
        sizes = [n - 3 * chunk, chunk, 2 * chunk]
        opt, grads = _optimizer(sizes, "bf", "fb", 21, lr=1e-3, max_norm=0.5)
        for k in range(2):
            ref, g = _Reference(opt), grads(k)
            opt.step(g)
            ref.step(g, 1e-3, 0.5)
        out = [torch.empty_like(t, dtype=torch.float32) for t in g]
        want = _norm64(g)
        assert abs(clip_grads(g, 0.25 * want, out=out).item() - want) <= NORM_TOL * want
        assert all(((o.double() - 0.25 * t.double()).abs() <= (NORM_TOL + 4 * 2.0 ** -24) * t.double().abs()).all() for o, t in zip(out, g))


@pytest.mark.parametrize("count", [17, 64, 65, 200, 203, 500])
def test_a_step_of_many_tensors(count):
    sizes = [(i * 53) % 2203 for i in range(count)]
    opt, grads = _optimizer(sizes, "bbf", "bf", 2, lr=1e-3, max_norm=0.1)
    for k in range(2):
        ref, g = _Reference(opt), grads(k)
        opt.step(g)
        ref.step(g, 1e-3, 0.1)


def test_offsets_past_31_bits():
    """A weight with more elements than 31 bits count, next to a small one: its first, middle and last elements."""
    import torch
    from paper_2607_08782_b200.training import AdamW, clip_grads
    n = (1 << 31) + 5003
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB")
    ends = [slice(0, 4099), slice((1 << 31) - 3000, (1 << 31) + 3000), slice(n - 4099, n)]
    g = [torch.zeros(n, dtype=torch.bfloat16, device="cuda"), torch.randn(1000, device="cuda")]
    w = [torch.zeros(n, dtype=torch.bfloat16, device="cuda"), torch.randn(1000, device="cuda")]
    for s in ends:
        g[0][s], w[0][s] = torch.randn(s.stop - s.start, device="cuda").bfloat16(), torch.randn(s.stop - s.start, device="cuda").bfloat16()
    opt = AdamW(w, lr=1e-2, max_norm=1.0)

    class Part:                                              # the optimizer as _Reference sees it, at some of the elements
        betas, eps, weight_decay = opt.betas, opt.eps, opt.weight_decay

        def __init__(self, s):
            self.weights, self.masters, self.exp_avg, self.exp_avg_sq = ([t[s]] for t in (w[0], opt.masters[0], opt.exp_avg[0], opt.exp_avg_sq[0]))
            self.steps = opt.steps
    parts = [(_Reference(Part(s)), s) for s in ends]
    want = _norm64([g[0][ends[0]], g[0][ends[1].start:], g[1]])          # the last two overlap
    got = opt.step(g)
    assert abs(got.item() - want) <= NORM_TOL * want
    for ref, s in parts:                                     # clipped by the norm of all
        part = g[0][s]
        ref.step([part], 1e-2, _norm64([part]) / want)
        ref.opt.steps = opt.steps
    assert not opt.exp_avg[0][5000:9000].any() and not w[0][5000:9000].any()
    before = [g[0][s].clone() for s in ends]
    clip_grads(g, 0.25 * want)
    for b, s in zip(before, ends):
        ref = b.double() * 0.25
        assert ((g[0][s].double() - ref).abs() <= (HALF["b"] + NORM_TOL + 2.0 ** -22) * ref.abs()).all()


def test_states_at_odd_addresses():
    """Weights that are views of one buffer, back to back."""
    import torch
    from paper_2607_08782_b200.training import AdamW
    for dtype in (torch.bfloat16, torch.float32):
        room = (torch.randn(20000, device="cuda") * 0.1).to(dtype)
        guard = room.clone()
        cuts = [0, 1, 4097, 4098, 9001, 19990]
        opt = AdamW([room[a:b] for a, b in zip(cuts, cuts[1:])], lr=1e-2, max_norm=1.0)
        g = _tensors([b - a for a, b in zip(cuts, cuts[1:])], "bf", 9)
        ref = _Reference(opt)
        opt.step(g)
        ref.step(g, 1e-2, 1.0)
        assert torch.equal(room[19990:], guard[19990:]), "what lies behind the last weight stays"


def test_weights_without_a_gradient_and_the_weights_own_gradients():
    import torch
    from paper_2607_08782_b200.training import AdamW
    w = [t.requires_grad_() for t in _tensors([300, 40, 5000], "bf", 10)]
    opt = AdamW(w, lr=1e-2, max_norm=1.0)
    w[0].grad, w[2].grad = (torch.randn_like(w[i]) for i in (0, 2))
    before = w[1].detach().clone()
    ref = _Reference(opt)
    norm = opt.step()
    ref.step([w[0].grad, None, w[2].grad], 1e-2, 1.0)
    assert torch.equal(w[1], before) and not opt.exp_avg[1].any()
    assert abs(norm.item() - _norm64([w[0].grad, w[2].grad])) <= 1e-5 * norm.item()
    for t in w:
        t.grad = None
    opt.step()
    assert int(opt.steps) == 2


@pytest.mark.parametrize("count", [3, 200])
@pytest.mark.parametrize("value", [float("inf"), float("nan")])
def test_a_step_that_is_not_finite_is_skipped(value, count):
    import torch
    from paper_2607_08782_b200.binding import DirectorError
    opt, grads = _optimizer([100 + i for i in range(count)], "bf", "bf", 11, lr=1e-2, max_norm=1.0)
    opt.step(grads(0))
    kept = [t.detach().clone() for t in (*opt.weights, *opt.exp_avg, *opt.exp_avg_sq, opt.steps)]
    bad = grads(1)
    bad[count // 2][50] = value
    norm = opt.step(bad)
    assert not math.isfinite(norm.item())
    assert all(torch.equal(a, b) for a, b in zip(kept, (*opt.weights, *opt.exp_avg, *opt.exp_avg_sq, opt.steps)))
    with pytest.raises(DirectorError):
        opt.check_status()
    opt.check_status()
    ref, g = _Reference(opt), grads(2)
    opt.step(g)
    ref.step(g, 1e-2, 1.0)


def test_gradients_of_zero_and_a_moment_of_zero():
    import torch
    opt, _ = _optimizer([5000, 3], "bf", "b", 12, lr=1e-2, max_norm=1.0)
    before = [w.clone() for w in opt.weights]
    norm = opt.step([torch.zeros_like(w) for w in opt.weights])
    assert norm.item() == 0.0 and all(torch.equal(a, b) for a, b in zip(before, opt.weights))


def test_far_steps_and_the_state_dict():
    import torch
    from paper_2607_08782_b200.training import AdamW
    opt, grads = _optimizer([4000, 17], "bf", "bf", 13, lr=1e-3, max_norm=1.0, betas=(0.9, 0.999))
    opt.step(grads(0))
    opt.steps.fill_(3_000_000_000)
    ref, g = _Reference(opt), grads(1)
    opt.step(g)
    ref.step(g, 1e-3, 1.0)
    twin = AdamW([torch.zeros_like(w) for w in opt.weights], lr=1e-3, max_norm=1.0, betas=(0.9, 0.999))
    for a, b in zip(twin.weights, opt.weights):
        a.copy_(b)
    twin.load_state_dict(opt.state_dict())
    for k in range(3):
        opt.step(grads(k))
        twin.step(grads(k))
    assert all(torch.equal(a, b) for a, b in zip((*opt.weights, *opt.exp_avg, *opt.exp_avg_sq, opt.steps, opt.masters[0]),
                                                 (*twin.weights, *twin.exp_avg, *twin.exp_avg_sq, twin.steps, twin.masters[0])))
    with pytest.raises(ValueError):
        twin.load_state_dict(dict(opt.state_dict(), exp_avg=opt.exp_avg[:1]))


def test_captured_steps_advance_and_follow_the_learning_rate():
    import torch
    from paper_2607_08782_b200.training import TensorList, clip_grads, grad_norm
    opt, grads = _optimizer([4000, 17, 70000], "bf", "bf", 14, lr=1e-3, max_norm=1.0)
    twin, _ = _optimizer([4000, 17, 70000], "bf", "bf", 14, lr=1e-3, max_norm=1.0)
    g = TensorList(grads(0))
    clipped = [torch.empty_like(t, dtype=torch.float32) for t in g]
    lr = torch.tensor([1e-3], device="cuda")
    norm0 = grad_norm(g)
    a, b = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(a):
        norm = opt.step(g, lr=lr)
    with torch.cuda.graph(b):
        norm2 = clip_grads(g, 0.5, out=clipped)
    other = torch.cuda.Stream()
    for k in range(5):
        for t, new in zip(g, grads(k)):
            t.copy_(new)
        lr.fill_(1e-3 / (k + 1))
        other.wait_stream(torch.cuda.current_stream())
        a.replay()
        with torch.cuda.stream(other):                        # two graphs at once, neither in the other's workspace
            b.replay()
        want = twin.step(g, lr=lr.item())
        torch.cuda.synchronize()
        assert torch.equal(norm, want) and torch.equal(norm2, want)
        assert all(torch.equal(x, y) for x, y in zip((*opt.weights, *opt.exp_avg, *opt.exp_avg_sq, opt.steps),
                                                     (*twin.weights, *twin.exp_avg, *twin.exp_avg_sq, twin.steps)))
        ref = [t.double() * min(1.0, 0.5 / want.item()) for t in g]
        assert all(((x.double() - y).abs() <= 2.0 ** -20 * y.abs()).all() for x, y in zip(clipped, ref))
    assert norm0.item() > 0


@pytest.mark.parametrize("sizes", [[4000, 17], [3_000_000, 5, 1_000_000], [(i * 37) % 901 for i in range(100)]])
def test_every_call_replayed_from_a_graph(sizes):
    """One launch, three, many tensors: norm, clipping in place and apart, a step, on inputs that changed since the capture."""
    import torch
    from paper_2607_08782_b200.training import TensorList, clip_grads, grad_norm
    g, h = TensorList(_tensors(sizes, "bf", 1)), TensorList(_tensors(sizes, "bf", 2))
    out = TensorList([torch.empty_like(t, dtype=torch.float32) for t in g])
    (opt, _), (twin, _) = (_optimizer(sizes, "bf", "bf", 16, lr=1e-3, max_norm=0.7) for _ in range(2))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        norms = [grad_norm(g), clip_grads(g, 0.9, out=out), clip_grads(h, 0.8), opt.step(g), grad_norm(h)]
    for k in range(3):
        new = [_tensors(sizes, "bf", 30 + k, 10.0 ** -k), _tensors(sizes, "bf", 40 + k)]
        for lst, values in zip((g, h), new):
            for t, v in zip(lst, values):
                t.copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        other = [torch.empty_like(t, dtype=torch.float32) for t in g]
        want = [grad_norm(new[0]), clip_grads(new[0], 0.9, out=other), clip_grads(new[1], 0.8), twin.step(new[0]), grad_norm(new[1])]
        assert all(torch.equal(a, b) for a, b in zip(norms, want))
        for mine, theirs in ((out, other), (h, new[1]), (opt.weights, twin.weights), (opt.exp_avg, twin.exp_avg), (opt.exp_avg_sq, twin.exp_avg_sq)):
            assert all(torch.equal(a, b) for a, b in zip(mine, theirs))
    assert int(opt.steps) == 3


def test_on_another_stream():
    import torch
    opt, grads = _optimizer([4000, 17, 700000], "bf", "bf", 15, lr=1e-3, max_norm=1.0)
    twin, _ = _optimizer([4000, 17, 700000], "bf", "bf", 15, lr=1e-3, max_norm=1.0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for k in range(3):
            norm = opt.step(grads(k))
    torch.cuda.current_stream().wait_stream(side)
    for k in range(3):
        want = twin.step(grads(k))
    assert torch.equal(norm, want) and all(torch.equal(a, b) for a, b in zip(opt.weights, twin.weights))


def test_refusals():
    import torch
    from paper_2607_08782_b200.binding import DirectorError
    from paper_2607_08782_b200.training import AdamW, TensorList, clip_grads, grad_norm
    t = torch.randn(64, device="cuda")
    for bad, error in ((t.double(), TypeError), (t.half(), TypeError), (t[::2], ValueError), (t.cpu(), ValueError)):
        with pytest.raises(error):
            grad_norm([t, bad])
    with pytest.raises(ValueError):
        clip_grads([t], 0.0)
    with pytest.raises(ValueError):
        clip_grads([t], math.nan)
    with pytest.raises(ValueError):
        clip_grads([t], 1.0, out=[torch.empty(63, device="cuda")])
    with pytest.raises(ValueError):
        clip_grads([t], 1.0, out=[])
    with pytest.raises(DirectorError):
        clip_grads([t, t], 1.0)
    with pytest.raises(DirectorError):
        clip_grads([t[:60]], 1.0, out=[t[4:]])
    with pytest.raises(ValueError):
        AdamW([None])
    opt = AdamW([t.clone(), t.clone().bfloat16()])
    for bad in ([t], [t, t[:3]], [t.view(8, 8), t]):
        with pytest.raises(ValueError):
            opt.step(bad)
    with pytest.raises(ValueError):
        opt.step([t, t], lr=torch.tensor([1e-3]))
    with pytest.raises(DirectorError):
        opt.step([t, t], lr=math.nan)
    with pytest.raises(DirectorError):
        AdamW([t, t]).step([t.clone(), t.clone()])
    with pytest.raises(DirectorError):
        AdamW([t]).step([t])
    with pytest.raises(DirectorError):
        AdamW([t], betas=(1.0, 0.9)).step([t.clone()])
    moved = [t.clone(), t.clone()]
    other = AdamW(moved)
    moved[1].data = t.clone()
    with pytest.raises(RuntimeError):
        other.step([t, t])
    assert int(other.steps) == 0
    assert int(opt.steps) == 0 and len(TensorList([t, None])) == 2


def test_the_c_entry_points_from_a_c_program(tmp_path):
    from test_gpu_c_abi import _build_and_run
    assert "0 mismatches" in _build_and_run(tmp_path, "step_from_c")


# ---- together ------------------------------------------------------------------------------------------------------


def _layer(seed=3, S=1):
    from paper_2607_08782_b200.finetune import make_layer
    X = np.zeros((8, 4), dtype=np.uint8)
    X[np.arange(8), np.arange(8) // 2] = 1
    X[0, 3] = 1
    return make_layer(96, 256, 256, 8, 2, S, 4, 3, X, seed)


def _batch(seed, T=96):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn((T, 8), generator=g, device="cuda"), torch.randn((T, 256), generator=g, device="cuda").bfloat16(),
            torch.randn((T, 256), generator=g, device="cuda").bfloat16())


def test_the_layers_gradients_with_the_balance_term():
    import torch
    layer = _layer()
    logits, x, dy = _batch(1)
    mask = torch.arange(96, device="cuda") % 5 != 0
    layer.forward_train(96, logits, x)
    plain = layer.backward(96, dy)["logits"].clone()
    layer.forward_train(96, logits, x)
    loss, counts = layer.balance_loss(96, logits, mask)
    weight = torch.tensor([0.3], device="cuda")
    both = layer.backward(96, dy, weight)["logits"].clone()
    alone = torch.empty((96, 8), device="cuda")
    layer.d.balance_loss_backward(96, logits, counts, mask, weight, plain, alone)
    assert torch.equal(both, alone) and int(counts[8]) == int(mask.sum()) and not torch.equal(both, plain)
    layer.d.check_device_status()
    with pytest.raises(RuntimeError):                        # no pass
        layer.backward(96, dy, weight)
    layer.forward_train(96, logits, x)
    with pytest.raises(RuntimeError):                        # the counts are another pass's
        layer.backward(96, dy, weight)
    with pytest.raises(ValueError):
        layer.balance_loss(96, logits[:95])
    with pytest.raises(RuntimeError):                        # the choices of the pass are 96 tokens'
        layer.balance_loss(95, logits)


def test_autograd_with_the_balance_term():
    import torch
    from torch.utils.checkpoint import checkpoint
    from paper_2607_08782_b200.finetune import moe_layer
    layer = _layer()
    for w in layer.w + layer.ws:
        w.requires_grad_()
    logits, x, dy = _batch(2)
    logits.requires_grad_()
    mask = (torch.arange(96, device="cuda") % 4 != 1).to(torch.uint8)

    def total(run):
        y, loss = run(lambda a, b: moe_layer(layer, a, b, balance=True, token_mask=mask), x, logits)
        return torch.autograd.grad((y.float() * dy.float()).sum() + 0.3 * loss.sum(), [logits, *layer.w, *layer.ws])
    got = total(lambda f, *a: f(*a))
    again = total(lambda f, *a: checkpoint(f, *a, use_reentrant=False))
    layer.forward_train(96, logits.detach(), x)
    layer.balance_loss(96, logits.detach(), mask)
    want = layer.backward(96, dy, torch.tensor([0.3], device="cuda"))
    for a, b, n in zip(got, again, ("logits", "w_gate", "w_up", "w_down", "ws_gate", "ws_up", "ws_down")):
        assert torch.equal(a, want[n]) and torch.equal(a, b), n
    y, loss = moe_layer(layer, x, logits, balance=True)      # the loss alone, and y alone
    only, = torch.autograd.grad(loss, [logits])
    assert only.abs().sum() > 0
    y, loss = moe_layer(layer, x, logits, balance=True)
    torch.autograd.grad(y.float().sum(), [logits])
    y, loss = moe_layer(layer, x, logits, balance=True)
    with torch.no_grad():
        logits.add_(1.0)
    with pytest.raises(RuntimeError):                        # the logits were changed in between
        loss.sum().backward()
    y, loss = moe_layer(layer, x, logits, balance=True)
    layer.balance_loss(96, logits, mask)
    with pytest.raises(RuntimeError):                        # the counts are no longer that term's
        loss.sum().backward()
    y = moe_layer(layer, x, logits)
    layer.balance_loss(96, logits, mask)                     # a pass without the term does not mind
    y.float().sum().backward()
    for bad in (dict(token_mask=mask), dict(balance=True, token_mask=mask[:5]), dict(balance=True, token_mask=mask.float())):
        with pytest.raises(ValueError):
            moe_layer(layer, x, logits, **bad)


def test_a_whole_step_captured_is_the_eager_step():
    """Forward pass, balance term, backward pass and update of a layer: replayed, it gives the eager steps' bits."""
    import torch
    from paper_2607_08782_b200.training import AdamW, TensorList
    names = ("w_gate", "w_up", "w_down", "ws_gate", "ws_up", "ws_down")
    eager, graphed = _layer(7), _layer(7)
    logits, x, dy = _batch(3)
    weight = torch.tensor([0.01], device="cuda")
    opts, lists, norms = [], [], []
    for layer in (eager, graphed):
        layer.enable_training()
        opts.append(AdamW(layer.w + layer.ws, lr=1e-3, weight_decay=0.1, max_norm=0.5))
        lists.append(TensorList([layer.grads[n] for n in names]))

    def step(layer, opt, grads):
        layer.forward_train(96, logits, x)
        layer.balance_loss(96, logits)
        layer.backward(96, dy, weight)
        return opt.step(grads)
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        assert torch.equal(step(eager, opts[0], lists[0]), step(graphed, opts[1], lists[1]))
    torch.cuda.current_stream().wait_stream(side)
    with torch.cuda.graph(graph):
        norm = step(graphed, opts[1], lists[1])
    for k in range(4):
        for t, new in zip((logits, x, dy), _batch(10 + k)):
            t.copy_(new)
        want = step(eager, opts[0], lists[0])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(norm, want)
        assert all(torch.equal(a, b) for a, b in zip(eager.w + eager.ws, graphed.w + graphed.ws))
    assert int(opts[1].steps) == 5
    graphed.d.check_device_status()
    opts[1].check_status()


def test_an_update_between_the_passes_is_noticed():
    import torch
    from paper_2607_08782_b200.finetune import moe_layer
    from paper_2607_08782_b200.training import AdamW
    layer = _layer(S=0)
    for w in layer.w:
        w.requires_grad_()
    logits, x, _ = _batch(4)
    y = moe_layer(layer, x, logits)
    AdamW(layer.w, lr=1e-3).step([torch.randn_like(w) for w in layer.w])
    with pytest.raises(RuntimeError):
        y.float().sum().backward()


@pytest.mark.parametrize("optimizer", ["torch", "adamw"])
def test_the_example_runs_with_each_of_them(optimizer):
    from paper_2607_08782_b200.finetune import train
    losses = train(steps=4, tokens=128, shared=1, optimizer=optimizer, max_norm=0.5, balance=0.01)
    assert np.isfinite(losses).all()
    import torch
    plain = train(steps=1, tokens=128, optimizer="torch")
    assert plain == train(steps=1, tokens=128, optimizer="adamw") and torch.isfinite(torch.tensor(plain)).all()
