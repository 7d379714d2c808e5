"""The backward pass's kernels against the fp64 definitions (oracle/director_grad_oracle.py).

Bounds are worst-case bounds of the arithmetic, element by element: a rounding to bf16 (eight significant bits) is off by at most
2^-8 of the value, an fp32 sum of n terms by at most n 2^-23 of the sum of magnitudes (2^-23 and not 2^-24, since the tensor cores may
truncate)."""
import numpy as np
import pytest

from oracle import director_grad_oracle as gro
from oracle import director_oracle as orc
from paper_2607_08782_b200 import synth

pytestmark = pytest.mark.gpu

U16, U32 = 2.0 ** -8, 2.0 ** -23


def _dev(a, dtype=None):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(dtype)


def _bf16(rng, *shape, scale=1.0):
    """(CUDA bf16 tensor, the same values in fp64)."""
    import torch
    t = (torch.from_numpy(rng.normal(size=shape) * scale)).to(torch.bfloat16)
    return t.cuda(), t.double().numpy()


def _np(t):
    return t.double().cpu().numpy()


def _context(T, H=256, F=128, E=8, K=2, S=0, R=2, C=8):
    from paper_2607_08782_b200.binding import Director
    return Director(T, H, F, E, K, S, R, C)


def _same_bits(a, b):
    import torch
    return torch.equal(a.view(torch.uint8), b.view(torch.uint8))


@pytest.mark.parametrize("T,H,K", [(1, 256, 1), (1, 4096, 8), (2, 512, 3), (33, 768, 2), (257, 256, 5), (1000, 1280, 8), (129, 4096, 6)])
def test_combine_backward(T, H, K):
    import torch
    rng = np.random.default_rng(T * 31 + H + K)
    d = _context(T, H=H, K=K)
    A = T * K
    dy, dy64 = _bf16(rng, T, H)
    yp, yp64 = _bf16(rng, A, H)
    inv = rng.permutation(A).reshape(T, K).astype(np.int32)
    w = rng.random((T, K)).astype(np.float32)
    dyp, dw = torch.full((A, H), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((T, K), 7.0, device="cuda")
    d.combine_backward(T, dy, yp, _dev(inv), _dev(w), dyp, dw)
    ref_dyp, ref_dw = gro.combine_backward(dy64, yp64, inv, w)
    assert (np.abs(_np(dyp) - ref_dyp) <= (U16 + U32) * np.abs(ref_dyp)).all()
    _, mag = gro.combine_backward(np.abs(dy64), np.abs(yp64), inv, w)
    assert (np.abs(_np(dw) - ref_dw) <= (H // 32 + 8) * U32 * mag).all()
    again_dyp, again_dw = torch.empty_like(dyp), torch.empty_like(dw)
    d.combine_backward(T, dy, yp, _dev(inv), _dev(w), again_dyp, again_dw)
    assert _same_bits(dyp, again_dyp) and _same_bits(dw, again_dw)
    assert d.last_status() == 0


def test_combine_backward_skips_rows_that_are_not_there():
    import torch
    rng = np.random.default_rng(5)
    T, K, H = 8, 2, 256
    d = _context(T, H=H, K=K)
    dy, dy64 = _bf16(rng, T, H)
    yp, yp64 = _bf16(rng, T * K, H)
    inv = rng.permutation(T * K).reshape(T, K).astype(np.int32)
    w = np.ones((T, K), dtype=np.float32)
    skipped = int(inv[3, 1])
    inv[3, 1] = -1
    dyp, dw = torch.full((T * K, H), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((T, K), 7.0, device="cuda")
    d.combine_backward(T, dy, yp, _dev(inv), _dev(w), dyp, dw)
    assert d.last_status() == 0
    assert float(dw[3, 1]) == 0.0 and bool((dyp[skipped] == 7.0).all())
    inv[4, 0] = T * K                                    # past the end: skipped and reported
    d.combine_backward(T, dy, yp, _dev(inv), _dev(w), dyp, dw)
    assert float(dw[4, 0]) == 0.0 and d.last_status() == 7 and d.last_status() == 0


def test_combine_backward_carries_infinities_and_nans():
    import torch
    rng = np.random.default_rng(6)
    T, K, H = 5, 2, 512
    d = _context(T, H=H, K=K)
    dy, _ = _bf16(rng, T, H)
    yp, _ = _bf16(rng, T * K, H)
    inv = np.arange(T * K, dtype=np.int32).reshape(T, K)
    dy[1, 300] = float("inf")
    yp[7, 5] = float("nan")                              # row of token 3
    dyp, dw = torch.empty_like(yp), torch.empty((T, K), device="cuda")
    d.combine_backward(T, dy, yp, _dev(inv), torch.ones((T, K), device="cuda"), dyp, dw)
    assert torch.isinf(dyp[2, 300]) and torch.isinf(dyp[3, 300]) and int(torch.isinf(dyp).sum()) == 2
    bad = ~torch.isfinite(dw)
    assert bad[1].all() and bad[3, 1] and int(bad.sum()) == 3


@pytest.mark.parametrize("T,H,K,shared", [(1, 256, 1, False), (1, 4096, 8, True), (33, 768, 3, True), (257, 512, 5, False),
                                          (1001, 256, 7, True), (500, 2048, 6, True), (64, 2048, 4, False)])
def test_dispatch_backward(T, H, K, shared):
    import torch
    rng = np.random.default_rng(T * 37 + H + K)
    d = _context(T, H=H, K=K)
    A = T * K
    dxp, dxp64 = _bf16(rng, A, H)
    add, add64 = _bf16(rng, T, H) if shared else (None, None)
    inv = rng.permutation(A).reshape(T, K).astype(np.int32)
    if T > 2:
        inv[1, 0] = -1
    dx = torch.full((T, H), 7.0, dtype=torch.bfloat16, device="cuda")
    d.dispatch_backward(T, dxp, _dev(inv), add, dx)
    ref = gro.dispatch_backward(dxp64, inv, add64)
    mag = gro.dispatch_backward(np.abs(dxp64), inv, None if add64 is None else np.abs(add64))
    assert (np.abs(_np(dx) - ref) <= U16 * np.abs(ref) + (K + 2) * U32 * mag).all()
    assert d.last_status() == 0


@pytest.mark.parametrize("T,E,K", [(1, 1, 1), (1, 256, 8), (15, 7, 3), (16, 60, 4), (17, 61, 8), (777, 60, 4), (1000, 128, 8),
                                   (33, 3, 2), (513, 255, 1)])
def test_route_backward(T, E, K):
    import torch
    rng = np.random.default_rng(T + E + K)
    d = _context(T, E=E, K=K, R=16, C=16)
    logits = rng.normal(size=(T, E)).astype(np.float32)
    idx, w = torch.empty((T, K), dtype=torch.int32, device="cuda"), torch.empty((T, K), device="cuda")
    d.route(T, _dev(logits), idx, w)
    dw = rng.normal(size=(T, K)).astype(np.float32)
    pad = 64                                             # canaries around the output
    buf = torch.full((T * E + 2 * pad,), 7.0, device="cuda")
    dl = buf[pad:pad + T * E].view(T, E)
    d.route_backward(T, idx, w, _dev(dw), dl)
    assert bool((buf[:pad] == 7).all()) and bool((buf[pad + T * E:] == 7).all())
    w64, i64 = _np(w), idx.cpu().numpy()
    ref = gro.route_backward(i64, w64, dw.astype(np.float64), E)
    mag = np.zeros((T, E))
    np.put_along_axis(mag, i64.astype(np.int64), w64 * (np.abs(dw) + np.sum(w64 * np.abs(dw), 1, keepdims=True)), axis=1)
    assert (np.abs(_np(dl) - ref) <= (K + 4) * U32 * mag).all()
    assert d.last_status() == 0


def test_route_backward_is_the_derivative_of_route():
    """Kernel against kernel: the gate's weights at logits moved a little along a direction (the choice unchanged)."""
    import torch
    rng = np.random.default_rng(9)
    T, E, K, eps = 300, 16, 4, 2.0 ** -7
    d = _context(T, E=E, K=K)
    base = np.argsort(rng.random((T, E)), axis=1) * 0.5          # logits half apart: a move of 2^-7 leaves the order
    direction = rng.uniform(-1, 1, size=(T, E))
    idx, w = torch.empty((T, K), dtype=torch.int32, device="cuda"), [torch.empty((T, K), device="cuda") for _ in range(3)]
    for k, s in enumerate((0.0, eps, -eps)):
        d.route(T, _dev((base + s * direction).astype(np.float32)), idx, w[k])
    dw = rng.normal(size=(T, K)).astype(np.float32)
    dl = torch.empty((T, E), device="cuda")
    d.route_backward(T, idx, w[0], _dev(dw), dl)
    slope = np.sum(dw * (_np(w[1]) - _np(w[2])), axis=1) / (2 * eps)
    # third derivatives of a softmax are below 1 per unit direction: eps^2 of the sum of |dw|; plus fp32 noise over 2 eps
    tol = (eps ** 2 + 8 * U32 / eps) * np.abs(dw).sum(1)
    assert (np.abs(slope - np.sum(_np(dl) * direction, axis=1)) <= tol).all()


def test_route_backward_reports_an_index_out_of_range():
    import torch
    d = _context(4, E=8, K=2)
    idx = torch.tensor([[0, 1], [2, 8], [-1, 3], [4, 5]], dtype=torch.int32, device="cuda")
    w, dw = torch.full((4, 2), 0.5, device="cuda"), torch.tensor([[1.0, 0.0]] * 4, device="cuda")
    dl = torch.empty((4, 8), device="cuda")
    d.route_backward(4, idx, w, dw, dl)
    assert d.last_status() == 7
    assert dl[1].tolist() == [0, 0, 0.25, 0, 0, 0, 0, 0] and dl[2].tolist() == [0, 0, 0, -0.25, 0, 0, 0, 0]


# ---- the forward pass of training ----------------------------------------------------------------------------------


class Ffn:
    """A grouped FFN over given segment lengths: inputs on the device and in fp64, and buffers for both passes."""

    def __init__(self, seed, lengths, X, C, H, F, K=1, S=0, scale=0.05):
        import torch
        rng = np.random.default_rng(seed)
        E, R = X.shape
        T = -(-int(sum(lengths)) // K)
        assert T * K == sum(lengths), "the segments hold T*K rows"
        self.T, self.A, self.H, self.F, self.E, self.S, self.K = T, T * K, H, F, E, S, K
        self.d = _context(T, H=H, F=F, E=E, K=K, S=S, R=R, C=C)
        self.d.set_placement(X)
        self.seg64 = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
        _, _, self.slot_expert = _tables(X, C)
        self.seg = _dev(self.seg64)
        self.xp, self.xp64 = _bf16(rng, self.A, H, scale=0.5)
        (self.wg, self.wg64), (self.wu, self.wu64) = _bf16(rng, E, F, H, scale=scale), _bf16(rng, E, F, H, scale=scale)
        self.wd, self.wd64 = _bf16(rng, E, H, F, scale=scale)
        dev = "cuda"
        self.codes = torch.full((self.A, F, 2), 99, dtype=torch.int8, device=dev)
        self.exps = torch.full((F // 16, self.A, 2), 99, dtype=torch.uint8, device=dev)
        self.yp = torch.full((self.A, H), 7.0, dtype=torch.bfloat16, device=dev)
        if S:
            self.x, self.x64 = _bf16(rng, T, H, scale=0.5)
            (self.sg, self.sg64), (self.su, self.su64) = _bf16(rng, S * F, H, scale=scale), _bf16(rng, S * F, H, scale=scale)
            self.sd, self.sd64 = _bf16(rng, H, S * F, scale=scale)
            self.codes_s = torch.full((T, S * F, 2), 99, dtype=torch.int8, device=dev)
            self.exps_s = torch.full((S * F // 16, T, 2), 99, dtype=torch.uint8, device=dev)
            self.y_s = torch.full((T, H), 7.0, dtype=torch.bfloat16, device=dev)

    def checkpoint(self):
        shared = (self.x, self.sg, self.su, self.sd, self.codes_s, self.exps_s, self.y_s) if self.S else ()
        self.d.expert_ffn_checkpoint(self.T, self.xp, self.seg, self.wg, self.wu, self.wd, self.codes, self.exps, self.yp, *shared)

    def preactivations(self, magnitudes=False):
        x, wg, wu = (np.abs(a) for a in (self.xp64, self.wg64, self.wu64)) if magnitudes else (self.xp64, self.wg64, self.wu64)
        g, u = np.zeros((self.A, self.F)), np.zeros((self.A, self.F))
        for k, e in enumerate(self.slot_expert):
            s = slice(int(self.seg64[k]), int(self.seg64[k + 1]))
            if e >= 0:
                g[s], u[s] = x[s] @ wg[e].T, x[s] @ wu[e].T
        return g, u


def _tables(X, C):
    """hosted / replicas / expert of every slot (-1 unused)."""
    E, R = X.shape
    slot_expert = np.full(R * C, -1)
    for j in range(R):
        for p, e in enumerate(np.nonzero(X[:, j])[0]):
            slot_expert[j * C + p] = e
    return None, None, slot_expert


def _kept(codes, exps, which):
    return gro.checkpoint_decode(codes[:, :, which].cpu().numpy(), exps[:, :, which].cpu().numpy())


def _check_kept(v64, mag, H, kept, label):
    """kept against the exact v64: half a step of the block's power of two (2^-7 of its largest, 1 % for values held at 127),
    on top of the fp32 sum of H products."""
    acc = H * U32 * mag
    big = np.repeat((np.abs(v64) + acc).reshape(len(v64), -1, 16).max(-1), 16, axis=1)
    assert (np.abs(kept - v64) <= 2.0 ** -7 * 1.01 * big + acc).all(), label


def _layout(name):
    """(lengths per slot, X, C): what a placement and a batch can come to."""
    one = np.ones((1, 1), dtype=np.uint8)
    if name == "one token":
        return [1], one, 1
    if name == "ragged":                                  # 4 experts on 2 ranks, odd lengths around the tile sizes
        X = np.array([[1, 0], [1, 0], [0, 1], [0, 1]], dtype=np.uint8)
        return [257, 31, 33, 255], X, 2
    if name == "empty experts and slots":                 # expert 1 has no rows, slot 2 of every rank is unused
        X = np.array([[1, 0], [1, 0], [0, 1], [0, 1]], dtype=np.uint8)
        return [63, 0, 0, 1, 128, 0], X, 3
    if name == "replicas":                                # expert 0 on three ranks, expert 2 on two
        X = np.array([[1, 1, 1], [1, 0, 0], [0, 1, 1]], dtype=np.uint8)
        return [100, 17, 99, 300, 98, 301], X, 2
    if name == "long":
        X = np.array([[1], [1]], dtype=np.uint8)
        return [1500, 77], X, 2
    raise ValueError(name)


LAYOUTS = ["one token", "ragged", "empty experts and slots", "replicas", "long"]


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("H,F,S", [(256, 128, 0), (512, 384, 1), (768, 256, 2)])
def test_checkpoint_forward(layout, H, F, S):
    import torch
    lengths, X, C = _layout(layout)
    f = Ffn(len(layout) + H, lengths, X, C, H, F, S=S)
    f.checkpoint()
    assert f.d.last_status() == 0
    # the outputs are the bits of the inference forward on the tensor cores
    yp, ys = torch.empty_like(f.yp), torch.empty((f.T, H), dtype=torch.bfloat16, device="cuda")
    f.d.set_ffn_variant(6)
    f.d.expert_ffn(f.T, f.xp, f.seg, f.wg, f.wu, f.wd, yp, *((f.x, f.sg, f.su, f.sd, ys) if S else ()))
    assert _same_bits(f.yp, yp) and (not S or _same_bits(f.y_s, ys))
    g, u = f.preactivations()
    mg, mu = f.preactivations(True)
    _check_kept(g, mg, H, _kept(f.codes, f.exps, 0), "gate")
    _check_kept(u, mu, H, _kept(f.codes, f.exps, 1), "up")
    if S:
        for w64, which in ((f.sg64, 0), (f.su64, 1)):
            _check_kept(f.x64 @ w64.T, np.abs(f.x64) @ np.abs(w64).T, H, _kept(f.codes_s, f.exps_s, which), f"shared {which}")
    # decoding is exact in bf16
    gate, up = (torch.empty((f.A, F), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    f.d.checkpoint_decode(f.A, F, f.codes, f.exps, gate, up)
    assert np.array_equal(_np(gate), _kept(f.codes, f.exps, 0)) and np.array_equal(_np(up), _kept(f.codes, f.exps, 1))
    # and again
    codes, exps = f.codes.clone(), f.exps.clone()
    f.checkpoint()
    assert torch.equal(codes, f.codes) and torch.equal(exps, f.exps)


def test_checkpoint_with_the_up_array_in_front():
    """The gate|up tile interleaves the two arrays by address; the pairs of the checkpoint are (gate, up) either way."""
    import torch
    lengths, X, C = _layout("ragged")
    f = Ffn(3, lengths, X, C, 256, 256)
    both = torch.empty((2, *f.wg.shape), dtype=torch.bfloat16, device="cuda")
    for first in (0, 1):
        both[first], both[1 - first] = f.wg, f.wu
        f.wg, f.wu = both[first], both[1 - first]
        f.codes.fill_(99)
        f.checkpoint()
        g, u = f.preactivations()
        mg, mu = f.preactivations(True)
        _check_kept(g, mg, 256, _kept(f.codes, f.exps, 0), f"gate, first={first}")
        _check_kept(u, mu, 256, _kept(f.codes, f.exps, 1), f"up, first={first}")
        f.wg, f.wu = both[first].clone(), both[1 - first].clone()


def test_checkpoint_of_rows_that_are_not_finite_or_zero_or_tiny():
    import torch
    lengths, X, C = _layout("ragged")
    f = Ffn(8, lengths, X, C, 256, 128)
    f.xp[5] = 0.0
    f.xp[6, 17] = float("nan")
    f.xp[300, 200] = float("inf")
    f.xp[301] = f.xp[301] * 1e-30
    f.xp64 = _np(f.xp)
    f.checkpoint()
    e = f.exps.cpu().numpy()
    assert (e[:, 6] == 255).all() and (e[:, 300] == 255).all()
    ok = np.ones(f.A, dtype=bool)
    ok[[6, 300]] = False
    assert (e[:, ok] < 255).all()
    assert not f.codes[5].any() and (e[:, 5] == 1).all()
    g, u = _kept(f.codes, f.exps, 0), _kept(f.codes, f.exps, 1)
    assert np.isnan(g[~ok]).all() and np.isnan(u[~ok]).all()
    with np.errstate(all="ignore"):
        g64, _ = f.preactivations()
        mag, _ = f.preactivations(True)
    _check_kept(g64[ok], mag[ok], 256, g[ok], "finite rows")
    assert np.abs(g[301]).max() > 0


# ---- refusals ------------------------------------------------------------------------------------------------------


def test_refusals_of_the_moving_kernels():
    import torch
    from paper_2607_08782_b200.binding import DirectorError
    T, H, K = 4, 256, 2
    d = _context(T, H=H, K=K)
    b = torch.zeros((T * K, H), dtype=torch.bfloat16, device="cuda")
    t = torch.zeros((T, H), dtype=torch.bfloat16, device="cuda")
    inv, w = torch.zeros((T, K), dtype=torch.int32, device="cuda"), torch.zeros((T, K), device="cuda")
    dl = torch.zeros((T, 8), device="cuda")
    codes, exps = torch.zeros((T, 32, 2), dtype=torch.int8, device="cuda"), torch.zeros((2, T, 2), dtype=torch.uint8, device="cuda")
    g = torch.zeros((T, 32), dtype=torch.bfloat16, device="cuda")
    for bad in (0, T + 1, -1):
        with pytest.raises((DirectorError, ValueError)):
            d.combine_backward(bad, t, b, inv, w, b.clone(), w.clone())
        with pytest.raises((DirectorError, ValueError)):
            d.dispatch_backward(bad, b, inv, None, t)
        with pytest.raises((DirectorError, ValueError)):
            d.route_backward(bad, inv, w, w.clone(), dl)
    with pytest.raises(TypeError):
        d.combine_backward(T, t.float(), b, inv, w, b.clone(), w.clone())
    with pytest.raises(TypeError):
        d.route_backward(T, inv.long(), w, w.clone(), dl)
    with pytest.raises(ValueError):                       # a strided view
        d.dispatch_backward(T, torch.zeros((T * K, 2 * H), dtype=torch.bfloat16, device="cuda")[:, :H], inv, None, t)
    with pytest.raises(ValueError):
        d.dispatch_backward(T, b[:-1], inv, None, t)
    with pytest.raises(DirectorError):                    # not 16-byte aligned
        d.route_backward(T, inv, w, w.clone(), torch.zeros(T * 8 + 1, device="cuda")[1:])
    for rows, F in ((0, 32), (T, 0), (T, 24)):
        with pytest.raises(DirectorError):
            d.checkpoint_decode(rows, F, codes, exps, g, g.clone())
    lib, null = d.lib, None
    assert lib.director_combine_backward(d._ctx, T, null, null, null, null, null, null, null) == 1
    assert lib.director_dispatch_backward(None, T, null, null, null, null, null) == 1
    assert lib.director_route_backward(d._ctx, T, null, null, null, null, null) == 1
    assert lib.director_checkpoint_decode(d._ctx, T, 32, null, null, null, null, null) == 1
    assert d.last_status() == 0


def test_refusals_of_the_checkpoint_forward():
    import torch
    from paper_2607_08782_b200.binding import DirectorError
    lengths, X, C = _layout("ragged")
    f = Ffn(3, lengths, X, C, 256, 128)
    args = [f.xp, f.seg, f.wg, f.wu, f.wd, f.codes, f.exps, f.yp]
    with pytest.raises(DirectorError):
        f.d.expert_ffn_checkpoint(f.T + 1, torch.zeros((f.A + 1, 256), dtype=torch.bfloat16, device="cuda"), f.seg, f.wg, f.wu, f.wd,
                                  torch.zeros((f.A + 1, 128, 2), dtype=torch.int8, device="cuda"),
                                  torch.zeros((8, f.A + 1, 2), dtype=torch.uint8, device="cuda"),
                                  torch.zeros((f.A + 1, 256), dtype=torch.bfloat16, device="cuda"))
    for k, wrong in ((0, f.xp.float()), (5, f.codes.view(torch.uint8)), (6, f.exps.view(torch.int8)), (1, f.seg.long())):
        with pytest.raises(TypeError):
            f.d.expert_ffn_checkpoint(f.T, *args[:k], wrong, *args[k + 1:])
    with pytest.raises(ValueError):
        f.d.expert_ffn_checkpoint(f.T, *args[:5], f.codes[:-1], *args[6:])
    with pytest.raises(DirectorError) as e:               # one array as gate and up
        f.d.expert_ffn_checkpoint(f.T, f.xp, f.seg, f.wg, f.wg, f.wd, f.codes, f.exps, f.yp)
    assert e.value.status == 5
    f.d.set_ffn_variant(1)
    with pytest.raises(DirectorError) as e:
        f.d.expert_ffn_checkpoint(f.T, *args)
    assert e.value.status == 5
    fresh = _context(8)
    assert fresh.lib.director_expert_ffn_checkpoint(fresh._ctx, 8, *([f.xp.data_ptr()] * 8), *([None] * 8)) == 2   # no placement


# ---- gradients of the expert FFN -----------------------------------------------------------------------------------


class FfnGradient(Ffn):
    """An Ffn whose forward has run, with gradients to be filled; canaries are 7."""

    def __init__(self, *a, dy_scale=0.1, **k):
        import torch
        super().__init__(*a, **k)
        rng = np.random.default_rng(a[0] + 999)
        self.checkpoint()
        self.dyp, self.dyp64 = _bf16(rng, self.A, self.H, scale=dy_scale)
        self.dxp = torch.full_like(self.xp, 7.0)
        self.dw = [torch.full_like(w, 7.0) for w in (self.wg, self.wu, self.wd)]
        if self.S:
            self.dy, self.dy64 = _bf16(rng, self.T, self.H, scale=dy_scale)
            self.dx_s = torch.full_like(self.x, 7.0)
            self.dws = [torch.full_like(w, 7.0) for w in (self.sg, self.su, self.sd)]

    def backward(self):
        shared = (self.x, self.dy, self.codes_s, self.exps_s, self.sg, self.su, self.sd, self.dx_s, *self.dws) if self.S else ()
        self.d.expert_ffn_backward(self.T, self.xp, self.dyp, self.seg, self.codes, self.exps, self.wg, self.wu, self.wd, self.dxp,
                                   *self.dw, *shared)

    def outputs(self):
        return [self.dxp, *self.dw] + ([self.dx_s, *self.dws] if self.S else [])


def _check_expert(label, x, dy, g, u, wg, wu, wd, got):
    """One expert's gradients (numpy: dx, dwg, dwu, dwd) against the definition.  Bounds: da and the products are fp32 sums; s =
    sigmoid(g) is off by a few units in the last place, more for large |g| (the argument of the exponential); dg, du and act
    are rounded to bf16; so are the results."""
    n, H, F = len(x), x.shape[1], g.shape[1]
    dx, dwg, dwu, dwd, dg, du, act = gro.swiglu_ffn_backward(x, dy, g, u, wg, wu, wd)
    s = 1 / (1 + np.exp(-g))
    eps = (8 + 1.2 * np.abs(g)) * U32
    da, t_da = dy @ wd, H * U32 * (np.abs(dy) @ np.abs(wd))
    slope = s * (1 + g * (1 - s))
    t_dg = U16 * np.abs(dg) * 1.01 + 1.01 * (np.abs(u * slope) * t_da + np.abs(da * u) * eps * s * (1 + 2 * np.abs(g)))
    t_du = U16 * np.abs(du) * 1.01 + 1.01 * np.abs(g) * s * (t_da + np.abs(da) * eps)
    t_act = (U16 + 2 * eps) * np.abs(act) * 1.01
    ax, ay, ag, au, aw = np.abs(x), np.abs(dy), np.abs(wg), np.abs(wu), n + 64
    for name, ref, val, tol in (
            ("dx", dx, got[0], t_dg @ ag + t_du @ au + 2 * F * U32 * (np.abs(dg) @ ag + np.abs(du) @ au)),
            ("dw_gate", dwg, got[1], t_dg.T @ ax + aw * U32 * (np.abs(dg).T @ ax)),
            ("dw_up", dwu, got[2], t_du.T @ ax + aw * U32 * (np.abs(du).T @ ax)),
            ("dw_down", dwd, got[3], ay.T @ t_act + aw * U32 * (ay.T @ np.abs(act)))):
        assert (np.abs(val - ref) <= (U16 * np.abs(ref) + tol) * 1.02 + 1e-30).all(), f"{label}: {name}"
        # errors of single roundings do not add up in step: the whole is off by about as much as one of them
        if ref.size > 512:
            assert np.linalg.norm(val - ref) <= U16 * np.linalg.norm(ref) + 1e-30, f"{label}: {name} as a whole"


def _check_backward(f, skip=()):
    g, u = _kept(f.codes, f.exps, 0), _kept(f.codes, f.exps, 1)
    dxp, dw = _np(f.dxp), [_np(w) for w in f.dw]
    for e in range(f.E):
        rows = np.concatenate([np.arange(f.seg64[k], f.seg64[k + 1]) for k in range(len(f.slot_expert)) if f.slot_expert[k] == e]
                              or [np.zeros(0)]).astype(int)
        if e in skip:
            continue
        if not len(rows):
            assert all(not w[e].any() for w in dw), f"expert {e} has no rows"
            continue
        _check_expert(f"expert {e}", f.xp64[rows], f.dyp64[rows], g[rows], u[rows], f.wg64[e], f.wu64[e], f.wd64[e],
                      (dxp[rows], dw[0][e], dw[1][e], dw[2][e]))
    if f.S:
        _check_expert("shared", f.x64, f.dy64, _kept(f.codes_s, f.exps_s, 0), _kept(f.codes_s, f.exps_s, 1), f.sg64, f.su64, f.sd64,
                      [_np(t) for t in (f.dx_s, *f.dws)])


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("H,F,S", [(256, 128, 0), (512, 384, 1), (768, 256, 2)])
def test_ffn_backward(layout, H, F, S):
    lengths, X, C = _layout(layout)
    f = FfnGradient(len(layout) + H, lengths, X, C, H, F, S=S)
    f.d.reserve_training()
    f.backward()
    assert f.d.last_status() == 0
    _check_backward(f)
    first = [t.clone() for t in f.outputs()]
    f.backward()
    assert all(_same_bits(a, b) for a, b in zip(first, f.outputs()))


@pytest.mark.parametrize("length", [1, 15, 16, 17, 47, 48, 63, 64, 65, 79, 80, 127, 128, 129, 191, 255, 256, 271, 513])
def test_ffn_backward_of_every_kind_of_segment_end(length):
    """The contraction of the weight gradients ends inside a 64-row step, inside an MMA, or on their borders."""
    X = np.array([[1], [1]], dtype=np.uint8)
    f = FfnGradient(length, [length, 37], X, 2, 256, 256)
    f.d.reserve_training()
    f.backward()
    assert f.d.last_status() == 0
    _check_backward(f)


@pytest.mark.parametrize("seed", range(8))
def test_ffn_backward_of_random_layouts(seed):
    rng = np.random.default_rng(seed)
    E, R = int(rng.choice([1, 3, 8, 17])), int(rng.choice([1, 2, 4]))
    C = min(16, -(-E // R) + int(rng.integers(0, 3)))
    if E > R * C:
        R = 2
        C = -(-E // R)
    X = np.zeros((E, R), dtype=np.uint8)
    for e in range(E):
        X[e, e % R] = 1
    for _ in range(6):
        e, j = int(rng.integers(E)), int(rng.integers(R))
        if not X[e, j] and X[:, j].sum() < C:
            X[e, j] = 1
    _, _, slot_expert = _tables(X, C)
    lengths = [int(rng.choice([0, 1, 5, 16, 64, 100, 300])) if e >= 0 else 0 for e in slot_expert]
    if not sum(lengths):
        lengths[int(np.argmax(slot_expert >= 0))] = 9
    f = FfnGradient(seed, lengths, X, C, int(rng.choice([256, 512, 1024])), int(rng.choice([128, 256, 640])), S=int(rng.choice([0, 1])))
    f.d.reserve_training()
    f.backward()
    assert f.d.last_status() == 0
    _check_backward(f)


def test_ffn_backward_with_the_largest_tables():
    """256 experts on 64 ranks, every one of the 1024 slots taken (four replicas an expert) and most segments empty or one row long;
    a shared expert beside them."""
    rng = np.random.default_rng(77)
    E, R, C = 256, 64, 16
    X = np.zeros((E, R), dtype=np.uint8)
    for e in range(E):
        X[e, (e // 16 + 16 * np.arange(4)) % R] = 1
    assert (X.sum(0) == C).all()
    lengths = [int(v) for v in rng.choice([0, 0, 0, 0, 0, 0, 1, 1, 2, 17], size=R * C)]
    f = FfnGradient(77, lengths, X, C, 256, 128, S=1)
    f.d.reserve_training()
    f.backward()
    assert f.d.last_status() == 0
    _check_backward(f)


def test_what_is_not_finite_stays_with_its_expert():
    """An expert's rows full of NaN and infinity, next to another's in the permuted order: a step of the other's contraction
    that reads past its segment must not pick them up."""
    X = np.array([[1], [1], [1]], dtype=np.uint8)
    f = FfnGradient(4, [37, 30, 41], X, 3, 256, 256)
    f.d.reserve_training()
    bad = slice(37, 67)
    f.xp[bad] = float("nan")
    f.dyp[bad] = float("inf")
    f.codes[bad] = 5
    f.exps[:, bad] = 255
    f.backward()
    assert f.d.last_status() == 0
    _check_backward(f, skip=(1,))
    import torch
    assert all(not torch.isfinite(w[1]).any() for w in f.dw) and not torch.isfinite(f.dxp[bad]).any()


def test_ffn_backward_is_the_derivative():
    """Against central differences of the fp64 forward: the slope of <dy, y> along each gradient is the gradient's own length, up
    to what the 8-bit values cost (steps of 2^-6 of a block's largest: 0.6 % of a value on average, 2 % is far outside)."""
    X = np.array([[1, 1], [0, 1]], dtype=np.uint8)
    f = FfnGradient(11, [120, 0, 95, 9], X, 2, 256, 128, scale=0.08)
    f.d.reserve_training()
    f.backward()
    rows = {0: np.r_[0:120, 120:215], 1: np.r_[215:224]}
    for e in (0, 1):
        args = dict(x=f.xp64[rows[e]], wg=f.wg64[e], wu=f.wu64[e], wd=f.wd64[e])
        got = dict(x=_np(f.dxp)[rows[e]], wg=_np(f.dw[0])[e], wu=_np(f.dw[1])[e], wd=_np(f.dw[2])[e])
        for name, grad in got.items():
            size = np.linalg.norm(grad)
            step = 1e-4 * grad / size
            value = [np.sum(f.dyp64[rows[e]] * gro.swiglu_ffn(**{**args, name: args[name] + k * step})[0]) for k in (1, -1)]
            assert abs((value[0] - value[1]) / 2e-4 - size) <= 0.02 * size, (e, name)


def test_without_x_the_shared_experts_are_left_out():
    lengths, X, C = _layout("ragged")
    f = FfnGradient(12, lengths, X, C, 256, 128, S=1)
    f.d.reserve_training()
    f.codes.fill_(99)
    f.d.expert_ffn_checkpoint(f.T, f.xp, f.seg, f.wg, f.wu, f.wd, f.codes, f.exps, f.yp)
    f.d.expert_ffn_backward(f.T, f.xp, f.dyp, f.seg, f.codes, f.exps, f.wg, f.wu, f.wd, f.dxp, *f.dw)
    assert f.d.last_status() == 0 and bool((f.dx_s == 7).all()) and all(bool((w == 7).all()) for w in f.dws)
    f.S = 0
    _check_backward(f)


def test_refusals_of_the_ffn_gradient():
    import torch
    from paper_2607_08782_b200.binding import DirectorError
    lengths, X, C = _layout("ragged")
    f = FfnGradient(3, lengths, X, C, 256, 128)
    with pytest.raises(DirectorError) as e:
        f.backward()
    assert e.value.status == 3                            # no workspace yet
    f.d.reserve_training()
    f.d.reserve_training()
    f.backward()
    good = [f.xp, f.dyp, f.seg, f.codes, f.exps, f.wg, f.wu, f.wd, f.dxp, *f.dw]
    for k, wrong in ((1, f.dyp.float()), (2, f.seg.long()), (3, f.codes.view(torch.uint8)), (11, f.dw[2].float())):
        with pytest.raises(TypeError):
            f.d.expert_ffn_backward(f.T, *good[:k], wrong, *good[k + 1:])
    for k, wrong in ((0, f.xp[:-1]), (9, f.dw[0][1:]), (5, f.wg.transpose(1, 2))):
        with pytest.raises(ValueError):
            f.d.expert_ffn_backward(f.T, *good[:k], wrong, *good[k + 1:])
    lib, ptr = f.d.lib, f.xp.data_ptr()
    call = lib.director_expert_ffn_backward
    assert call(None, f.T, *([ptr] * 12), *([None] * 12)) == 1
    assert call(f.d._ctx, 0, *([ptr] * 12), *([None] * 12)) == 1
    assert call(f.d._ctx, f.T + 1, *([ptr] * 12), *([None] * 12)) == 1
    assert call(f.d._ctx, f.T, *([ptr] * 11), None, *([None] * 12)) == 1
    assert call(f.d._ctx, f.T, *([ptr] * 11), ptr + 2, *([None] * 12)) == 1
    fresh = _context(8)
    assert call(fresh._ctx, 8, *([ptr] * 12), *([None] * 12)) == 2      # no placement
    assert f.d.last_status() == 0
