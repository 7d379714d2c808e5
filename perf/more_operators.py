"""What turns the layer's gradients into a training step, operator by operator: cases, inputs, plain forms, 64-bit results.

  balance    the router's balance term.  N valid tokens, counts[e] = their assignments to expert e, f = counts / (K N),
             p[t] = softmax(logits[t]), P = sum over the valid tokens of p[t] / N:   loss = E sum_e f[e] P[e],
             dlogits[t,e] = added[t,e] + dloss E/N p[t,e] (f[e] - sum_j f[j] p[t,j])   (0 for a token that is not valid)
  grad_norm  norm = sqrt of the sum of squares over all elements of many tensors
  clip       out = g min(1, max_norm / norm) for all of them, as fp32 gradients for an optimizer that takes those
  update     AdamW on the clipped gradients g' = g min(1, max_norm / norm), t the number of the step:
             m = b1 m + (1 - b1) g',  v = b2 v + (1 - b2) g'^2,  w = w - lr wd w - lr (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps),
             bf16 weights with fp32 masters, fp32 weights (the router's) without

The tensors of the last three are those of MoE layers: per layer w_gate, w_up, w_down of E experts, the same of S shared experts side
by side, and the router [E,H], which is fp32.  bucket: the gradients lie back to back in one buffer per type, as data-parallel training
reduces them, so that odd sizes put the tensors behind them at odd addresses."""
import math

import torch

own = False

LR, BETA1, BETA2, EPS, DECAY = 1e-4, 0.9, 0.95, 1e-8, 0.1
_handles = {}       # the framework's context of the shape in use, kept between calls as a training program keeps it


def listed():
    return [
        # the router of the fine-tuning example's layer, a micro-batch of 48 tokens: latency counts
        dict(name="balance_48", op="balance", T=48, E=8, K=2, mask=False, backward=True, added=True),
        # validation over a padded batch of a Qwen1.5-MoE-shaped router: loss and counts alone
        dict(name="balance_eval_4093", op="balance", T=4093, E=60, K=4, mask=True, backward=False, added=False),
        # a DeepSeek-V2-Lite-shaped training batch, added to the gate's own gradient
        dict(name="balance_8192", op="balance", T=8192, E=64, K=6, mask=False, backward=True, added=True),
        # the longest batch with the most experts, padded
        dict(name="balance_131072", op="balance", T=131072, E=256, K=8, mask=True, backward=True, added=False),
        # the fine-tuning example's own layer: eight experts of 256 x 256
        dict(name="norm_tiny", op="grad_norm", layers=1, E=8, H=256, F=256, S=0, grads="bf16", bucket=False),
        # 48 layers of a small model with odd widths, 336 tensors back to back in two buckets
        dict(name="norm_many", op="grad_norm", layers=48, E=8, H=251, F=357, S=1, grads="bf16", bucket=True),
        # a Mixtral-8x7B-shaped layer's gradients
        dict(name="norm_large", op="grad_norm", layers=1, E=8, H=4096, F=14336, S=0, grads="bf16", bucket=False),
        # the fine-tuning example's own layer with a shared expert
        dict(name="clip_tiny", op="clip", layers=1, E=8, H=256, F=256, S=1, grads="bf16", bucket=False),
        # a DeepSeek-V2-Lite-shaped layer
        dict(name="clip_large", op="clip", layers=1, E=64, H=2048, F=1408, S=2, grads="bf16", bucket=False),
        # the fine-tuning example's own layer
        dict(name="update_tiny", op="update", layers=1, E=8, H=256, F=256, S=0, grads="bf16", bucket=False, clip=True),
        # two layers of odd widths, fp32 gradients back to back in a bucket, no clipping
        dict(name="update_odd", op="update", layers=2, E=13, H=509, F=381, S=1, grads="fp32", bucket=True, clip=False),
        # a Qwen3-30B-A3B-shaped layer
        dict(name="update_large", op="update", layers=1, E=128, H=2048, F=768, S=0, grads="bf16", bucket=False, clip=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_MOST = {"grad_norm": 1_400_000_000, "clip": 560_000_000, "update": 600_000_000}      # elements of the largest listed cases


def draw(rng):
    """One more case: sizes over the whole range, no dearer than the largest listed case of its operator."""
    op = rng.choice(["balance", "balance", "grad_norm", "clip", "update", "update"])
    if op == "balance":
        E = rng.choice([1, 2, 3, 8, 13, 32, 60, 64, 100, 128, 160, 251, 256])
        backward = rng.random() < 0.75
        return dict(op=op, T=_log_int(rng, 1, 131072), E=E, K=rng.randint(1, max(1, min(8, E - 1))), mask=rng.random() < 0.5, backward=backward,
                    added=backward and rng.random() < 0.5)
    while True:
        S = rng.choice([0, 0, 1, 2])
        layers = _log_int(rng, 1, {"grad_norm": 48, "clip": 8, "update": 2}[op])
        case = dict(op=op, layers=layers, E=rng.choice([2, 3, 8, 13, 60, 64, 128]), H=_log_int(rng, 16, 4096), F=_log_int(rng, 16, 8192), S=S,
                    grads=rng.choice(["bf16", "bf16", "fp32"]), bucket=rng.random() < 0.5)
        if op == "update":
            case["clip"] = rng.random() < 0.7
        if sum(n for n, _ in _sizes(case)) <= _MOST[op]:
            return case


def _sizes(case):
    """(elements, whether a router's) of every tensor."""
    E, H, F, S = (case[k] for k in ("E", "H", "F", "S"))
    layer = [(E * F * H, False)] * 3 + [(S * F * H, False)] * (3 if S else 0) + [(E * H, True)]
    return layer * case["layers"]


# ---- inputs --------------------------------------------------------------------------------------------------------


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (_prepare_balance if case["op"] == "balance" else _prepare_tensors)(case, g)


def _prepare_balance(case, g):
    """Logits with a bias per expert, so that some are hot; the gate's choice among them; padding at the sequences' ends."""
    T, E, K = case["T"], case["E"], case["K"]
    logits = torch.randn((T, E), generator=g, device="cuda") + torch.randn((E,), generator=g, device="cuda")
    st = dict(case=case, logits=logits, topk_idx=logits.topk(K, dim=1).indices.int(), mask=None, added=None)
    if case["mask"]:
        length = max(1, min(T, 509))                                             # sequences of 509 places, filled to between half and all
        fill = (length * (0.5 + 0.5 * torch.rand((-(-T // length),), generator=g, device="cuda"))).ceil().long()
        t = torch.arange(T, device="cuda")
        st["mask"] = (t % length < fill[t // length]).to(torch.uint8)
    st["loss"] = torch.empty((1,), device="cuda")
    st["counts"] = torch.empty((E + 1,), dtype=torch.int64, device="cuda")
    if case["backward"]:
        st["dloss"] = torch.rand((1,), generator=g, device="cuda") * 0.02 + 0.001     # the weight of the balance term in the loss
        st["dlogits"] = torch.empty_like(logits)
        if case["added"]:
            st["added"] = torch.randn((T, E), generator=g, device="cuda") * (1e-3 / T)
    if own:
        st["d"] = _handle(case)
    return st


def _handle(case):
    from paper_2607_08782_b200.binding import Director
    key = tuple(case[k] for k in ("T", "E", "K"))
    if key not in _handles:
        _handles.clear()
        T, E, K = key
        _handles[key] = Director(T, 256, 128, E, K, 0, 16, 16)
    return _handles[key]


def _prepare_tensors(case, g):
    op, sizes = case["op"], _sizes(case)
    grad_types = [torch.float32 if router or case["grads"] == "fp32" else torch.bfloat16 for _, router in sizes]
    scale = torch.rand((len(sizes),), generator=g, device="cuda") * 1e-3 + 1e-5

    def normal(n, dtype, factor):
        return torch.randn((n,), generator=g, device="cuda", dtype=dtype).mul_(factor)
    grads = [normal(n, t, s) for (n, _), t, s in zip(sizes, grad_types, scale)]
    if case["bucket"]:
        grads = _in_buckets(grads)
    st = dict(case=case, grads=grads)
    norm = math.sqrt(sum(float(x.float().square().sum(dtype=torch.float64)) for x in grads))
    st["max_norm"] = 0.37 * norm if case.get("clip", True) else math.inf            # a step that has to be clipped
    if op == "clip":
        st["out"] = [torch.empty_like(x, dtype=torch.float32) for x in grads]
    if op == "update":
        # the 1000 steps before this one have left their moments
        st["masters"] = [normal(n, torch.float32, 0.02) for n, _ in sizes]
        st["weights"] = [m if router else m.bfloat16() for m, (_, router) in zip(st["masters"], sizes)]
        st["m"] = [normal(n, torch.float32, s * 0.3) for (n, _), s in zip(sizes, scale)]
        st["v"] = [normal(n, torch.float32, s).square_().add_((s * 0.1) ** 2) for (n, _), s in zip(sizes, scale)]
        st["steps"] = torch.full((1,), 1000, dtype=torch.int64, device="cuda")
    if own:
        _own_tensors(st)
    return st


def _in_buckets(grads):
    flat = {t: torch.cat([x for x in grads if x.dtype is t]) for t in {x.dtype for x in grads}}
    at, views = dict.fromkeys(flat, 0), []
    for x in grads:
        views.append(flat[x.dtype][at[x.dtype]:at[x.dtype] + x.numel()])
        at[x.dtype] += x.numel()
    return views


def _own_tensors(st):
    from paper_2607_08782_b200.training import AdamW, TensorList
    st["grad_list"] = TensorList(st["grads"])
    if "out" in st:
        st["out_list"] = TensorList(st["out"])
    if "weights" in st:
        st["optimizer"] = AdamW(st["weights"], lr=LR, betas=(BETA1, BETA2), eps=EPS, weight_decay=DECAY, max_norm=st["max_norm"])
        st["optimizer"].load_state_dict({k: st.pop(n) for k, n in dict(steps="steps", masters="masters", exp_avg="m", exp_avg_sq="v").items()})


# ---- one pass ------------------------------------------------------------------------------------------------------


def run(st):
    return (_run_own if own else _run_plain)(st)


def _run_own(st):
    op = st["case"]["op"]
    if op == "balance":
        c, d = st["case"], st["d"]
        d.balance_loss(c["T"], st["logits"], st["topk_idx"], st["mask"], st["loss"], st["counts"])
        out = {"loss": st["loss"], "counts": st["counts"]}
        if c["backward"]:
            d.balance_loss_backward(c["T"], st["logits"], st["counts"], st["mask"], st["dloss"], st["added"], st["dlogits"])
            out["dlogits"] = st["dlogits"]
        return out
    from paper_2607_08782_b200 import training
    if op == "grad_norm":
        return training.grad_norm(st["grad_list"])
    if op == "clip":
        norm = training.clip_grads(st["grad_list"], st["max_norm"], out=st["out_list"])
        return {"norm": norm, "grads": st["out"]}
    opt = st["optimizer"]
    norm = opt.step(st["grad_list"])
    out = {"weights": opt.weights, "masters": [m for m in opt.masters if m is not None], "m": opt.exp_avg, "v": opt.exp_avg_sq, "steps": opt.steps}
    return dict(out, norm=norm) if norm is not None else out


def _run_plain(st):
    return {"balance": _plain_balance, "grad_norm": _plain_norm, "clip": _plain_clip, "update": _plain_update}[st["case"]["op"]](st)


def _plain_balance(st):
    c = st["case"]
    T, E, K = c["T"], c["E"], c["K"]
    valid = torch.ones((T, 1), dtype=torch.bool, device="cuda") if st["mask"] is None else st["mask"].bool().unsqueeze(1)
    z = (st["logits"] - st["logits"].amax(dim=1, keepdim=True)).exp()
    p = torch.where(valid, z / z.sum(dim=1, keepdim=True), 0.0)
    counts = torch.zeros((E,), dtype=torch.int64, device="cuda")
    counts.index_add_(0, st["topk_idx"].long().view(-1), valid.long().expand(T, K).reshape(-1))
    N = valid.sum()
    f = counts.double() / (K * N)
    loss = (E * (f * p.sum(dim=0, dtype=torch.float64) / N).sum()).float().view(1)
    out = {"loss": loss, "counts": torch.cat([counts, N.view(1)])}
    if c["backward"]:
        f = ((E * counts - counts.sum()).double() / (E * K * N)).float()     # less its mean, which the difference below cancels
        d = st["dloss"] * (E / N) * p * (f - (p * f).sum(dim=1, keepdim=True))
        out["dlogits"] = d if st["added"] is None else d + st["added"]
    return out


def _norm_of(grads):
    return torch.stack([x.float().square().sum(dtype=torch.float64) for x in grads]).sum().sqrt()


def _factor(norm, max_norm):
    return (max_norm / norm).clamp(max=1.0).float()


def _plain_norm(st):
    return _norm_of(st["grads"]).float()


def _plain_clip(st):
    norm = _norm_of(st["grads"])
    c = _factor(norm, st["max_norm"])
    return {"norm": norm.float(), "grads": [o.copy_(x.float() * c) for o, x in zip(st["out"], st["grads"])]}


def _plain_update(st):
    out = {}
    c = 1.0
    if math.isfinite(st["max_norm"]):
        norm = _norm_of(st["grads"])
        out["norm"], c = norm.float(), _factor(norm, st["max_norm"])
    st["steps"] += 1
    t = st["steps"].double()
    rate1, rate2 = (LR / (1 - BETA1 ** t)).float(), (1 / (1 - BETA2 ** t).sqrt()).float()
    for w, master, x, m, v in zip(st["weights"], st["masters"], st["grads"], st["m"], st["v"]):
        x = x.float() * c
        m.mul_(BETA1).add_(x * (1 - BETA1))
        v.mul_(BETA2).add_(x * x * (1 - BETA2))
        master.mul_(1 - LR * DECAY).sub_(rate1 * m / (v.sqrt() * rate2 + EPS))
        w.copy_(master)
    return dict(out, weights=st["weights"], masters=[m for m, w in zip(st["masters"], st["weights"]) if w.dtype is torch.bfloat16], m=st["m"],
                v=st["v"], steps=st["steps"])


# ---- 64 bits -------------------------------------------------------------------------------------------------------


def exact(case, seed):
    """The definitions in 64 bits on the inputs of prepare."""
    global own
    before, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = before
    if case["op"] == "balance":
        return _exact_balance(st)
    square = sum(float(torch.dot(x.double(), x.double())) for x in st["grads"])
    norm = torch.tensor(math.sqrt(square), dtype=torch.float64)
    if case["op"] == "grad_norm":
        return norm
    c = min(1.0, st["max_norm"] / math.sqrt(square))
    if case["op"] == "clip":
        return {"norm": norm, "grads": [x.double() * c for x in st["grads"]]}
    t = int(st["steps"]) + 1
    weights, masters, ms, vs = [], [], [], []
    for w, master, x, m, v in zip(st["weights"], st["masters"], st["grads"], st["m"], st["v"]):
        g = c * x.double()
        m = BETA1 * m.double() + (1 - BETA1) * g
        v = BETA2 * v.double() + (1 - BETA2) * g ** 2
        new = master.double()
        new = new - LR * DECAY * new - LR * (m / (1 - BETA1 ** t)) / (torch.sqrt(v / (1 - BETA2 ** t)) + EPS)
        weights.append(new)
        if w.dtype is torch.bfloat16:
            masters.append(new)
        ms.append(m)
        vs.append(v)
    out = {"weights": weights, "masters": masters, "m": ms, "v": vs, "steps": torch.tensor([t], dtype=torch.int64)}
    return dict(out, norm=norm) if case["clip"] else out


def _exact_balance(st):
    c = st["case"]
    T, E, K = c["T"], c["E"], c["K"]
    rows = torch.arange(T, device="cuda") if st["mask"] is None else st["mask"].nonzero().view(-1)
    N = rows.numel()
    x = st["logits"].double()[rows]
    p = (x - torch.logsumexp(x, dim=1, keepdim=True)).exp()
    counts = torch.bincount(st["topk_idx"].long()[rows].flatten(), minlength=E)
    f = counts.double() / (N * K)
    out = {"loss": (E * torch.dot(f, p.mean(dim=0))).view(1), "counts": torch.cat([counts, torch.tensor([N], device="cuda")])}
    if c["backward"]:
        d = torch.zeros((T, E), dtype=torch.float64, device="cuda")
        d[rows] = float(st["dloss"]) * E / N * p * (f - (p @ f).unsqueeze(1))
        out["dlogits"] = d if st["added"] is None else d + st["added"].double()
    return out


# ---- what a pass cannot do without -----------------------------------------------------------------------------------


def work(case):
    if case["op"] == "balance":
        T, E, K = case["T"], case["E"], case["K"]
        arrays = 1 + (1 + bool(case["added"]) if case["backward"] else 0)
        return {"bytes": 4 * T * E * arrays + 4 * T * K + (T if case["mask"] else 0), "flops": (16 if case["backward"] else 6) * T * E}
    total = flops = 0
    for n, router in _sizes(case):
        g = 4 if router or case["grads"] == "fp32" else 2
        total += n * (g + {"grad_norm": 0, "clip": 4, "update": 16 + (8 if router else 10)}[case["op"]])
        flops += n * {"grad_norm": 2, "clip": 3, "update": 16}[case["op"]]
    return {"bytes": total, "flops": flops}
