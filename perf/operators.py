"""The backward half of the expert-parallel MoE layer, operator by operator: cases, inputs, plain forms, 64-bit results.

Operators (T tokens of width H, K experts chosen per token out of E, expert width F, A = T*K assignments ("rows"),
inv_row[t,s] = row of token t's s-th choice in the order sorted by expert slot):

  combine_backward   y[t] = sum_s w[t,s] yp[inv_row[t,s]]      ->  dyp[inv_row[t,s]] = w[t,s] dy[t],  dw[t,s] = <dy[t], yp[inv_row[t,s]]>
  dispatch_backward  xp[inv_row[t,s]] = x[t] (+ shared experts) ->  dx[t] = sum_s dxp[inv_row[t,s]] (+ dx_shared[t])
  route_backward     w[t] = softmax of the chosen logits        ->  dlogits[t, idx[t,s]] = w[t,s] (dw[t,s] - sum_j w[t,j] dw[t,j]), 0 elsewhere
  ffn_checkpoint     g = xp Wg^T, u = xp Wu^T, yp = (silu(g) u) Wd^T, and g, u kept in 8 bits: 16 consecutive features of a row share a
                     power of two, value = code * 2^(e - 127), |code| <= 127
  ffn_backward       from dyp, xp and the 8-bit g, u:  da = dyp Wd,  du = da silu(g),  dg = da u silu'(g),  dxp = dg Wg + du Wu,
                     dWg[e] = dg^T xp,  dWu[e] = du^T xp,  dWd[e] = dyp^T (silu(g) u), sums over the rows of all of e's replicas

Shared experts (S > 0) are one more FFN of width S*F over all tokens."""
import math

import torch

own = False

BLOCK = 16          # features that share a scale in the 8-bit checkpoint
_handles = {}       # the framework's context of the shape in use, kept between calls as a training program keeps it


def listed():
    return [
        # a fine-tuning micro-batch of 64 tokens, 128 experts: latency counts
        dict(name="combine_grad_64", op="combine_backward", T=64, H=2048, F=128, E=128, K=8, S=0, R=16, C=9, hot=8, skew=1.4),
        # a DeepSeek-V2-Lite-shaped batch
        dict(name="combine_grad_8192", op="combine_backward", T=8192, H=2048, F=128, E=64, K=6, S=0, R=8, C=9, hot=8, skew=1.2),
        # the largest batch of the Qwen3-30B-A3B-shaped sweep
        dict(name="combine_grad_32768", op="combine_backward", T=32768, H=2048, F=128, E=128, K=8, S=0, R=16, C=9, hot=16, skew=1.4),
        # an odd little batch of wide rows
        dict(name="dispatch_grad_77", op="dispatch_backward", T=77, H=4096, F=128, E=8, K=2, S=0, R=8, C=2, hot=2, skew=1.0),
        # a Qwen1.5-MoE-shaped batch, the shared experts' gradient added on the way
        dict(name="dispatch_grad_16384", op="dispatch_backward", T=16384, H=2048, F=128, E=60, K=4, S=1, R=8, C=8, hot=4, skew=1.2),
        # the gate of an odd batch with 60 experts
        dict(name="route_grad_777", op="route_backward", T=777, H=256, F=128, E=60, K=4, S=0, R=8, C=8, hot=0, skew=1.2),
        # the gate of the largest batch
        dict(name="route_grad_32768", op="route_backward", T=32768, H=256, F=128, E=128, K=8, S=0, R=16, C=9, hot=0, skew=1.4),
        # 64 tokens over 128 experts: every expert's weights for a handful of rows
        dict(name="ffn_checkpoint_64", op="ffn_checkpoint", T=64, H=2048, F=768, E=128, K=8, S=0, R=16, C=9, hot=16, skew=1.4),
        # a DeepSeek-V2-Lite-shaped layer with its two shared experts
        dict(name="ffn_checkpoint_8192", op="ffn_checkpoint", T=8192, H=2048, F=1408, E=64, K=6, S=2, R=8, C=9, hot=8, skew=1.2),
        # the tiny layer
        dict(name="ffn_grad_64", op="ffn_backward", T=64, H=256, F=512, E=8, K=2, S=0, R=4, C=2, hot=0, skew=1.2),
        # Qwen3-30B-A3B-shaped, an odd batch: 64 rows an expert on average, some with none
        dict(name="ffn_grad_1021", op="ffn_backward", T=1021, H=2048, F=768, E=128, K=8, S=0, R=16, C=9, hot=16, skew=1.4),
        # Mixtral-8x7B-shaped, the two hottest experts replicated
        dict(name="ffn_grad_4096", op="ffn_backward", T=4096, H=4096, F=14336, E=8, K=2, S=0, R=8, C=2, hot=2, skew=1.0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: sizes over the whole range, no dearer than the largest listed case of its operator."""
    op = rng.choice(["combine_backward", "dispatch_backward", "route_backward", "ffn_checkpoint", "ffn_backward"])
    while True:
        E = rng.choice([2, 3, 8, 13, 32, 60, 64, 100, 128])
        K = rng.randint(1, min(8, E))
        T = _log_int(rng, 1, 32768)
        H = 256 * rng.choice([1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 11, 13, 14, 15, 16])
        F = 128
        S = rng.choice([0, 0, 0, 1, 2]) if op in ("ffn_checkpoint", "ffn_backward", "dispatch_backward") else 0
        R = rng.choice([1, 2, 4, 8, 16])
        C = -(-E // R) + rng.randint(0, 2)
        if C > 16 or T == 3072:
            continue
        case = dict(op=op, T=T, H=H, F=F, E=E, K=K, S=S, R=R, C=C, hot=rng.randint(0, R * C - E), skew=round(rng.uniform(0.0, 1.6), 2))
        if op in ("combine_backward", "dispatch_backward"):
            if T * K * H <= 32768 * 8 * 2048:
                return case
        elif op == "route_backward":
            return dict(case, H=256)
        else:
            case["F"] = F = 128 * _log_int(rng, 1, 112)
            if 3072 in (F, S * F):
                continue
            # no more work, no more weights and no more rows than the largest listed layer has
            if (T * (K + S) * H * F <= 4096 * 2 * 4096 * 14336 and (E + S) * H * F <= 8 * 4096 * 14336 and T * (K + S) * F <= 4 * 4096 * 2 * 14336
                    and T * K * H <= 32768 * 8 * 2048):
                return case


def work(case):
    T, H, F, E, K, S = (case[k] for k in ("T", "H", "F", "E", "K", "S"))
    A = T * K
    if case["op"] == "combine_backward":
        return {"bytes": 2 * T * H + 4 * A * H + 12 * A, "flops": 3 * A * H}
    if case["op"] == "dispatch_backward":
        return {"bytes": 2 * A * H + 2 * T * H * (2 if S else 1) + 4 * A, "flops": (A + (T if S else 0)) * H}
    if case["op"] == "route_backward":
        return {"bytes": 12 * A + 4 * T * E, "flops": 4 * A}
    rows_f = A * F + T * S * F                                   # (row, feature) pairs, routed and shared
    weights = 3 * (E + S) * F * H
    kept = rows_f * (2 + 2 / BLOCK)                              # bytes of the 8-bit g and u
    rows_h = A * H + (T * H if S else 0)
    if case["op"] == "ffn_checkpoint":                           # the 8-bit values written, and once more as bf16 numbers
        touched = 3 * (min(E, A) + S) * F * H                    # an expert without rows need not be read
        return {"bytes": 2 * rows_h * 2 + kept + 2 * touched + 4 * rows_f, "flops": 6 * rows_f * H}
    return {"bytes": 2 * rows_h * 3 + kept + 2 * 2 * weights, "flops": 12 * rows_f * H}


# ---- inputs ------------------------------------------------------------------------------------------------------


def _placement(case):
    """X[e][j] = 1 iff rank j hosts expert e: blocks of consecutive experts, then the `hot` first experts (the most
    frequently chosen ones) once more each, on the first rank with a free slot that does not host them yet."""
    E, R, C = case["E"], case["R"], case["C"]
    X = torch.zeros((E, R), dtype=torch.uint8)
    X[torch.arange(E), torch.arange(E) * R // E] = 1
    load = X.sum(0, dtype=torch.int64)
    e = 0
    for _ in range(case["hot"]):
        for _ in range(E):
            free = [j for j in range(R) if load[j] < C and not X[e, j]]
            if free:
                X[e, free[-1]] = 1
                load[free[-1]] += 1
                e = (e + 1) % E
                break
            e = (e + 1) % E
    return X


def _tables(X, C):
    """Slot of every replica, replicas by (expert, rank); the first replica of each expert, and its number of replicas."""
    pos = torch.cumsum(X.long(), 0) - 1
    e, j = torch.nonzero(X, as_tuple=True)
    count = X.sum(1, dtype=torch.int64)
    return e, j * C + pos[e, j], torch.cumsum(count, 0) - count, count


def _bf16(g, *shape, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale).bfloat16()


def _checkpoint(values):
    """(codes, exps) of fp32 values [rows, features]: 16 consecutive features share a power of two, chosen so that the largest
    magnitude gets a code of 64 to 127."""
    rows, F = values.shape
    v = values.view(rows, F // BLOCK, BLOCK)
    e = (torch.frexp(v.abs().amax(-1))[1] + 120).clamp(min=1)      # biased exponent of the largest magnitude, minus 6
    codes = torch.round(v * _power(254 - e).unsqueeze(-1)).clamp(-127, 127)
    return codes.view(rows, F).to(torch.int8), e.to(torch.uint8)


def _power(biased):
    """2^(biased - 127) in fp32."""
    return (biased.int() << 23).view(torch.float32)


def _kept(g, rows, F, H):
    """The 8-bit checkpoint of a layer's gate and up values as a forward pass leaves it: codes [rows, F, 2], exps [F/16, rows, 2]."""
    codes = torch.empty((rows, F, 2), dtype=torch.int8, device="cuda")
    exps = torch.empty((F // BLOCK, rows, 2), dtype=torch.uint8, device="cuda")
    for which in (0, 1):
        for lo in range(0, rows, 4096):
            v = torch.randn((min(rows, lo + 4096) - lo, F), generator=g, device="cuda") * (0.01 * math.sqrt(H))
            c, e = _checkpoint(v)
            codes[lo:lo + 4096, :, which] = c
            exps[:, lo:lo + 4096, which] = e.t()
    return codes, exps


def prepare(case, seed):
    T, H, F, E, K, S, R, C = (case[k] for k in ("T", "H", "F", "E", "K", "S", "R", "C"))
    A, op = T * K, case["op"]
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1000003 + 17)
    # the gate: logits ~ N(0,1) plus a rank-frequency bias, the K largest
    bias = -case["skew"] * torch.log(1.0 + torch.arange(E, device="cuda", dtype=torch.float32))
    top = torch.topk(torch.randn((T, E), generator=g, device="cuda") + bias, K, dim=1)
    st = dict(case=case, topk_idx=top.indices.int().contiguous(), topk_w=torch.softmax(top.values, 1).contiguous())
    # the permutation: the n-th assignment of an expert (tokens ascending) goes to its replica n mod r, segments in slot order
    X = _placement(case)
    rep_expert, rep_slot, first, count = (t.cuda() for t in _tables(X, C))
    experts = st["topk_idx"].long().flatten()
    order = torch.argsort(experts, stable=True)
    starts = torch.cumsum(torch.bincount(experts, minlength=E), 0) - torch.bincount(experts, minlength=E)
    nth = torch.empty_like(experts)
    nth[order] = torch.arange(A, device="cuda") - starts[experts[order]]
    slot = rep_slot[first[experts] + nth % count[experts]]
    by_slot = torch.argsort(slot, stable=True)
    inv_row = torch.empty(A, dtype=torch.int32, device="cuda")
    inv_row[by_slot] = torch.arange(A, dtype=torch.int32, device="cuda")
    st["inv_row"] = inv_row.view(T, K)
    sizes = torch.bincount(slot, minlength=R * C)
    st["seg_offsets"] = torch.cat([sizes.new_zeros(1), torch.cumsum(sizes, 0)]).int()
    if op == "combine_backward":
        st.update(dy=_bf16(g, T, H, scale=1e-3), yp=_bf16(g, A, H, scale=0.5))
        st.update(dyp=torch.empty_like(st["yp"]), dtopk_w=torch.empty((T, K), device="cuda"))
    elif op == "dispatch_backward":
        st.update(dxp=_bf16(g, A, H, scale=1e-3), dx_shared=_bf16(g, T, H, scale=1e-3) if S else None)
        st.update(dx=torch.empty((T, H), dtype=torch.bfloat16, device="cuda"))
    elif op == "route_backward":
        st.update(dtopk_w=torch.randn((T, K), generator=g, device="cuda") * 0.1, dlogits=torch.empty((T, E), device="cuda"))
    else:
        # the rows of each expert, over all of its replicas' segments (the plain form and the 64-bit one walk the experts)
        row_expert = experts[by_slot]
        by_expert = torch.argsort(row_expert, stable=True)
        st["rows"] = torch.split(by_expert, torch.bincount(row_expert, minlength=E).tolist())
        x = _bf16(g, T, H, scale=0.5)
        st["xp"] = x[by_slot // K].contiguous()
        st["w"] = (_bf16(g, E, F, H, scale=0.02), _bf16(g, E, F, H, scale=0.02), _bf16(g, E, H, F, scale=0.02))
        if S:
            st["x"], st["ws"] = x, (_bf16(g, S * F, H, scale=0.02), _bf16(g, S * F, H, scale=0.02), _bf16(g, H, S * F, scale=0.02))
        if op == "ffn_checkpoint":
            _outputs_checkpoint(st, A, T, H, F, S)
        else:
            st["kept"] = _kept(g, A, F, H)
            st["dyp"] = _bf16(g, A, H, scale=1e-3)
            if S:
                st["kept_shared"], st["dy"] = _kept(g, T, S * F, H), _bf16(g, T, H, scale=1e-3)
            st["dxp"] = torch.empty_like(st["xp"])
            st["dw"] = tuple(torch.empty_like(w) for w in st["w"])
            if S:
                st["dx_shared"], st["dws"] = torch.empty_like(x), tuple(torch.empty_like(w) for w in st["ws"])
    if own:
        st["d"] = _handle(case, X)
    return st


def _outputs_checkpoint(st, A, T, H, F, S):
    def room(rows, width):
        return (torch.empty((rows, width, 2), dtype=torch.int8, device="cuda"),
                torch.empty((width // BLOCK, rows, 2), dtype=torch.uint8, device="cuda"))

    def rows_of(rows, width):
        return torch.empty((rows, width), dtype=torch.bfloat16, device="cuda")
    st["yp"], st["kept"], st["gu"] = rows_of(A, H), room(A, F), (rows_of(A, F), rows_of(A, F))
    if S:
        st["y_shared"], st["kept_shared"], st["gu_shared"] = rows_of(T, H), room(T, S * F), (rows_of(T, S * F), rows_of(T, S * F))


def _handle(case, X):
    from paper_2607_08782_b200.binding import Director
    key = tuple(case[k] for k in ("T", "H", "F", "E", "K", "S", "R", "C", "hot", "op"))
    if key not in _handles:
        _handles.clear()
        d = Director(*key[:8])
        d.set_placement(X.numpy())
        if case["op"] == "ffn_backward":
            d.reserve_training()
        _handles[key] = d
    return _handles[key]


# ---- one pass ----------------------------------------------------------------------------------------------------


def run(st):
    return (_run_own if own else _run_plain)(st)


def _run_own(st):
    c, d = st["case"], st["d"]
    T, op, S = c["T"], c["op"], c["S"]
    if op == "combine_backward":
        d.combine_backward(T, st["dy"], st["yp"], st["inv_row"], st["topk_w"], st["dyp"], st["dtopk_w"])
        return {"dyp": st["dyp"], "dtopk_w": st["dtopk_w"]}
    if op == "dispatch_backward":
        d.dispatch_backward(T, st["dxp"], st["inv_row"], st["dx_shared"], st["dx"])
        return st["dx"]
    if op == "route_backward":
        d.route_backward(T, st["topk_idx"], st["topk_w"], st["dtopk_w"], st["dlogits"])
        return st["dlogits"]
    if op == "ffn_checkpoint":
        shared = (st["x"], *st["ws"], *st["kept_shared"], st["y_shared"]) if S else ()
        d.expert_ffn_checkpoint(T, st["xp"], st["seg_offsets"], *st["w"], *st["kept"], st["yp"], *shared)
        d.checkpoint_decode(T * c["K"], c["F"], *st["kept"], *st["gu"])        # the 8-bit values as the numbers they stand for
        out = {"yp": st["yp"], "g": st["gu"][0], "u": st["gu"][1]}
        if S:
            d.checkpoint_decode(T, S * c["F"], *st["kept_shared"], *st["gu_shared"])
            out.update(y_shared=st["y_shared"], g_shared=st["gu_shared"][0], u_shared=st["gu_shared"][1])
        return out
    shared = (st["x"], st["dy"], *st["kept_shared"], *st["ws"], st["dx_shared"], *st["dws"]) if S else ()
    d.expert_ffn_backward(T, st["xp"], st["dyp"], st["seg_offsets"], *st["kept"], *st["w"], st["dxp"], *st["dw"], *shared)
    out = {"dxp": st["dxp"], "dw_gate": st["dw"][0], "dw_up": st["dw"][1], "dw_down": st["dw"][2]}
    if S:
        out.update(dx_shared=st["dx_shared"], dws_gate=st["dws"][0], dws_up=st["dws"][1], dws_down=st["dws"][2])
    return out



def _decode(kept, which):
    """The values that the codes stand for, bf16 (a code of 7 bits and a sign times a power of two is exact in it)."""
    codes, exps = kept
    rows, F = codes.shape[:2]
    scale = _power(exps[:, :, which]).t()                                                # [rows, F/16]
    v = codes[:, :, which].reshape(rows, F // BLOCK, BLOCK).bfloat16()
    return (v * scale.unsqueeze(-1).bfloat16()).view(rows, F)


def _run_plain(st):
    c = st["case"]
    T, H, F, E, K, S, op = (c[k] for k in ("T", "H", "F", "E", "K", "S", "op"))
    if op == "combine_backward":
        dy, inv = st["dy"].float(), st["inv_row"].long()
        dtopk_w = (dy.unsqueeze(1) * st["yp"][inv].float()).sum(-1)
        dyp = torch.empty_like(st["yp"])
        dyp[inv] = (st["topk_w"].unsqueeze(-1) * dy.unsqueeze(1)).bfloat16()
        return {"dyp": dyp, "dtopk_w": dtopk_w}
    if op == "dispatch_backward":
        dx = st["dxp"][st["inv_row"].long()].float().sum(1)
        return (dx + st["dx_shared"].float() if S else dx).bfloat16()
    if op == "route_backward":
        w, dw = st["topk_w"], st["dtopk_w"]
        dl = w * (dw - (w * dw).sum(1, keepdim=True))
        return torch.zeros((T, E), device=w.device).scatter_(1, st["topk_idx"].long(), dl)
    # the expert products: segments have lengths of their own, so the experts are walked one after the other - padding them to one
    # batched product would do several times the work of a skewed batch
    if op == "ffn_checkpoint":
        yp = torch.empty((T * K, H), dtype=torch.bfloat16, device="cuda")
        gu = [torch.empty((T * K, F), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        for e, rows in enumerate(st["rows"]):
            if len(rows):
                yp[rows], gu[0][rows], gu[1][rows] = _ffn_plain(st["xp"][rows], *(w[e] for w in st["w"]))
        out = {"yp": yp, "g": gu[0], "u": gu[1]}
        if S:
            out["y_shared"], out["g_shared"], out["u_shared"] = _ffn_plain(st["x"], *st["ws"])
        return out
    dxp = torch.empty((T * K, H), dtype=torch.bfloat16, device="cuda")
    dw = [torch.zeros_like(w) for w in st["w"]]
    for e, rows in enumerate(st["rows"]):
        if len(rows):
            kept = (st["kept"][0][rows], st["kept"][1][:, rows])
            dxp[rows], dw[0][e], dw[1][e], dw[2][e] = _ffn_grad_plain(st["xp"][rows], st["dyp"][rows], kept, *(w[e] for w in st["w"]))
    out = {"dxp": dxp, "dw_gate": dw[0], "dw_up": dw[1], "dw_down": dw[2]}
    if S:
        out["dx_shared"], out["dws_gate"], out["dws_up"], out["dws_down"] = _ffn_grad_plain(st["x"], st["dy"], st["kept_shared"], *st["ws"])
    return out


def _round8(v):
    """fp32 values as the 8-bit checkpoint holds them."""
    rows, F = v.shape
    b = v.view(rows, F // BLOCK, BLOCK)
    e = (torch.frexp(b.abs().amax(-1, keepdim=True))[1] + 120).clamp(min=1)
    codes = torch.round(b * _power(254 - e)).clamp(-127, 127)
    return (codes * _power(e)).view(rows, F).bfloat16()


def _ffn_plain(x, wg, wu, wd):
    x = x.float()
    g, u = x @ wg.float().t(), x @ wu.float().t()
    y = (g / (1 + torch.exp(-g)) * u) @ wd.float().t()
    return y.bfloat16(), _round8(g), _round8(u)


def _ffn_grad_plain(x, dy, kept, wg, wu, wd):
    x, dy = x.float(), dy.float()
    g, u = _decode(kept, 0).float(), _decode(kept, 1).float()
    s = 1 / (1 + torch.exp(-g))
    da = dy @ wd.float()
    du, dg = da * (g * s), da * u * (s * (1 + g * (1 - s)))
    return ((dg @ wg.float() + du @ wu.float()).bfloat16(), (dg.t() @ x).bfloat16(), (du.t() @ x).bfloat16(),
            (dy.t() @ (g * s * u)).bfloat16())


# ---- 64 bits -----------------------------------------------------------------------------------------------------


def exact(case, seed):
    """The definitions in 64 bits.  What is rounded at the end of an operator - to bf16, or to the 8 bits of the checkpoint - is
    given here unrounded."""
    st = prepare(case, seed)
    T, H, F, E, K, S, op = (case[k] for k in ("T", "H", "F", "E", "K", "S", "op"))
    f64 = torch.float64
    inv = st["inv_row"].long()
    if op == "combine_backward":
        dyp = torch.zeros((T * K, H), dtype=f64, device="cuda")
        dw = torch.zeros((T, K), dtype=f64, device="cuda")
        for s in range(K):
            dyp.index_copy_(0, inv[:, s], st["dy"].to(f64) * st["topk_w"][:, s:s + 1].to(f64))
            dw[:, s] = torch.einsum("th,th->t", st["dy"].to(f64), st["yp"][inv[:, s]].to(f64))
        return {"dyp": dyp, "dtopk_w": dw}
    if op == "dispatch_backward":
        dx = st["dx_shared"].to(f64) if S else torch.zeros((T, H), dtype=f64, device="cuda")
        for s in range(K):
            dx = dx + st["dxp"][inv[:, s]].to(f64)
        return dx
    if op == "route_backward":
        w, dw = st["topk_w"].to(f64), st["dtopk_w"].to(f64)
        jac = torch.diag_embed(w) - w.unsqueeze(2) * w.unsqueeze(1)              # d w / d chosen logits
        dl = torch.einsum("tsj,tj->ts", jac, dw)
        out = torch.zeros((T, E), dtype=f64, device="cuda")
        for s in range(K):
            out[torch.arange(T, device="cuda"), st["topk_idx"][:, s].long()] += dl[:, s]
        return out
    if op == "ffn_checkpoint":
        out = {"yp": torch.zeros((T * K, H), dtype=f64, device="cuda"), "g": torch.zeros((T * K, F), dtype=f64, device="cuda"),
               "u": torch.zeros((T * K, F), dtype=f64, device="cuda")}
        for e, rows in enumerate(st["rows"]):
            out["g"][rows] = st["xp"][rows].to(f64) @ st["w"][0][e].to(f64).t()
            out["u"][rows] = st["xp"][rows].to(f64) @ st["w"][1][e].to(f64).t()
            out["yp"][rows] = (out["g"][rows] * torch.sigmoid(out["g"][rows]) * out["u"][rows]) @ st["w"][2][e].to(f64).t()
        if S:
            gs, us = (st["x"].to(f64) @ w.to(f64).t() for w in st["ws"][:2])
            out.update(y_shared=(gs * torch.sigmoid(gs) * us) @ st["ws"][2].to(f64).t(), g_shared=gs, u_shared=us)
        return out
    out = {"dxp": torch.zeros((T * K, H), dtype=f64, device="cuda")}
    for name, w in zip(("dw_gate", "dw_up", "dw_down"), st["w"]):
        out[name] = torch.zeros(w.shape, dtype=f64, device="cuda")
    for e, rows in enumerate(st["rows"]):
        kept = (st["kept"][0][rows], st["kept"][1][:, rows])
        out["dxp"][rows], out["dw_gate"][e], out["dw_up"][e], out["dw_down"][e] = _ffn_grad_64(
            st["xp"][rows], st["dyp"][rows], kept, *(w[e] for w in st["w"]))
    if S:
        out["dx_shared"], out["dws_gate"], out["dws_up"], out["dws_down"] = _ffn_grad_64(st["x"], st["dy"], st["kept_shared"], *st["ws"])
    return out


def _ffn_grad_64(x, dy, kept, wg, wu, wd):
    x, dy, wg, wu, wd = (t.double() for t in (x, dy, wg, wu, wd))
    codes, exps = kept
    scale = torch.exp2(exps.double() - 127).repeat_interleave(BLOCK, dim=0).permute(1, 0, 2)    # [rows, F, 2]
    g, u = (codes.double() * scale).unbind(-1)
    sig = torch.sigmoid(g)
    da = dy @ wd
    dg, du = da * u * (sig + g * sig * (1 - sig)), da * g * sig
    return dg @ wg + du @ wu, dg.t() @ x, du.t() @ x, dy.t() @ (g * sig * u)
