"""Plain fp64 definitions of the layer's backward pass (the forward's are in director_oracle.py).

Written from the formulas, one expert and one choice at a time; shares no code with the CUDA path.  All arguments are
fp64 arrays of the values in question (bf16 inputs are converted by the caller), all results fp64, unrounded."""
from __future__ import annotations

import numpy as np

BLOCK = 16      # features of a row that share a scale in the 8-bit checkpoint


def combine_backward(dy, yp, inv_row, topk_w):
    """y[t] = sum_s w[t,s] yp[inv_row[t,s]]  ->  (dyp, dw).  Assignments with inv_row < 0 take no part."""
    dyp = np.zeros_like(yp)
    dw = np.zeros(inv_row.shape, dtype=np.float64)
    for t in range(inv_row.shape[0]):
        for s in range(inv_row.shape[1]):
            r = int(inv_row[t, s])
            if r >= 0:
                dyp[r] = float(topk_w[t, s]) * dy[t]
                dw[t, s] = np.dot(dy[t], yp[r])
    return dyp, dw


def dispatch_backward(dxp, inv_row, dx_shared=None):
    """xp[inv_row[t,s]] = x[t]  ->  dx."""
    T, K = inv_row.shape
    dx = np.zeros((T, dxp.shape[1])) if dx_shared is None else dx_shared.copy()
    for t in range(T):
        for s in range(K):
            if inv_row[t, s] >= 0:
                dx[t] += dxp[inv_row[t, s]]
    return dx


def route_backward(topk_idx, topk_w, dtopk_w, E):
    """w = softmax of the chosen logits  ->  dlogits, through the Jacobian dw_i/dl_j = w_i (delta_ij - w_j)."""
    T, K = topk_idx.shape
    dl = np.zeros((T, E))
    for t in range(T):
        w = topk_w[t].astype(np.float64)
        jac = np.diag(w) - np.outer(w, w)
        for s in range(K):
            dl[t, topk_idx[t, s]] += jac[s] @ dtopk_w[t]
    return dl


def checkpoint_encode(v):
    """v [rows, F] -> (codes int8 [rows, F], exps uint8 [F/16, rows])."""
    rows, F = v.shape
    codes = np.zeros((rows, F), dtype=np.int8)
    exps = np.zeros((F // BLOCK, rows), dtype=np.uint8)
    for r in range(rows):
        for b in range(F // BLOCK):
            x = v[r, b * BLOCK:(b + 1) * BLOCK].astype(np.float64)
            if not np.isfinite(x).all():
                exps[b, r] = 255
                continue
            big = np.max(np.abs(x))
            biased = 127 + int(np.floor(np.log2(big))) if big > 0 else 0
            if big > 0 and 2.0 ** (biased - 127) > big:      # log2 rounded up to the next power
                biased -= 1
            e = max(biased - 6, 1)
            exps[b, r] = e
            codes[r, b * BLOCK:(b + 1) * BLOCK] = np.clip(np.rint(x * 2.0 ** (127 - e)), -127, 127)
    return codes, exps


def checkpoint_decode(codes, exps):
    """(codes [rows, F], exps [F/16, rows]) -> the values kept, NaN in blocks with exponent 255."""
    e = exps.astype(np.float64).T                                   # [rows, F/16]
    scale = np.where(e == 255, np.nan, 2.0 ** (e - 127.0))
    return codes.astype(np.float64) * np.repeat(scale, BLOCK, axis=1)


def swiglu_ffn(x, wg, wu, wd):
    """x [n, H] through one expert: (y, g, u)."""
    g, u = x @ wg.T, x @ wu.T
    return (g / (1.0 + np.exp(-g)) * u) @ wd.T, g, u


def swiglu_ffn_backward(x, dy, g, u, wg, wu, wd):
    """Gradients of swiglu_ffn at x, given the gate and up values to use: (dx, dwg, dwu, dwd, dg, du, act)."""
    sig = 1.0 / (1.0 + np.exp(-g))
    act = g * sig * u
    da = dy @ wd
    du = da * g * sig
    dg = da * u * (sig + g * sig * (1.0 - sig))
    return dg @ wg + du @ wu, dg.T @ x, du.T @ x, dy.T @ act, dg, du, act


def expert_ffn_backward(xp, dyp, seg_offsets, slot_expert, g, u, w_gate, w_up, w_down):
    """Grouped: the rows of segment g belong to expert slot_expert[g]; an expert's weight gradients sum over all of its
    segments (its replicas share one weight array).  Returns (dxp, dw_gate, dw_up, dw_down)."""
    dxp = np.zeros_like(xp)
    dw = [np.zeros(w.shape, dtype=np.float64) for w in (w_gate, w_up, w_down)]
    for k, e in enumerate(slot_expert):
        lo, hi = int(seg_offsets[k]), int(seg_offsets[k + 1])
        if hi <= lo or e < 0:
            continue
        s = slice(lo, hi)
        dxp[s], a, b, c, _, _, _ = swiglu_ffn_backward(xp[s], dyp[s], g[s], u[s], w_gate[e], w_up[e], w_down[e])
        dw[0][e] += a
        dw[1][e] += b
        dw[2][e] += c
    return dxp, dw[0], dw[1], dw[2]
