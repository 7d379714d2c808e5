"""Device-tensor convenience around the C entry points: owns the output tensors of one MoE layer
and calls the five stages in order on the current stream.  Allocation and marshalling only."""
from __future__ import annotations

import numpy as np
import torch

from .binding import Director, _need


def bf16_bits_to_tensor(bits: np.ndarray, device="cuda") -> torch.Tensor:
    """uint16 bf16 bit patterns (numpy) -> torch.bfloat16 tensor on `device` (bit-exact)."""
    t = torch.from_numpy(np.ascontiguousarray(bits).view(np.int16))
    return t.to(device).view(torch.bfloat16)


def tensor_to_bf16_bits(t: torch.Tensor) -> np.ndarray:
    return t.detach().contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


class LayerGraph(torch.cuda.CUDAGraph):
    """A captured pass of a layer.  Its replays write to the layer's buffers, as the pass itself does."""
    layer = None
    T = 0

    def replay(self):
        self.layer._give_up_pass()
        self.layer.routed = self.T
        super().replay()


class MoELayer:
    """Routed experts w_gate/w_up [E,F,H], w_down [E,H,F]; optional shared experts ws_gate/ws_up [S*F,H],
    ws_down [H,S*F] (all torch.bfloat16 CUDA tensors, kept by reference)."""

    def __init__(self, T_max, H, F, E, K, S, R, C_max, w_gate, w_up, w_down, ws_gate=None, ws_up=None,
                 ws_down=None, device="cuda"):
        self.dims = dict(T_max=T_max, H=H, F=F, E=E, K=K, S=S, R=R, C_max=C_max)
        self.d = Director(T_max, H, F, E, K, S, R, C_max)
        self.ffn_variant = 2
        # (T, x, placement, pass) of the training forward whose buffers are intact: its backward pass may run.  No two passes of
        # the layer have the same number.
        self.trained = None
        self.passes = 0
        self.routed = 0            # tokens whose choices topk_idx and topk_w hold
        # (T, logits, token_mask, pass, number) of the pass's balance_loss() whose counts are intact; no two of them have the same number.
        self.balanced = None
        self.balances = 0
        self.w = (w_gate, w_up, w_down)
        self.ws = (ws_gate, ws_up, ws_down)
        A, G = T_max * K, R * C_max
        i32 = dict(dtype=torch.int32, device=device)
        self.topk_idx = torch.empty((T_max, K), **i32)
        self.topk_w = torch.empty((T_max, K), dtype=torch.float32, device=device)
        self.xp = torch.empty((A, H), dtype=torch.bfloat16, device=device)
        self.yp = torch.empty((A, H), dtype=torch.bfloat16, device=device)
        self.row_token = torch.empty((A,), **i32)
        self.inv_row = torch.empty((T_max, K), **i32)
        self.dest_rank = torch.empty((T_max, K), **i32)
        self.seg_offsets = torch.empty((G + 1,), **i32)
        self.y = torch.empty((T_max, H), dtype=torch.bfloat16, device=device)
        self.y_shared = torch.empty((T_max, H), dtype=torch.bfloat16, device=device) if S > 0 else None
        i64 = dict(dtype=torch.int64, device=device)
        self.workload = torch.empty((R, E), **i64)
        self.rank_load = torch.empty((R,), **i64)
        self.dispatch_tokens = torch.empty((R, R), **i64)
        self.dispatch_bytes = torch.empty((R, R), **i64)     # bit pattern of uint64

    def _give_up_pass(self):
        """No backward pass of the last training forward may run any more; what it would have read of the caller's is let go."""
        self.trained = self.balanced = None

    def set_placement(self, X: np.ndarray):
        self.d.set_placement(X)

    def set_ffn_variant(self, variant: int):
        """Tile scheme of the expert GEMMs (see director_set_ffn_variant); only scheme 2 can gather from x."""
        self.d.set_ffn_variant(variant)
        self.ffn_variant = variant

    def route(self, T, logits):
        self._give_up_pass()
        self.d.route(T, logits, self.topk_idx, self.topk_w)
        self.routed = T

    def set_replica_policy(self, policy: int):
        """0: round-robin over an expert's replicas; 1: locality first (see director_set_replica_policy)."""
        self.d.set_replica_policy(policy)

    def dispatch(self, T, x, indices_only=False, token_src_rank=None):
        self._give_up_pass()
        xp = None if indices_only else self.xp
        if token_src_rank is None:
            self.d.dispatch(T, x, self.topk_idx, xp, self.row_token, self.inv_row, self.dest_rank, self.seg_offsets)
        else:
            self.d.dispatch_src(T, x, self.topk_idx, token_src_rank, xp, self.row_token, self.inv_row,
                                self.dest_rank, self.seg_offsets)

    def dedup_dispatch_tokens(self, T, token_src_rank=None):
        """[R,R] int64: tokens each rank sends to each rank when a token goes to a rank once (after dispatch)."""
        R = self.dims["R"]
        if getattr(self, "dedup_tokens", None) is None:
            self.dedup_tokens = torch.empty((R, R), dtype=torch.int64, device=self.topk_idx.device)
        self.d.dedup_dispatch_tokens(T, self.dest_rank, token_src_rank, self.dedup_tokens)
        return self.dedup_tokens

    def expert_ffn_gather(self, T, x):
        """The routed experts read their rows from x through row_token (no permuted copy)."""
        S = self.dims["S"]
        self._give_up_pass()
        self.d.expert_ffn_gather(T, x, self.row_token, self.seg_offsets, *self.w, self.yp,
                                 *(self.ws if S > 0 else (None, None, None)), self.y_shared if S > 0 else None)

    def expert_ffn(self, T, x=None):
        S = self.dims["S"]
        self._give_up_pass()
        self.d.expert_ffn(T, self.xp, self.seg_offsets, *self.w, self.yp,
                          x if S > 0 else None, *(self.ws if S > 0 else (None, None, None)),
                          self.y_shared if S > 0 else None)

    def combine(self, T):
        self.d.combine(T, self.yp, self.inv_row, self.topk_w, self.y_shared, self.y)

    def expert_ffn_combine(self, T, x=None):
        """Expert FFN with the combine fused into the down projection's epilogue (fp32 atomic adds into an accumulator
        of y: not bit-reproducible, and slower than the two separate steps - see director_expert_ffn_combine)."""
        d = self.dims
        if getattr(self, "y_acc", None) is None:
            dev = self.y.device
            self.y_acc = torch.empty((d["T_max"], d["H"]), dtype=torch.float32, device=dev)
            self.row_weight = torch.empty((d["T_max"] * d["K"],), dtype=torch.float32, device=dev)
        S = d["S"]
        self.d.expert_ffn_combine(T, self.xp, self.seg_offsets, self.row_token, self.inv_row, self.topk_w, *self.w,
                                  x if S > 0 else None, *(self.ws if S > 0 else (None, None, None)), self.y_acc,
                                  self.row_weight, self.y)

    # -- training ----------------------------------------------------------------------------------
    def enable_training(self):
        """Allocates what a training step keeps between its two passes (the 8-bit gate and up values) and its gradients; a layer
        that only serves never holds them.  Calling it again does nothing."""
        if getattr(self, "grads", None) is not None:
            return
        d, dev = self.dims, self.y.device
        T, A, H, F, SF = d["T_max"], d["T_max"] * d["K"], d["H"], d["F"], d["S"] * d["F"]
        self.d.reserve_training()
        self.kept = (torch.empty((A, F, 2), dtype=torch.int8, device=dev), torch.empty((F // 16, A, 2), dtype=torch.uint8, device=dev))
        self.dyp, self.dxp = torch.empty_like(self.yp), torch.empty_like(self.xp)
        self.dtopk_w = torch.empty_like(self.topk_w)
        grads = dict(x=torch.empty((T, H), dtype=torch.bfloat16, device=dev),
                     logits=torch.empty((T, d["E"]), dtype=torch.float32, device=dev),
                     **{n: torch.empty_like(w) for n, w in zip(("w_gate", "w_up", "w_down"), self.w)})
        if SF > 0:
            self.kept_shared = (torch.empty((T, SF, 2), dtype=torch.int8, device=dev),
                                torch.empty((SF // 16, T, 2), dtype=torch.uint8, device=dev))
            self.dx_shared = torch.empty_like(grads["x"])
            grads.update({n: torch.empty_like(w) for n, w in zip(("ws_gate", "ws_up", "ws_down"), self.ws)})
        self.grads = grads

    def forward_train(self, T, logits, x, token_src_rank=None):
        """The layer's forward pass, keeping what backward() needs (xp, yp, the gate's weights, the 8-bit gate and up values) in the
        layer's buffers; returns y[:T].  x has to stay as it is until backward(), and so have the weights.  Another pass of the layer
        takes the buffers, and so does a replay of capture()'s graph; replays of a graph that was captured in some other way go
        unnoticed, and must not come between the two passes.  token_src_rank (int32 [T]): see dispatch()."""
        _need("forward_train", ("logits", logits, torch.float32, T * self.dims["E"]), ("x", x, torch.bfloat16, T * self.dims["H"]))
        if token_src_rank is not None:
            _need("forward_train", ("token_src_rank", token_src_rank, torch.int32, T))
        self.enable_training()
        self.route(T, logits)
        self.dispatch(T, x, token_src_rank=token_src_rank)
        shared = (x, *self.ws, *self.kept_shared, self.y_shared) if self.dims["S"] > 0 else ()
        self.d.expert_ffn_checkpoint(T, self.xp, self.seg_offsets, *self.w, *self.kept, self.yp, *shared)
        self.combine(T)
        self.passes += 1
        self.trained = (T, x.detach(), self.d.placement_id(), self.passes)     # x without the graph that made it
        return self.y[:T]

    def balance_loss(self, T, logits, token_mask=None):
        """The router's balance term over the batch that forward_train() (or route()) just took, E sum_e f_e P_e, fp32 [1], and the
        experts' counts, int64 [E+1], the last entry the number of valid tokens (see director_balance_loss): buffers of the layer,
        overwritten by the next call.  logits: as for forward_train(); they and token_mask (uint8 or bool [T], 0 for padding) have
        to stay as they are until backward().  For more tokens than the layer routed last it raises a RuntimeError."""
        if self.trained is not None and self.trained[0] != T:
            raise RuntimeError(f"balance_loss() of {T} tokens after a forward_train() of {self.trained[0]}")
        if T > self.routed:                               # the places behind hold another batch's choices, or nothing
            raise RuntimeError(f"balance_loss() of {T} tokens, but the layer has routed {self.routed}")
        if getattr(self, "balance", None) is None:
            dev = self.y.device
            self.balance = (torch.empty((1,), dtype=torch.float32, device=dev), torch.empty((self.dims["E"] + 1,), dtype=torch.int64, device=dev))
        self.balanced = None
        self.d.balance_loss(T, logits, self.topk_idx, token_mask, *self.balance)
        self.balances += 1
        if self.trained is not None:                      # else there is no backward pass to keep them for
            self.balanced = (T, logits.detach(), token_mask, self.passes, self.balances)
        return self.balance

    def backward(self, T, dy, dbalance=None):
        """Gradients of the forward_train() before, given dy = dL/dy [T,H] (bf16): a dict of x [T,H], logits [T,E], w_gate, w_up,
        w_down and, with shared experts, ws_gate, ws_up, ws_down - views of the layer's buffers, overwritten by the next call.
        dbalance: dL/d balance_loss(), fp32 [1], whose part of the logits' gradient is added (after a balance_loss() of this pass).
        Under another placement than forward_train()'s, or after another pass of the layer, it raises a RuntimeError."""
        if self.trained is None or self.trained[0] != T:
            raise RuntimeError("backward() needs the buffers of a forward_train() of the same batch size, with no pass of the layer in between")
        _, x, placement, number = self.trained
        if self.d.placement_id() != placement:            # the rows lie in its segments, and the gradients read its tables
            raise RuntimeError("backward() needs the placement that forward_train() ran under, which has been changed since")
        if dbalance is not None and (self.balanced is None or self.balanced[0] != T or self.balanced[3] != number):
            raise RuntimeError("backward() with dbalance needs a balance_loss() of the pass")
        balanced = self.balanced
        _need("backward", ("dy", dy, torch.bfloat16, T * self.dims["H"]))
        if dbalance is not None:
            _need("backward", ("dbalance", dbalance, torch.float32, 1))
        self._give_up_pass()
        g = self.grads
        self.d.combine_backward(T, dy, self.yp, self.inv_row, self.topk_w, self.dyp, self.dtopk_w)
        with_shared = self.dims["S"] > 0
        shared = (x, dy, *self.kept_shared, *self.ws, self.dx_shared, g["ws_gate"], g["ws_up"], g["ws_down"]) if with_shared else ()
        self.d.expert_ffn_backward(T, self.xp, self.dyp, self.seg_offsets, *self.kept, *self.w, self.dxp, g["w_gate"], g["w_up"],
                                   g["w_down"], *shared)
        self.d.dispatch_backward(T, self.dxp, self.inv_row, self.dx_shared if with_shared else None, g["x"])
        self.d.route_backward(T, self.topk_idx, self.topk_w, self.dtopk_w, g["logits"])
        if dbalance is not None:
            logits, mask = balanced[1:3]
            self.d.balance_loss_backward(T, logits, self.balance[1], mask, dbalance, g["logits"], g["logits"])
        return {n: t[:T] if n in ("x", "logits") else t for n, t in g.items()}

    def placement_cost(self, T, token_src_rank=None):
        self.d.placement_cost(T, self.topk_idx, token_src_rank, self.workload, self.rank_load,
                              self.dispatch_tokens, self.dispatch_bytes)

    def forward(self, T, logits, x, with_cost=True, fused=False, fused_combine=False):
        """One pass of the whole layer on device tensors; returns y[:T] (a view of the owned buffer).
        fused: dispatch produces indices only and the expert GEMM gathers its rows from x.  Off by default: the
        weight-stationary GEMM re-reads a token tile once per weight block, so the gather is repeated 2F/256 times
        and costs more than the single row copy it saves."""
        # a batch small enough for the weight-streaming FFN kernels needs no permuted copy either: they stage a
        # segment's few rows from x themselves
        gather = (fused and self.ffn_variant == 2) or (self.d.batch_streams_weights(T) and not fused_combine)
        self._give_up_pass()
        if with_cost:          # front end in one call (a single launch for decode-sized batches)
            self.d.route_dispatch_cost(T, logits, x, self.topk_idx, self.topk_w, None if gather else self.xp,
                                       self.row_token, self.inv_row, self.dest_rank, self.seg_offsets, self.workload,
                                       self.rank_load, self.dispatch_tokens, self.dispatch_bytes)
            self.routed = T
        else:
            self.route(T, logits)
            self.dispatch(T, x, indices_only=gather)
        if fused_combine and not gather:          # combine inside the down projection (opt-in, see expert_ffn_combine)
            self.expert_ffn_combine(T, x)
            return self.y[:T]
        if gather:
            self.expert_ffn_gather(T, x)
        else:
            self.expert_ffn(T, x)
        self.combine(T)
        return self.y[:T]

    def capture(self, T, logits, x, with_cost=True, fused=False, fused_combine=False):
        """Records one pass of the layer (fixed T, fixed input and output buffers) into a CUDA graph and returns it;
        `graph.replay()` re-runs the pass with a single launch, which matters for decode-sized batches where the
        handful of kernel launches cost more than the kernels.  Per-kernel profiling must be off while capturing."""
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):                      # first pass outside the capture: lazy module loading
            self.forward(T, logits, x, with_cost, fused, fused_combine)
        torch.cuda.current_stream().wait_stream(side)
        graph = LayerGraph()
        graph.layer, graph.T = self, T
        with torch.cuda.graph(graph):
            self.forward(T, logits, x, with_cost, fused, fused_combine)
        return graph
