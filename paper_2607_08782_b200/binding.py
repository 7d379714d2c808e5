"""Thin ctypes binding of ``libdirector.so`` (see ``include/director.h``).

Argument marshalling only: torch tensors supply device memory and the current CUDA stream; every
step of the layer runs in the library's own kernels.  There is no fallback: if the library is
missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes
from ctypes import POINTER, c_char_p, c_double, c_float, c_int, c_int32, c_int64, c_uint8, c_uint64, c_void_p

from . import build as _build

STATUS_NAMES = {
    0: "DIRECTOR_OK", 1: "DIRECTOR_ERR_INVALID_ARG", 2: "DIRECTOR_ERR_PLACEMENT", 3: "DIRECTOR_ERR_WORKSPACE",
    4: "DIRECTOR_ERR_CUDA", 5: "DIRECTOR_ERR_UNSUPPORTED", 6: "DIRECTOR_ERR_TIMEOUT", 7: "DIRECTOR_ERR_BAD_INDEX",
    8: "DIRECTOR_ERR_NONFINITE", 9: "DIRECTOR_ERR_STATIC_LIMIT",
}

# every symbol include/director.h declares
EXPORTED = (
    "director_create", "director_destroy", "director_set_placement", "director_route", "director_dispatch",
    "director_expert_ffn", "director_combine", "director_placement_cost", "director_layer_forward_host",
    "director_last_status", "director_launch_count", "director_set_profiling", "director_kernel_time",
    "director_status_string", "director_dispatch_index_static", "director_layer_submit_host",
    "director_layer_wait_host", "director_set_ffn_variant", "director_batch_streams_weights", "director_expert_ffn_combine", "director_placement_cost_batch",
    "director_expert_ffn_gather", "director_set_replica_policy", "director_dispatch_src",
    "director_dedup_dispatch_tokens", "director_route_dispatch_cost", "director_layer_forward",
    "director_reserve_placements", "director_select_placement", "director_set_profiling_filter",
    "director_selftest_bounded_wait", "director_gemm_sm_mhz", "director_gemm_counters",
    "director_combine_backward", "director_dispatch_backward", "director_route_backward",
    "director_expert_ffn_checkpoint", "director_checkpoint_decode", "director_reserve_training",
    "director_expert_ffn_backward", "director_balance_loss", "director_balance_loss_backward", "director_grad_workspace_bytes",
    "director_grad_norm", "director_clip_grads", "director_adamw_step",
)

REPLICA_ROUND_ROBIN, REPLICA_LOCAL_FIRST = 0, 1


class DirectorShape(ctypes.Structure):
    _fields_ = [(n, c_int32) for n in ("T_max", "H", "F", "E", "K", "S", "R", "C_max")]


class DirectorTensor(ctypes.Structure):
    _fields_ = [("data", c_void_p), ("numel", c_int64), ("type", c_int32), ("reserved", c_int32)]


class DirectorParam(ctypes.Structure):
    _fields_ = [("weight", c_void_p), ("master", c_void_p), ("exp_avg", c_void_p), ("exp_avg_sq", c_void_p), ("numel", c_int64),
                ("type", c_int32), ("reserved", c_int32)]


class DirectorAdamW(ctypes.Structure):
    _fields_ = [(n, c_double) for n in ("lr", "beta1", "beta2", "eps", "weight_decay", "max_norm")]


FP32, BF16 = 0, 1
SMALL_TENSORS, SMALL_BYTES = 64, 4 << 20          # what director_grad_norm needs no workspace for


class DirectorError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {STATUS_NAMES.get(status, status)}")


_lib = None


def load_library(rebuild_if_stale: bool = True) -> ctypes.CDLL:
    """Loads libdirector.so from the package directory (building it first if the sources are newer).
    Raises if it cannot be built or loaded - there is no other implementation to fall back to."""
    global _lib
    if _lib is not None:
        return _lib
    path = _build.build_director() if rebuild_if_stale else _build.DIRECTOR_LIB
    lib = ctypes.CDLL(str(path))
    vp = c_void_p
    lib.director_create.argtypes = [POINTER(DirectorShape), POINTER(vp)]
    lib.director_destroy.argtypes = [vp]
    lib.director_set_placement.argtypes = [vp, vp, vp]
    lib.director_route.argtypes = [vp, c_int32, vp, vp, vp, vp]
    lib.director_dispatch.argtypes = [vp, c_int32, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.director_expert_ffn.argtypes = [vp, c_int32] + [vp] * 12
    lib.director_expert_ffn_gather.argtypes = [vp, c_int32] + [vp] * 12
    lib.director_combine.argtypes = [vp, c_int32, vp, vp, vp, vp, vp, vp]
    lib.director_expert_ffn_combine.argtypes = [vp, c_int32] + [vp] * 16
    lib.director_placement_cost.argtypes = [vp, c_int32, vp, vp, vp, vp, vp, vp, vp]
    lib.director_layer_forward_host.argtypes = [vp, c_int32] + [vp] * 12
    lib.director_layer_forward.argtypes = [vp, c_int32] + [vp] * 14
    lib.director_placement_cost_batch.argtypes = [vp, vp, c_int32, vp, vp, vp, vp, vp]
    lib.director_layer_submit_host.argtypes = [vp, c_int32] + [vp] * 13
    lib.director_layer_wait_host.argtypes = [vp, c_int64]
    lib.director_dispatch_index_static.argtypes = [c_int32] * 5 + [vp] * 9
    lib.director_last_status.argtypes = [vp, vp]
    lib.director_launch_count.argtypes = [vp]
    lib.director_launch_count.restype = c_int64
    lib.director_set_profiling.argtypes = [vp, c_int32]
    lib.director_set_profiling_filter.argtypes = [vp, c_char_p]
    lib.director_set_ffn_variant.argtypes = [vp, c_int32]
    lib.director_batch_streams_weights.argtypes = [vp, c_int32]
    lib.director_set_replica_policy.argtypes = [vp, c_int32]
    lib.director_reserve_placements.argtypes = [vp, c_int32]
    lib.director_select_placement.argtypes = [vp, c_int32]
    lib.director_route_dispatch_cost.argtypes = [vp, c_int32] + [vp] * 14
    lib.director_dispatch_src.argtypes = [vp, c_int32] + [vp] * 9
    lib.director_dedup_dispatch_tokens.argtypes = [vp, c_int32, vp, vp, vp, vp]
    lib.director_selftest_bounded_wait.argtypes = [vp, c_uint64, vp, vp]
    lib.director_gemm_sm_mhz.argtypes = [vp, c_int32, POINTER(c_double)]
    lib.director_gemm_sm_mhz.restype = c_double
    lib.director_gemm_counters.argtypes = [vp, c_int32, POINTER(c_int64)]
    lib.director_combine_backward.argtypes = [vp, c_int32] + [vp] * 7
    lib.director_dispatch_backward.argtypes = [vp, c_int32] + [vp] * 5
    lib.director_route_backward.argtypes = [vp, c_int32] + [vp] * 5
    lib.director_expert_ffn_checkpoint.argtypes = [vp, c_int32] + [vp] * 16
    lib.director_reserve_training.argtypes = [vp]
    lib.director_expert_ffn_backward.argtypes = [vp, c_int32] + [vp] * 24
    lib.director_checkpoint_decode.argtypes = [vp, c_int32, c_int32] + [vp] * 5
    lib.director_balance_loss.argtypes = [vp, c_int32] + [vp] * 6
    lib.director_balance_loss_backward.argtypes = [vp, c_int32] + [vp] * 7
    lib.director_grad_workspace_bytes.argtypes = []
    lib.director_grad_norm.argtypes = [c_int32] + [vp] * 4
    lib.director_clip_grads.argtypes = [c_int32, vp, vp, c_float, vp, vp, vp]
    lib.director_adamw_step.argtypes = [c_int32] + [vp] * 9
    lib.director_kernel_time.argtypes = [vp, c_char_p, POINTER(c_int64)]
    lib.director_kernel_time.restype = c_double
    lib.director_status_string.argtypes = [c_int]
    lib.director_status_string.restype = c_char_p
    for name in EXPORTED:
        if name not in ("director_launch_count", "director_kernel_time", "director_status_string", "director_gemm_sm_mhz"):
            getattr(lib, name).restype = c_int
    lib.director_grad_workspace_bytes.restype = c_int64
    _lib = lib
    return lib


def _ptr(t):
    """Device (or host) address of a torch tensor / numpy array / None."""
    if t is None:
        return None
    if hasattr(t, "data_ptr"):
        return t.data_ptr()
    return t.ctypes.data


# torch's dtypes and its raw-stream query, looked up once by the first context (torch is imported no earlier than that)
_BF16 = _F32 = _I32 = _I64 = _I8 = _U8 = _BOOL = _raw_stream = _current_device = None


def _bind_torch():
    global _BF16, _F32, _I32, _I64, _I8, _U8, _BOOL, _raw_stream, _current_device
    import torch
    _BF16, _F32, _I32, _I64, _I8, _U8, _BOOL = (torch.bfloat16, torch.float32, torch.int32, torch.int64, torch.int8, torch.uint8,
                                                torch.bool)
    _current_device = torch.cuda.current_device
    _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _need(where: str, *tensors):
    """Checks the tensors of a training call, (name, tensor, dtype, elements) each, and returns their addresses.  The C entry
    points see bare addresses; a tensor of another type, a strided view or one too short would be read as something else."""
    addresses = []
    for name, t, dtype, numel in tensors:
        if t.dtype is not dtype:
            raise TypeError(f"{where}: {name} is {t.dtype}, {dtype} is needed")
        if not t.is_contiguous() or not t.is_cuda:
            raise ValueError(f"{where}: {name} has to be a contiguous CUDA tensor")
        if t.numel() < numel:
            raise ValueError(f"{where}: {name} has {t.numel()} elements, {numel} are needed")
        addresses.append(t.data_ptr())
    return addresses


def _mask(where: str, mask, T: int):
    """Address of a token mask (uint8 or bool [T], a byte each), None for none."""
    if mask is None:
        return None
    return _need(where, ("token_mask", mask, _BOOL if mask.dtype is _BOOL else _U8, T))[0]


def _stream():
    """The current stream of the current device, as torch.cuda.current_stream() has it (which builds an object for it: 3 us, as
    long as a launch)."""
    if _raw_stream is not None:
        return _raw_stream(_current_device())
    import torch
    return torch.cuda.current_stream().cuda_stream


def _check(status: int, where: str):
    if status != 0:
        raise DirectorError(status, where)


class Director:
    """One MoE layer context: shape, placement and workspace.  Methods mirror the C entry points and
    take torch CUDA tensors (bf16 tensors as torch.bfloat16).  One context serves one stream at a time."""

    def __init__(self, T_max: int, H: int, F: int, E: int, K: int, S: int, R: int, C_max: int):
        self.lib = load_library()
        _bind_torch()
        self.shape = DirectorShape(T_max, H, F, E, K, S, R, C_max)
        self._ctx = c_void_p()
        _check(self.lib.director_create(ctypes.byref(self.shape), ctypes.byref(self._ctx)), "director_create")
        self._slot, self._fills = 0, {}

    def close(self):
        if getattr(self, "_ctx", None) is not None and self._ctx.value:
            self.lib.director_destroy(self._ctx)
            self._ctx = c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- placement -----------------------------------------------------------------------------
    def set_placement(self, X):
        """X: numpy uint8 [E, R] (C-contiguous)."""
        import numpy as np
        X = np.ascontiguousarray(X, dtype=np.uint8)
        assert X.shape == (self.shape.E, self.shape.R)
        _check(self.lib.director_set_placement(self._ctx, X.ctypes.data, _stream()), "director_set_placement")
        self._fills[self._slot] = self._fills.get(self._slot, 0) + 1

    def placement_id(self):
        """Names the current placement's tables: another value once set_placement() has filled the slot anew, or while
        another slot is selected."""
        return self._slot, self._fills.get(self._slot, 0)

    # -- stages --------------------------------------------------------------------------------
    def route(self, T, logits, topk_idx, topk_w):
        _check(self.lib.director_route(self._ctx, T, _ptr(logits), _ptr(topk_idx), _ptr(topk_w), _stream()),
               "director_route")

    def dispatch(self, T, x, topk_idx, xp, row_token, inv_row, dest_rank, seg_offsets):
        _check(self.lib.director_dispatch(self._ctx, T, _ptr(x), _ptr(topk_idx), _ptr(xp), _ptr(row_token),
                                          _ptr(inv_row), _ptr(dest_rank), _ptr(seg_offsets), _stream()),
               "director_dispatch")

    def route_dispatch_cost(self, T, logits, x, topk_idx, topk_w, xp, row_token, inv_row, dest_rank, seg_offsets,
                            workload, rank_load, dispatch_tokens, dispatch_bytes):
        _check(self.lib.director_route_dispatch_cost(
            self._ctx, T, _ptr(logits), _ptr(x), _ptr(topk_idx), _ptr(topk_w), _ptr(xp), _ptr(row_token), _ptr(inv_row),
            _ptr(dest_rank), _ptr(seg_offsets), _ptr(workload), _ptr(rank_load), _ptr(dispatch_tokens),
            _ptr(dispatch_bytes), _stream()), "director_route_dispatch_cost")

    def dispatch_src(self, T, x, topk_idx, token_src_rank, xp, row_token, inv_row, dest_rank, seg_offsets):
        _check(self.lib.director_dispatch_src(self._ctx, T, _ptr(x), _ptr(topk_idx), _ptr(token_src_rank), _ptr(xp),
                                              _ptr(row_token), _ptr(inv_row), _ptr(dest_rank), _ptr(seg_offsets),
                                              _stream()), "director_dispatch_src")

    def reserve_placements(self, n: int):
        _check(self.lib.director_reserve_placements(self._ctx, n), "director_reserve_placements")

    def select_placement(self, slot: int):
        _check(self.lib.director_select_placement(self._ctx, slot), "director_select_placement")
        self._slot = slot

    def set_replica_policy(self, policy: int):
        _check(self.lib.director_set_replica_policy(self._ctx, policy), "director_set_replica_policy")

    def dedup_dispatch_tokens(self, T, dest_rank, token_src_rank, dedup_tokens):
        _check(self.lib.director_dedup_dispatch_tokens(self._ctx, T, _ptr(dest_rank), _ptr(token_src_rank),
                                                       _ptr(dedup_tokens), _stream()),
               "director_dedup_dispatch_tokens")

    def expert_ffn(self, T, xp, seg_offsets, w_gate, w_up, w_down, yp, x=None, ws_gate=None, ws_up=None,
                   ws_down=None, y_shared=None):
        _check(self.lib.director_expert_ffn(self._ctx, T, _ptr(xp), _ptr(seg_offsets), _ptr(w_gate), _ptr(w_up),
                                            _ptr(w_down), _ptr(yp), _ptr(x), _ptr(ws_gate), _ptr(ws_up),
                                            _ptr(ws_down), _ptr(y_shared), _stream()), "director_expert_ffn")

    def expert_ffn_gather(self, T, x, row_token, seg_offsets, w_gate, w_up, w_down, yp, ws_gate=None, ws_up=None,
                          ws_down=None, y_shared=None):
        _check(self.lib.director_expert_ffn_gather(self._ctx, T, _ptr(x), _ptr(row_token), _ptr(seg_offsets),
                                                   _ptr(w_gate), _ptr(w_up), _ptr(w_down), _ptr(yp), _ptr(ws_gate),
                                                   _ptr(ws_up), _ptr(ws_down), _ptr(y_shared), _stream()),
               "director_expert_ffn_gather")

    def expert_ffn_combine(self, T, xp, seg_offsets, row_token, inv_row, topk_w, w_gate, w_up, w_down, x, ws_gate, ws_up,
                           ws_down, y_acc, row_weight, y):
        _check(self.lib.director_expert_ffn_combine(self._ctx, T, _ptr(xp), _ptr(seg_offsets), _ptr(row_token),
                                                    _ptr(inv_row), _ptr(topk_w), _ptr(w_gate), _ptr(w_up), _ptr(w_down),
                                                    _ptr(x), _ptr(ws_gate), _ptr(ws_up), _ptr(ws_down), _ptr(y_acc),
                                                    _ptr(row_weight), _ptr(y), _stream()), "director_expert_ffn_combine")

    def combine(self, T, yp, inv_row, topk_w, y_shared, y):
        _check(self.lib.director_combine(self._ctx, T, _ptr(yp), _ptr(inv_row), _ptr(topk_w), _ptr(y_shared),
                                         _ptr(y), _stream()), "director_combine")

    # -- backward pass -------------------------------------------------------------------------
    def combine_backward(self, T, dy, yp, inv_row, topk_w, dyp, dtopk_w):
        """Gradient of combine: dyp = each row's weight times its token's dy, dtopk_w = the dot products of dy and yp."""
        TK, H = T * self.shape.K, self.shape.H
        args = _need("combine_backward", ("dy", dy, _BF16, T * H), ("yp", yp, _BF16, TK * H), ("inv_row", inv_row, _I32, TK),
                     ("topk_w", topk_w, _F32, TK), ("dyp", dyp, _BF16, TK * H), ("dtopk_w", dtopk_w, _F32, TK))
        _check(self.lib.director_combine_backward(self._ctx, T, *args, _stream()), "director_combine_backward")

    def dispatch_backward(self, T, dxp, inv_row, dx_shared, dx):
        """Gradient of dispatch's row copies: dx = the sum of a token's rows of dxp (+ dx_shared, which may be None)."""
        TK, H = T * self.shape.K, self.shape.H
        dxp, inv_row, dx = _need("dispatch_backward", ("dxp", dxp, _BF16, TK * H), ("inv_row", inv_row, _I32, TK), ("dx", dx, _BF16, T * H))
        if dx_shared is not None:
            dx_shared, = _need("dispatch_backward", ("dx_shared", dx_shared, _BF16, T * H))
        _check(self.lib.director_dispatch_backward(self._ctx, T, dxp, inv_row, dx_shared, dx, _stream()), "director_dispatch_backward")

    def route_backward(self, T, topk_idx, topk_w, dtopk_w, dlogits):
        """Gradient of route: dlogits [T,E], zero where an expert was not chosen."""
        TK = T * self.shape.K
        args = _need("route_backward", ("topk_idx", topk_idx, _I32, TK), ("topk_w", topk_w, _F32, TK), ("dtopk_w", dtopk_w, _F32, TK),
                     ("dlogits", dlogits, _F32, T * self.shape.E))
        _check(self.lib.director_route_backward(self._ctx, T, *args, _stream()), "director_route_backward")

    # -- the router's balance term ---------------------------------------------------------------
    def balance_loss(self, T, logits, topk_idx, token_mask, loss, counts):
        """loss (fp32 [1]) and counts (int64 [E+1], the last entry the number of valid tokens) of a batch; token_mask: uint8 or
        bool [T], or None."""
        s = self.shape
        logits, topk_idx, loss, counts = _need("balance_loss", ("logits", logits, _F32, T * s.E), ("topk_idx", topk_idx, _I32, T * s.K),
                                               ("loss", loss, _F32, 1), ("counts", counts, _I64, s.E + 1))
        _check(self.lib.director_balance_loss(self._ctx, T, logits, topk_idx, _mask("balance_loss", token_mask, T), loss, counts, _stream()),
               "director_balance_loss")

    def balance_loss_backward(self, T, logits, counts, token_mask, dloss, added, dlogits):
        """dlogits = added (fp32 [T,E], may be dlogits itself, or None) + the balance term's gradient for dloss (fp32 [1])."""
        TE = T * self.shape.E
        logits, counts, dloss, dlogits = _need("balance_loss_backward", ("logits", logits, _F32, TE), ("counts", counts, _I64, self.shape.E + 1),
                                               ("dloss", dloss, _F32, 1), ("dlogits", dlogits, _F32, TE))
        if added is not None:
            added, = _need("balance_loss_backward", ("added", added, _F32, TE))
        _check(self.lib.director_balance_loss_backward(self._ctx, T, logits, counts, _mask("balance_loss_backward", token_mask, T), dloss,
                                                       added, dlogits, _stream()), "director_balance_loss_backward")

    def expert_ffn_checkpoint(self, T, xp, seg_offsets, w_gate, w_up, w_down, codes, exps, yp, x=None, ws_gate=None,
                              ws_up=None, ws_down=None, codes_shared=None, exps_shared=None, y_shared=None):
        """expert_ffn for training: also keeps the gate and up values in 8 bits (codes int8 [T*K,F,2], exps uint8
        [F/16,T*K,2]; the shared experts' likewise) for expert_ffn_backward."""
        s = self.shape
        TK = T * s.K
        W = s.E * s.F * s.H
        args = _need("expert_ffn_checkpoint", ("xp", xp, _BF16, TK * s.H), ("seg_offsets", seg_offsets, _I32, s.R * s.C_max + 1),
                     ("w_gate", w_gate, _BF16, W), ("w_up", w_up, _BF16, W), ("w_down", w_down, _BF16, W),
                     ("codes", codes, _I8, 2 * TK * s.F), ("exps", exps, _U8, TK * s.F // 8), ("yp", yp, _BF16, TK * s.H))
        shared = [None] * 7
        if s.S > 0 and x is not None:
            SF = s.S * s.F
            shared = _need("expert_ffn_checkpoint", ("x", x, _BF16, T * s.H), ("ws_gate", ws_gate, _BF16, SF * s.H),
                           ("ws_up", ws_up, _BF16, SF * s.H), ("ws_down", ws_down, _BF16, SF * s.H),
                           ("codes_shared", codes_shared, _I8, 2 * T * SF), ("exps_shared", exps_shared, _U8, T * SF // 8),
                           ("y_shared", y_shared, _BF16, T * s.H))
        _check(self.lib.director_expert_ffn_checkpoint(self._ctx, T, *args, *shared, _stream()), "director_expert_ffn_checkpoint")

    def reserve_training(self):
        """Allocates the workspace of expert_ffn_backward (once; later calls do nothing)."""
        _check(self.lib.director_reserve_training(self._ctx), "director_reserve_training")

    def expert_ffn_backward(self, T, xp, dyp, seg_offsets, codes, exps, w_gate, w_up, w_down, dxp, dw_gate, dw_up, dw_down,
                            x=None, dy=None, codes_shared=None, exps_shared=None, ws_gate=None, ws_up=None, ws_down=None,
                            dx_shared=None, dws_gate=None, dws_up=None, dws_down=None):
        """Gradients of expert_ffn_checkpoint from the gate and up values it kept (after reserve_training)."""
        s = self.shape
        TK, W = T * s.K, s.E * s.F * s.H
        args = _need("expert_ffn_backward", ("xp", xp, _BF16, TK * s.H), ("dyp", dyp, _BF16, TK * s.H),
                     ("seg_offsets", seg_offsets, _I32, s.R * s.C_max + 1), ("codes", codes, _I8, 2 * TK * s.F),
                     ("exps", exps, _U8, TK * s.F // 8), ("w_gate", w_gate, _BF16, W), ("w_up", w_up, _BF16, W),
                     ("w_down", w_down, _BF16, W), ("dxp", dxp, _BF16, TK * s.H), ("dw_gate", dw_gate, _BF16, W),
                     ("dw_up", dw_up, _BF16, W), ("dw_down", dw_down, _BF16, W))
        shared = [None] * 11
        if s.S > 0 and x is not None:
            SF = s.S * s.F
            shared = _need("expert_ffn_backward", ("x", x, _BF16, T * s.H), ("dy", dy, _BF16, T * s.H),
                           ("codes_shared", codes_shared, _I8, 2 * T * SF), ("exps_shared", exps_shared, _U8, T * SF // 8),
                           ("ws_gate", ws_gate, _BF16, SF * s.H), ("ws_up", ws_up, _BF16, SF * s.H),
                           ("ws_down", ws_down, _BF16, SF * s.H), ("dx_shared", dx_shared, _BF16, T * s.H),
                           ("dws_gate", dws_gate, _BF16, SF * s.H), ("dws_up", dws_up, _BF16, SF * s.H),
                           ("dws_down", dws_down, _BF16, SF * s.H))
        _check(self.lib.director_expert_ffn_backward(self._ctx, T, *args, *shared, _stream()), "director_expert_ffn_backward")

    def checkpoint_decode(self, rows, F, codes, exps, gate, up):
        """The values that a checkpoint of `rows` rows of F features stands for, into gate and up (bf16 [rows,F])."""
        args = _need("checkpoint_decode", ("codes", codes, _I8, 2 * rows * F), ("exps", exps, _U8, rows * F // 8),
                     ("gate", gate, _BF16, rows * F), ("up", up, _BF16, rows * F))
        _check(self.lib.director_checkpoint_decode(self._ctx, rows, F, *args, _stream()), "director_checkpoint_decode")

    def placement_cost(self, T, topk_idx, token_src_rank, workload, rank_load, dispatch_tokens, dispatch_bytes):
        _check(self.lib.director_placement_cost(self._ctx, T, _ptr(topk_idx), _ptr(token_src_rank), _ptr(workload),
                                                _ptr(rank_load), _ptr(dispatch_tokens), _ptr(dispatch_bytes),
                                                _stream()), "director_placement_cost")

    def placement_cost_batch(self, workload, n, X, rank_load, dispatch_tokens, summary):
        """n candidate placements X (CUDA uint8 [n,E,R]) against one workload matrix (CUDA int64 [R,E])."""
        _check(self.lib.director_placement_cost_batch(self._ctx, _ptr(workload), n, _ptr(X), _ptr(rank_load),
                                                      _ptr(dispatch_tokens), _ptr(summary), _stream()),
               "director_placement_cost_batch")

    def layer_forward(self, T, logits, x, w_gate, w_up, w_down, ws_gate, ws_up, ws_down, y, workload, rank_load,
                      dispatch_tokens, dispatch_bytes):
        """The whole layer on device tensors in one call (intermediates stay in the context's workspace)."""
        _check(self.lib.director_layer_forward(self._ctx, T, _ptr(logits), _ptr(x), _ptr(w_gate), _ptr(w_up),
                                               _ptr(w_down), _ptr(ws_gate), _ptr(ws_up), _ptr(ws_down), _ptr(y),
                                               _ptr(workload), _ptr(rank_load), _ptr(dispatch_tokens),
                                               _ptr(dispatch_bytes), _stream()), "director_layer_forward")

    def layer_forward_host(self, T, logits, x, w_gate, w_up, w_down, ws_gate, ws_up, ws_down, y,
                           rank_load=None, dispatch_bytes=None):
        """logits, x, y, rank_load, dispatch_bytes: host (pinned torch CPU tensors or numpy); weights: device."""
        _check(self.lib.director_layer_forward_host(self._ctx, T, _ptr(logits), _ptr(x), _ptr(w_gate), _ptr(w_up),
                                                    _ptr(w_down), _ptr(ws_gate), _ptr(ws_up), _ptr(ws_down), _ptr(y),
                                                    _ptr(rank_load), _ptr(dispatch_bytes), _stream()),
               "director_layer_forward_host")

    def layer_submit_host(self, T, logits, x, w_gate, w_up, w_down, ws_gate, ws_up, ws_down, y,
                          rank_load=None, dispatch_bytes=None) -> int:
        """Enqueues one batch (host buffers as for layer_forward_host) and returns its ticket; at most two
        batches may be in flight."""
        ticket = c_int64(-1)
        _check(self.lib.director_layer_submit_host(self._ctx, T, _ptr(logits), _ptr(x), _ptr(w_gate), _ptr(w_up),
                                                   _ptr(w_down), _ptr(ws_gate), _ptr(ws_up), _ptr(ws_down), _ptr(y),
                                                   _ptr(rank_load), _ptr(dispatch_bytes), _stream(),
                                                   ctypes.byref(ticket)), "director_layer_submit_host")
        return int(ticket.value)

    def layer_wait_host(self, ticket: int):
        _check(self.lib.director_layer_wait_host(self._ctx, ticket), "director_layer_wait_host")

    # -- status / instrumentation --------------------------------------------------------------
    def last_status(self) -> int:
        return int(self.lib.director_last_status(self._ctx, _stream()))

    def check_device_status(self):
        _check(self.last_status(), "device status")

    def selftest_bounded_wait(self, limit_ns: int, waited_ns=None):
        """Launches the kernel whose bounded wait expires by construction (see director_selftest_bounded_wait)."""
        _check(self.lib.director_selftest_bounded_wait(self._ctx, int(limit_ns), _ptr(waited_ns), _stream()),
               "director_selftest_bounded_wait")

    def set_ffn_variant(self, variant: int):
        _check(self.lib.director_set_ffn_variant(self._ctx, variant), "director_set_ffn_variant")

    def batch_streams_weights(self, T: int) -> bool:
        """True if a batch of T tokens takes the weight-streaming FFN kernels (which need no permuted copy of x)."""
        rc = int(self.lib.director_batch_streams_weights(self._ctx, T))
        if rc < 0:
            raise DirectorError(-rc, "director_batch_streams_weights")
        return rc == 1

    def gemm_sm_mhz(self, which: int = 0):
        """(SM MHz, longest CTA's microseconds) of the most recent gate|up (0) or down (1) GEMM launch, measured
        by the kernel itself (cycle counter against the global timer)."""
        busy = c_double(0.0)
        mhz = float(self.lib.director_gemm_sm_mhz(self._ctx, which, ctypes.byref(busy)))
        if mhz < 0:
            raise DirectorError(4, "director_gemm_sm_mhz")
        return mhz, float(busy.value)

    def gemm_counters(self, which: int = 0) -> dict:
        """What the most recent gate|up (0) or down (1) GEMM launch measured about itself (see
        director_gemm_counters), as derived figures."""
        raw = (c_int64 * 12)()
        _check(self.lib.director_gemm_counters(self._ctx, which, raw), "director_gemm_counters")
        c = [int(v) for v in raw]
        pairs = max(c[11] // 2, 1)
        return {
            "sm_mhz": c[0] / c[1] * 1e3 if c[1] else 0.0,
            "cycles_per_cta": c[0] / max(c[11], 1),
            "k_steps_per_pair": c[4] / pairs, "items_per_pair": c[5] / pairs,
            "cycles_per_k_step": c[3] / c[4] if c[4] else 0.0,
            "issuer_wait_for_accumulator_frac": c[2] / (c[0] / 2) if c[0] else 0.0,
            "issuer_k_loop_frac": c[3] / (c[0] / 2) if c[0] else 0.0,
            "epilogue_drain_cycles_per_tile": c[7] / c[8] if c[8] else 0.0,
            "epilogue_wait_cycles_per_tile": c[6] / c[8] if c[8] else 0.0,
            "longest_cta_us": c[10] * 1e-3,
        }

    def launch_count(self) -> int:
        return int(self.lib.director_launch_count(self._ctx))

    def set_profiling(self, enabled, only: str | None = None):
        """Device timing: True / 1 = events around every kernel, 2 = one pair of events around every stage, False /
        0 = off; `only`: time just the kernels whose name contains this string (per-kernel mode)."""
        _check(self.lib.director_set_profiling_filter(self._ctx, only.encode() if only else None),
               "director_set_profiling_filter")
        _check(self.lib.director_set_profiling(self._ctx, int(enabled)), "director_set_profiling")

    def kernel_time(self, name_substr: str):
        """(total milliseconds, launches) of kernels whose name contains name_substr since profiling was enabled."""
        n = c_int64(0)
        ms = float(self.lib.director_kernel_time(self._ctx, name_substr.encode(), ctypes.byref(n)))
        if ms < 0:
            raise DirectorError(4, "director_kernel_time")
        return ms, int(n.value)


def status_string(status: int) -> str:
    return load_library().director_status_string(status).decode()


def dispatch_index_static(T, K, E, R, C_max, topk_idx, rep_start, rep_slot, row_token, inv_row, dest_rank,
                          seg_offsets, device_status=None):
    """Context-free, allocation-free dispatch indices (director_dispatch_index_static): for callers
    that may not allocate device memory.  All tensor arguments are caller-owned CUDA int32 tensors."""
    st = load_library().director_dispatch_index_static(
        T, K, E, R, C_max, _ptr(topk_idx), _ptr(rep_start), _ptr(rep_slot), _ptr(row_token), _ptr(inv_row),
        _ptr(dest_rank), _ptr(seg_offsets), _ptr(device_status), _stream())
    _check(st, "director_dispatch_index_static")
