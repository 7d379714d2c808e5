"""From the gradients of a training step to the next weights: the global gradient norm, clipping by it, and AdamW with the clipping
done on the way.  Any number of tensors, of a layer or of a whole model, bf16 or fp32 each.

    grads = TensorList([layer.grads[n] for n in ("w_gate", "w_up", "w_down")])     # buffers that stay where they are
    optimizer = AdamW(layer.w, lr=1e-4, max_norm=1.0)
    ...
    norm = optimizer.step(grads)                  # or step() for the weights' .grad, or step(list of tensors)

Everything runs on the current stream and can be captured into a CUDA graph; nothing is read back.  Results have the same bits on
every run.  Marshalling only: the work is done by the library's kernels (see include/director.h)."""
from __future__ import annotations

import ctypes
import math

import torch

from . import binding
from .binding import BF16, FP32, SMALL_BYTES, SMALL_TENSORS, DirectorAdamW, DirectorError, DirectorParam, DirectorTensor, _check, load_library

_TYPES = {torch.float32: FP32, torch.bfloat16: BF16}


class TensorList:
    """Tensors that calls take together: their addresses, looked up once.  Contiguous fp32 or bf16 CUDA tensors of one device, of any
    size; None stands for a gradient that does not exist (AdamW.step leaves its weight as it is).  The list keeps the tensors; their
    memory has to stay where it is (in-place changes are fine, set_() or resize_() are not)."""

    def __init__(self, tensors):
        self.tensors = list(tensors)
        self.array = (DirectorTensor * max(1, len(self.tensors)))()
        self.shapes = [None if t is None else t.shape for t in self.tensors]
        self.device = None
        for i, t in enumerate(self.tensors):
            if t is None:
                continue
            kind = _TYPES.get(t.dtype)
            if kind is None:
                raise TypeError(f"tensor {i} is {t.dtype}, fp32 or bf16 is needed")
            if not t.is_cuda or not t.is_contiguous():
                raise ValueError(f"tensor {i} has to be a contiguous CUDA tensor")
            if self.device is None:
                self.device = t.device
            elif t.device != self.device:
                raise ValueError(f"tensor {i} is on {t.device}, the ones before it on {self.device}")
            a = self.array[i]
            a.data, a.numel, a.type = t.data_ptr(), t.numel(), kind
        self.live = [t for t in self.tensors if t is not None and not t.is_inference()]
        self.numels = [a.numel for a in self.array[:len(self.tensors)]]
        self.small = len(self.tensors) <= SMALL_TENSORS and sum(a.numel * (4 if a.type == FP32 else 2) for a in self.array) <= SMALL_BYTES
        if self.device is None:
            self.device = torch.device("cuda", torch.cuda.current_device())

    def __len__(self):
        return len(self.tensors)

    def __iter__(self):
        return iter(self.tensors)


def _as_list(tensors) -> TensorList:
    return tensors if isinstance(tensors, TensorList) else TensorList(tensors)


def _begin(device: torch.device):
    """The library and the current stream, which has to be one of the tensors' device."""
    lib = load_library()
    if binding._raw_stream is None:
        binding._bind_torch()
    current = binding._current_device()
    if device.index != current:
        raise ValueError(f"the tensors are on {device}, the current device is cuda:{current}")
    return lib, binding._stream()


_words = 0        # of a workspace, in fp32


def _norm_and_workspace(lib, device, small=False):
    """A place for the norm and, unless the call is small, the address of a workspace, in one allocation.  Made anew by each call, on its
    stream: calls that overlap, captured ones too, never share it."""
    if small:
        return torch.empty_strided((), (), dtype=torch.float32, device=device), None        # 0.9 us less than torch.empty(())
    global _words
    if _words == 0:
        _words = lib.director_grad_workspace_bytes() // 4
    room = torch.empty(_words + 1, dtype=torch.float32, device=device)
    return room[_words], room.data_ptr()


def grad_norm(grads) -> torch.Tensor:
    """The square root of the sum of squares over all elements of all tensors (a TensorList or a sequence): fp32, no dimensions."""
    grads = _as_list(grads)
    lib, stream = _begin(grads.device)
    norm, workspace = _norm_and_workspace(lib, grads.device, grads.small)
    _check(lib.director_grad_norm(len(grads), grads.array, norm.data_ptr(), workspace, stream), "director_grad_norm")
    return norm


def clip_grads(grads, max_norm: float, out=None) -> torch.Tensor:
    """Scales the gradients (a TensorList or a sequence) by min(1, max_norm / norm), in place or into `out` (tensors of the same
    lengths, fp32 or bf16: fp32 gradients for an optimizer that takes those), and returns the norm before clipping (fp32, no
    dimensions).  Where it is infinite or NaN nothing is scaled."""
    grads = _as_list(grads)
    out = grads if out is None else _as_list(out)
    if out.numels != grads.numels:
        raise ValueError("clip_grads: out has to have a tensor of the same length for every gradient")
    if not max_norm > 0:
        raise ValueError(f"clip_grads: max_norm is {max_norm}, a positive number is needed")
    if out.device != grads.device:
        raise ValueError(f"clip_grads: the gradients are on {grads.device}, out is on {out.device}")
    lib, stream = _begin(grads.device)
    norm, workspace = _norm_and_workspace(lib, grads.device)
    _check(lib.director_clip_grads(len(grads), grads.array, out.array, max_norm, norm.data_ptr(), workspace, stream), "director_clip_grads")
    torch.autograd.graph.increment_version(out.live)          # autograd is told that they were changed in place
    return norm


class AdamW:
    """AdamW over bf16 weights, each with an fp32 master, and fp32 weights (contiguous CUDA tensors that share no memory, kept by
    reference and updated in place, at the addresses that they and the state have now); Adam where weight_decay is 0.  Gradients above
    max_norm in their global norm are scaled down to it on the way (the gradients themselves stay as they are).  A step whose norm is
    infinite or NaN is skipped; with max_norm = infinity the norm is not taken, and such gradients reach the weights.  `lr` and the other
    numbers may be changed between steps; for a captured step, give `lr` as an fp32 CUDA tensor of one element, which the step reads when
    it runs.  One optimizer serves one stream at a time: its workspace and the norm that a step returns are its own.

    A step writes a bf16 weight from its master.  Weights that are given other values after the optimizer was made (a checkpoint is loaded)
    need masters_from_weights(): until then a step raises a RuntimeError.  It goes by autograd's count of in-place changes, so that it does not
    notice changes through .data, to weights that are part of a larger tensor (which has one count for all of it) or to inference tensors,
    nor by graph replays; those would be lost."""

    def __init__(self, weights, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.0, max_norm=math.inf):
        self.weights = list(weights)
        listed = TensorList(self.weights)
        if any(w is None for w in self.weights):
            raise ValueError("AdamW: a weight is None")
        self.device = listed.device
        self.lr, self.betas, self.eps, self.weight_decay, self.max_norm = lr, tuple(betas), eps, weight_decay, max_norm
        self.masters = [w.detach().float() if w.dtype is torch.bfloat16 else None for w in self.weights]
        self.exp_avg = [torch.zeros_like(w, dtype=torch.float32, requires_grad=False) for w in self.weights]
        self.exp_avg_sq = [torch.zeros_like(m) for m in self.exp_avg]
        self.steps = torch.zeros((1,), dtype=torch.int64, device=self.device)
        self.status = torch.zeros((1,), dtype=torch.int32, device=self.device)
        self._norm = torch.zeros((), dtype=torch.float32, device=self.device)
        self._workspace = torch.empty(load_library().director_grad_workspace_bytes(), dtype=torch.uint8, device=self.device)
        self._hyper, self._numbers, self._shapes, self._live = DirectorAdamW(), None, listed.shapes, listed.live
        self._hyper_at = ctypes.byref(self._hyper)
        self._addresses = [w.data_ptr() for w in self.weights]
        self._workspace_at, self._norm_at = self._workspace.data_ptr(), self._norm.data_ptr()
        # bf16 weights that have their memory, and so their count of in-place changes, to themselves; the counts' sum as of the last
        # time that weights and masters agreed.  The counts only grow.
        self._counted = [w for w, m in zip(self.weights, self.masters)
                         if m is not None and not w.is_inference() and w.untyped_storage().nbytes() == w.numel() * w.element_size()]
        self._changes = self._count_changes()
        self._params = (DirectorParam * max(1, len(self.weights)))()
        for i, w in enumerate(self.weights):
            p = self._params[i]
            p.weight, p.numel, p.type = w.data_ptr(), w.numel(), listed.array[i].type
            p.exp_avg, p.exp_avg_sq = self.exp_avg[i].data_ptr(), self.exp_avg_sq[i].data_ptr()
            p.master = self.masters[i].data_ptr() if self.masters[i] is not None else None

    def _count_changes(self) -> int:
        return sum([w._version for w in self._counted])

    def _check_weights(self):
        """Some bf16 weight was written since the last step: raises unless all are what their masters say (swapped out and back)."""
        advice = ("call masters_from_weights() to go on from the weights as they are, or load_state_dict(state_dict()) to go on from "
                  "the masters")
        if torch.cuda.is_current_stream_capturing():
            raise RuntimeError(f"AdamW.step: a bf16 weight was written since the last step, before this capture: {advice}")
        with torch.no_grad():
            for i, (w, m) in enumerate(zip(self.weights, self.masters)):
                for a, b in zip(w.view(-1).split(1 << 26), m.view(-1).split(1 << 26)) if m is not None else ():
                    b = b.to(torch.bfloat16)
                    if not ((a == b) | (a.isnan() & b.isnan())).all():
                        raise RuntimeError(f"AdamW.step: weight {i} was written since the last step, and would be overwritten from its master: {advice}")
        self._changes = self._count_changes()

    def masters_from_weights(self):
        """The masters become the bf16 weights as they are now (weights that were loaded into them); moments and step count stay."""
        with torch.no_grad():
            for w, m in zip(self.weights, self.masters):
                if m is not None:
                    m.copy_(w)
        self._changes = self._count_changes()

    def step(self, grads=None, lr=None) -> torch.Tensor | None:
        """One step on `grads` (a TensorList or a sequence, a tensor or None for each weight; default: the weights' .grad), with
        `lr` in place of the optimizer's if given (a number or an fp32 CUDA tensor of one element).  Returns the gradients' norm before
        clipping (fp32, no dimensions, overwritten by the next step), None where max_norm is infinite."""
        if [w.data_ptr() for w in self.weights] != self._addresses:
            raise RuntimeError("AdamW.step: a weight has moved to other memory since the optimizer was made")
        if sum([w._version for w in self._counted]) != self._changes:
            self._check_weights()
        grads = _as_list([w.grad for w in self.weights] if grads is None else grads)
        if grads.shapes != self._shapes:
            if len(grads) != len(self._shapes):
                raise ValueError(f"AdamW.step: {len(grads)} gradients for {len(self._shapes)} weights")
            for i, (g, w) in enumerate(zip(grads.shapes, self._shapes)):
                if g is not None and g != w:
                    raise ValueError(f"AdamW.step: gradient {i} is {tuple(g)}, its weight {tuple(w)}")
        if grads.device != self.device:
            raise ValueError(f"AdamW.step: the gradients are on {grads.device}, the weights on {self.device}")
        lib, stream = _begin(self.device)
        lr = self.lr if lr is None else lr
        lr_dev = None
        if type(lr) is not float and isinstance(lr, torch.Tensor):
            if lr.dtype is not torch.float32 or lr.numel() != 1 or lr.device != self.device:
                raise ValueError("AdamW.step: lr has to be a number or an fp32 tensor of one element on the weights' device")
            lr_dev, lr = lr.data_ptr(), 0.0
        beta1, beta2 = self.betas
        numbers = (lr, beta1, beta2, self.eps, self.weight_decay, self.max_norm)
        if numbers != self._numbers:                          # 0.2 us less than writing them each time
            h = self._hyper
            h.lr, h.beta1, h.beta2, h.eps, h.weight_decay, h.max_norm = numbers
            self._numbers = numbers
        norm, norm_at = (self._norm, self._norm_at) if self.max_norm != math.inf else (None, None)
        _check(lib.director_adamw_step(len(self._shapes), grads.array, self._params, self._hyper_at, lr_dev, self.steps.data_ptr(), norm_at,
                                       self.status.data_ptr(), self._workspace_at, stream),
               "director_adamw_step")
        torch.autograd.graph.increment_version(self._live)         # autograd is told that they were changed in place
        self._changes += len(self._counted)
        return norm

    def last_status(self) -> int:
        """Waits for the current stream; 8 (DIRECTOR_ERR_NONFINITE) if a step was skipped since the last call, else 0."""
        status = int(self.status.item())
        self.status.zero_()
        return status

    def check_status(self):
        """Raises a DirectorError if a step was skipped since the last call."""
        status = self.last_status()
        if status != 0:
            raise DirectorError(status, "AdamW.step")

    def state_dict(self) -> dict:
        """The state, as it is (no copies): steps, masters, exp_avg, exp_avg_sq."""
        return dict(steps=self.steps, masters=self.masters, exp_avg=self.exp_avg, exp_avg_sq=self.exp_avg_sq)

    def load_state_dict(self, state: dict):
        """Copies a state_dict() into this optimizer; the bf16 weights become their masters, rounded."""
        for name in ("masters", "exp_avg", "exp_avg_sq"):
            mine, theirs = getattr(self, name), list(state[name])
            if len(theirs) != len(mine) or any(m is not None and (t is None or t.shape != m.shape) for m, t in zip(mine, theirs)):
                raise ValueError(f"AdamW.load_state_dict: {name} does not fit the weights")
        with torch.no_grad():
            for name in ("masters", "exp_avg", "exp_avg_sq"):
                for m, t in zip(getattr(self, name), state[name]):
                    if m is not None:
                        m.copy_(t)
            for w, m in zip(self.weights, self.masters):
                if m is not None:
                    w.copy_(m)
            self.steps.copy_(state["steps"])
        self._changes = self._count_changes()
