"""AdamW's C entry point with masters and moments at any address that is a multiple of four bytes."""
import ctypes
import types

import pytest

pytestmark = pytest.mark.gpu

GUARD = 64


def _place(values, shift):
    """The values `shift` elements behind an aligned address; and the buffer that they lie in, NaN around them."""
    import torch
    room = torch.full((values.numel() + 2 * GUARD,), float("nan"), dtype=values.dtype, device="cuda")
    part = room[GUARD + shift:GUARD + shift + values.numel()]
    part.copy_(values)
    assert part.data_ptr() % 32 == (room.data_ptr() + (GUARD + shift) * values.element_size()) % 32
    return part, room


@pytest.mark.parametrize("which", ["master", "exp_avg", "exp_avg_sq", "all"])
@pytest.mark.parametrize("shift", [1, 2, 3, 4, 5, 6, 7])
@pytest.mark.parametrize("sizes", [(9000, 5, 2048), (900_000, 4097, 77)], ids=["one launch", "several"])
def test_state_at_odd_addresses(sizes, shift, which):
    """Several chunks of 2048 weights each, whole and ragged; two steps.  296 chunks are the most of one launch on 148 SMs."""
    import torch
    from paper_2607_08782_b200 import binding
    from paper_2607_08782_b200.binding import BF16, FP32, DirectorAdamW, DirectorParam, DirectorTensor
    from test_gpu_training import _Reference
    g = torch.Generator(device="cuda").manual_seed(shift)
    kinds = [torch.bfloat16, torch.float32, torch.bfloat16]
    at = {n: shift if which in (n, "all") else 0 for n in ("master", "exp_avg", "exp_avg_sq")}
    weights, masters, ms, vs, grads, rooms = [], [], [], [], [], []

    def keep(values, shift):
        part, room = _place(values, shift)
        rooms.append((room, part.data_ptr() - room.data_ptr(), part))
        return part
    params, tensors = (DirectorParam * 3)(), (DirectorTensor * 3)()
    for i, (n, kind) in enumerate(zip(sizes, kinds)):
        start = torch.randn(n, generator=g, device="cuda") * 0.1
        weights.append(keep(start.to(kind), 0))
        masters.append(keep(start, at["master"]) if kind is torch.bfloat16 else None)
        ms.append(keep(torch.randn(n, generator=g, device="cuda") * 1e-3, at["exp_avg"]))
        vs.append(keep(torch.rand(n, generator=g, device="cuda") * 1e-5, at["exp_avg_sq"]))
        grads.append((torch.randn(n, generator=g, device="cuda") * 1e-2).to(kinds[(i + 1) % 3]))
        p, t = params[i], tensors[i]
        p.weight, p.numel, p.type = weights[i].data_ptr(), n, BF16 if kind is torch.bfloat16 else FP32
        p.master = masters[i].data_ptr() if masters[i] is not None else None
        p.exp_avg, p.exp_avg_sq = ms[i].data_ptr(), vs[i].data_ptr()
        t.data, t.numel, t.type = grads[i].data_ptr(), n, BF16 if grads[i].dtype is torch.bfloat16 else FP32
    lib = binding.load_library()
    steps, status = torch.full((1,), 10, dtype=torch.int64, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    norm, work = torch.zeros(1, device="cuda"), torch.empty(lib.director_grad_workspace_bytes(), dtype=torch.uint8, device="cuda")
    opt = types.SimpleNamespace(weights=weights, masters=masters, exp_avg=ms, exp_avg_sq=vs, steps=steps, betas=(0.9, 0.95), eps=1e-8, weight_decay=0.1)
    h = DirectorAdamW(3e-3, 0.9, 0.95, 1e-8, 0.1, 0.5)
    for _ in range(2):
        ref = _Reference(opt)
        rc = lib.director_adamw_step(3, tensors, params, ctypes.byref(h), None, steps.data_ptr(), norm.data_ptr(), status.data_ptr(), work.data_ptr(),
                                     torch.cuda.current_stream().cuda_stream)
        assert rc == 0
        ref.step(grads, 3e-3, 0.5)
    assert int(status) == 0
    for room, offset, part in rooms:
        first = offset // room.element_size()
        assert room[:first].isnan().all() and room[first + part.numel():].isnan().all(), "what lies around an array stays"
