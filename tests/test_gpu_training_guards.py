"""What the training calls have to notice: indexes out of range, buffers that are no longer a forward pass's own, arguments of
the wrong kind."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("K", [1, 2, 3, 6, 8])
@pytest.mark.parametrize("H", [256, 768])
def test_dispatch_backward_skips_and_reports_a_row_past_the_end(K, H):
    import torch
    from paper_2607_08782_b200.binding import Director
    T = 9
    A = T * K
    d = Director(T, H, 128, 8, K, 0, 2, 8)
    room = torch.full((A + 4, H), 100.0, dtype=torch.bfloat16, device="cuda")     # the rows behind the batch's are no part of it
    room[:A] = (torch.arange(A, device="cuda") % 16).to(torch.bfloat16).unsqueeze(1)
    inv = torch.randperm(A, generator=torch.Generator().manual_seed(K)).int().view(T, K).cuda()
    add = torch.full((T, H), 0.5, dtype=torch.bfloat16, device="cuda")
    for bad in (A, A + 3):
        table = inv.clone()
        table[4, K - 1] = bad
        for shared in (None, add):
            dx = torch.full((T, H), 7.0, dtype=torch.bfloat16, device="cuda")
            d.dispatch_backward(T, room, table, shared, dx)
            assert d.last_status() == 7 and d.last_status() == 0
            rows = room[:A].float()[table.clamp(max=A - 1).long()] * (table < A).unsqueeze(-1)
            assert torch.equal(dx.float(), rows.sum(1) + (0.5 if shared is not None else 0.0))    # small whole numbers: exact
    table[4, K - 1] = -1                                                          # nothing there is no error
    d.dispatch_backward(T, room, table, None, dx)
    assert d.last_status() == 0
