"""The FFN gradient with full token tiles.  A launch takes tiles of 256 rows where they come to at least as many work items as the GPU
has CTA pairs, else of 128, else of 64, so that a layout chosen around 256 rows runs 256-row tiles only if it is large enough.
Bounds as in test_gpu_backward.py."""
import numpy as np
import pytest

from test_gpu_backward import FfnGradient, _check_backward, _same_bits

pytestmark = pytest.mark.gpu

# six experts on three ranks, three of them with a replica; segments around one, two, three and four tiles
X = np.array([[1, 1, 0], [1, 1, 0], [1, 0, 1], [1, 0, 0], [0, 1, 0], [0, 1, 0]], dtype=np.uint8)
LENGTHS = [256, 257, 255, 511, 513, 767, 769, 1000, 1, 0, 0, 0]


def _tile(lengths, blocks, shared=(0, 0)):
    """Rows of a launch's token tiles: `blocks` work items a tile of a routed segment; shared: (rows, blocks) of the shared experts."""
    import torch
    pairs = torch.cuda.get_device_properties(0).multi_processor_count // 2
    if max(*lengths, shared[0]) <= 64:
        return 64
    for tile in (256, 128):
        if sum(-(-n // tile) for n in lengths) * blocks + -(-shared[0] // tile) * shared[1] >= pairs:
            return tile
    return 64


@pytest.mark.parametrize("H,F,S,tiles", [(1024, 1024, 0, (256, 256)), (1024, 896, 1, (256, 256)), (768, 896, 0, (256, 128)),
                                         (768, 768, 0, (128, 128))])
def test_ffn_backward_with_full_tiles(H, F, S, tiles):
    rows = sum(LENGTHS)
    assert tiles == (_tile(LENGTHS, -(-F // 256), (S * rows, -(-S * F // 256))), _tile(LENGTHS, H // 256, (S * rows, H // 256)))
    f = FfnGradient(H + F, LENGTHS, X, 4, H, F, S=S)
    f.d.reserve_training()
    f.backward()
    assert f.d.last_status() == 0
    _check_backward(f)
    first = [t.clone() for t in f.outputs()]
    f.backward()
    assert all(_same_bits(a, b) for a, b in zip(first, f.outputs()))


def test_ffn_backward_with_paced_segment_ends():
    """A contraction of 256 steps (F = 8192), segments with a ragged end behind full tiles."""
    lengths = [2800, 700, 1100, 1]
    assert _tile(lengths, 1024 // 256) == 256
    f = FfnGradient(5, lengths, np.ones((4, 1), dtype=np.uint8), 4, 1024, 8192, scale=0.02)
    f.d.reserve_training()
    f.backward()
    assert f.d.last_status() == 0
    _check_backward(f)
    first = [t.clone() for t in f.outputs()]
    f.backward()
    assert all(_same_bits(a, b) for a, b in zip(first, f.outputs()))
