"""What the comparisons of test_gpu_update_bits would notice, without a GPU: mistakes planted in the 64-bit model of the kernels (update_rounded), a missing second half
of an operand, a missing last entry, are further off than its bounds allow; and the model agrees with the definition as far as its bits go."""
import pytest
import torch

import loss_plain as plain
import test_gpu_update_bits as gpu
import update_rounded as rounded
from test_gpu_orthogonal import matrix

MISTAKES = ["x_lo", "ab_lo", "a_lo_b", "twofold"]
# the largest cost minutes here, and are no different
SIZES = [c for c in gpu.CASES + gpu.WIDE if c[0] * c[1] * min(c[:2]) < 4e8]


@pytest.mark.parametrize("rows,cols,tiles,steps", [c for c in SIZES if c in gpu.CASES])
def test_lost_halves_show(rows, cols, tiles, steps):
    g = matrix(rows, cols, 0)
    assert steps == 5 or rounded.twofold_steps(-(-min(rows, cols) // 64) * 64, True) == steps
    want = rounded.update(g, steps, True, tiles)
    allowed = rounded.update_spread(g, want, torch.float32, steps, tiles) + plain.U32 * float(want.norm())
    for mistake in MISTAKES:
        off = float((rounded.update(g, steps, True, tiles, lost=mistake) - want).norm())
        assert off > 2 * allowed, (mistake, off / allowed)


@pytest.mark.parametrize("rows,cols,tiles,steps", SIZES)
def test_a_lost_eight_shows(rows, cols, tiles, steps):
    """the last entries of the last row, left at zero or at what another row has: those of the row before it, or of the same row's eights"""
    g = matrix(rows, cols, 0)
    for result in (torch.float32, torch.bfloat16):
        want = rounded.update(g, steps, result == torch.float32, tiles)
        for stale in (torch.zeros(cols, dtype=torch.float64), want[rows // 2 - 1] if rows > 1 else -want[0]):
            got = want.to(result)
            last = (cols - 1) // 8 * 8
            got[-1, last:] = stale[last:]
            with pytest.raises(AssertionError):
                gpu.compare(got, g, tiles, steps)
        gpu.compare(want.to(result), g, tiles, steps)


@pytest.mark.parametrize("rows,cols", [(64, 64), (100, 300), (20, 4001)])
def test_the_model_has_22_bits(rows, cols):
    """every operand of 22 bits is off by 2^-23 of itself at most, 2^11 times less than one of 11"""
    g = matrix(rows, cols, 0)
    want = plain.orthogonalized(g)
    assert float((rounded.update(g, tiles=False) - want).norm()) <= plain.orthogonal_bound(g) / 2 ** 10
    assert float((rounded.update(g, fp32=False, tiles=True) - want).norm()) <= plain.orthogonal_bound(g)
