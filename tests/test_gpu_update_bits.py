"""Orthogonalised updates on the GPU against the same steps with the same roundings in 64 bits (update_rounded): results of 22 bits where they are held and
multiplied so, and each entry for itself, at the ends of rows, slices and tiles too."""
import pytest
import torch

import paper_1802_04434_amd as ss
import update_rounded as rounded
from test_gpu_orthogonal import DEV, NAN, matrix, scratch_for

pytestmark = pytest.mark.gpu

# matrices taken whole, in slices (of 128 and of 64) and in tiles; rows and columns, whether in tiles, steps: in tiles also as many as multiply 22 bits throughout
CASES = ([(r, c, False, 5) for r, c in ((1, 7), (3, 5), (9, 1), (40, 40), (63, 65), (33, 90), (128, 129), (100, 300), (20, 4001), (2001, 90), (1501, 121), (50, 5003))]
         + [(r, c, True, s) for r, c, s in ((131, 205, 3), (257, 150, 3), (201, 259, 2), (301, 699, 2), (603, 521, 1), (521, 2003, 1), (2003, 521, 1))]
         + [(r, c, True, 5) for r, c in ((131, 205), (257, 150), (301, 699), (699, 301))])
# of which the bound is too wide to tell 22 bits from 11, but not an entry that is missing
WIDE = [(603, 521, True, 5), (521, 2003, True, 5), (1031, 1101, True, 5), (2050, 1030, True, 5), (1031, 1101, True, 1)]


def compare(got, g, tiles, steps):
    sums = rounded.Sums()
    want = rounded.update(g, steps, got.dtype == torch.float32, tiles, sums)
    spread, half = rounded.update_spread(g, want, got.dtype, steps, tiles), rounded.HALF[got.dtype]
    off = (got.double() - want).abs()
    assert float(off.norm()) <= spread + half * float(want.norm()), (float(off.norm()), spread)
    # an entry is off by a sum of many roundings, in rows whose norms differ by less than 2.7, 8 of the bound's three deviations, and by a few that are far larger than the others, which the bound over
    # all entries does not feel; where there are few entries it is off by no more than all of them
    entry = half * want.abs() + (spread if g.numel() < 256 else 8 * spread / g.numel() ** 0.5) + rounded.flipped(sums.largest)
    assert (off <= entry).all(), float((off / entry).max())


@pytest.mark.parametrize("rows,cols,tiles,steps", CASES + WIDE)
def test_updates_to_the_last_bits(rows, cols, tiles, steps):
    """a stack of three, as slices of wider rows, in either type of result; and the whole step, which with beta 0 from parameters of zero by -1 gives the update itself, to the bit"""
    xs = torch.stack([matrix(rows, cols, seed) for seed in range(3)]).to(DEV)
    g = torch.full((3, rows + 1, cols + 3), NAN, device=DEV)[:, :rows, :cols].copy_(xs)
    scratch, results = scratch_for(rows, cols, 3), {}
    for dtype in (torch.float32, torch.bfloat16):
        out = torch.full((3, rows, cols), NAN, dtype=dtype, device=DEV)
        ss.orthogonalize(g, out, scratch, steps=steps)
        results[dtype] = out
        for i in range(3):
            compare(out[i], xs[i], tiles, steps)
    m, x = torch.full_like(xs, 3.0), torch.zeros_like(xs)
    ss.orthogonal_step(g, m, 0.0, -1.0, x, scratch.fill_(0xFF), steps=steps)
    assert torch.equal(m, xs) and torch.equal(x, results[torch.float32])
