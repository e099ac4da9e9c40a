"""The exact operands on the CPU: they are what they say, and a mistake planted in the oracle (a block, a group or a step of the sum
lost, doubled or taken from elsewhere) shows in the result, however long the sum."""
import numpy as np
import pytest
import torch

import mx4_exact as exact
import mx4_plain as plain

COLUMNS = [33, 520, 4100, 10_241, 20_000, 32_801, 70_000, 300_000]


@pytest.mark.parametrize("cols", COLUMNS[:6])
def test_operands_are_their_own_quantisation(cols):
    data, scales, values = exact.operand(1, 5, cols)
    want, want_scales = plain.quantize(values.numpy())
    assert np.array_equal(data.numpy(), want) and np.array_equal(scales.numpy(), want_scales)
    assert np.array_equal(plain.values(data.numpy(), scales.numpy(), cols), values.numpy())


@pytest.mark.parametrize("cols", COLUMNS)
def test_planted_mistakes_show(cols):
    x, w = exact.operand(2, 9, cols)[2], exact.operand(3, 7, cols)[2]
    want = exact.product(x, w)
    assert torch.equal(want.float().double(), want)                  # no rounding to be allowed for
    for width in (32, 128, 256, 512):
        for start in {0, cols // width // 2 * width, (cols - 1) // width * width}:
            here = w[:, start:start + width].t()
            part, first = x[:, start:start + width] @ here, x[:, :here.shape[0]] @ here
            assert not torch.equal(want - part, want) and not torch.equal(want + part, want)
            assert start == 0 or not torch.equal(want - part + first, want)
