"""The norm where its lists fill a launch: a full table of tensors, a last launch with one tensor that is added to the slots of the launches
before it, and the tickets of every level back at zero."""
import math

import pytest
import torch

import paper_1802_04434_amd as ss

pytestmark = pytest.mark.gpu
DEV = "cuda"
PER = 256                       # tensors of a launch
# The kernel's squares are exact and its fp64 sums off by under 2^-30; rounding the root to fp32 is 2^-24 of it.
NORM = 2.0 ** -24 * (1 + 2.0 ** -20)
TICKETS = 17 * 8                # lines of 64 bytes, as 64-bit words: one for all, sixteen for groups of blocks


def lists():
    big = 1_000_003             # many units: as many blocks as there are
    yield "full table", [7 + i for i in range(PER)]
    yield "full table, blocks as well", [20_001 + i for i in range(PER)]
    yield "one element in a launch of its own", [100 + i for i in range(PER)] + [1]
    yield "one element after blocks as many as there are", [30_000 + i for i in range(PER)] + [1]
    yield "one element, then blocks as many as there are", [1] * PER + [big] * 3
    yield "two full tables", [50 + i % 9000 for i in range(2 * PER)]
    yield "two full tables and one element", [8192] * (2 * PER) + [1]
    yield "empty ones between do not count", [n for i in range(PER + 1) for n in (0, 11 + i)]
    yield "few blocks, then fewer", [1] * PER + [2] * PER + [3]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("name", [n for n, _ in lists()])
def test_norm_of_full_launches(name, dtype):
    lengths = dict(lists())[name]
    gen = torch.Generator(device=DEV)
    gen.manual_seed(len(lengths))
    g = [torch.randn(n, device=DEV, generator=gen).to(dtype) for n in lengths]
    ws, norm = ss.new_grad_norm_workspace(), torch.full((1,), 9.0, device=DEV)
    ws[TICKETS:] = -1           # slots hold anything before: NaN
    want = math.sqrt(math.fsum(float(t.double().square().sum()) for t in g))
    got = []
    for _ in range(3):
        got.append(float(ss.grad_norm(g, norm, ws)))
        assert not ws[:TICKETS].any()
    assert abs(got[0] - want) <= NORM * want, (got[0], want)
    assert got[0] == got[1] == got[2]


@pytest.mark.parametrize("at", [0, PER - 1, PER, 2 * PER])
def test_each_launch_counts(at):
    """a tensor that is all of the norm, in the first launch, at its end, in the second and in the last"""
    g = [torch.zeros(1 + i % 5000, device=DEV) for i in range(2 * PER + 1)]
    g[at][-1] = 3.0
    ws, norm = ss.new_grad_norm_workspace(), torch.empty(1, device=DEV)
    assert float(ss.grad_norm(g, norm, ws)) == 3.0
    g[at][-1] = math.nan
    assert math.isnan(float(ss.grad_norm(g, norm, ws)))
    g[at][-1] = 0.0             # nothing of it is left in the workspace
    assert float(ss.grad_norm(g, norm, ws)) == 0.0
    assert not ws[:TICKETS].any()
