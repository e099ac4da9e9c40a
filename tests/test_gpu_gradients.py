"""The norm over many gradients and clipping on the GPU, against the formula in 64 bits; clipping, whose every rounding is
fixed, bit for bit."""
import math

import numpy as np
import pytest
import torch

import paper_1802_04434_amd as ss

pytestmark = pytest.mark.gpu
DEV = "cuda"
# The kernel's squares are exact and its fp64 sums off by under 2^-30; rounding the root to fp32 is 2^-24 of it.
NORM = 2.0 ** -24 * (1 + 2.0 ** -20)

LISTS = {"one": [1], "short": [3, 1, 7, 2], "one unit": [2048, 4096, 2047, 2049, 4095, 4097], "empty ones": [0, 5, 0, 0, 9000, 0, 70_001, 0], "all empty": [0, 0, 0],
         "none": [], "many": [(37 * i * i) % 5003 for i in range(400)], "exactly one launch": [100 + i for i in range(176)], "one more": [100 + i for i in range(177)],
         "two launches": [64] * 352, "large": [1_000_003, 12, 3_333_333, 1, 2_500_000], "beyond the blocks": [5_000_011, 8_000_001]}


def gradients(lengths, types, seed=0, offset=0):
    """normal gradients as they come from an allocator, or (offset) as parts of one buffer at any element"""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed + sum(lengths))
    out = []
    for i, n in enumerate(lengths):
        dtype = {"f32": torch.float32, "bf16": torch.bfloat16}[types if types != "mixed" else ("f32" if i % 3 else "bf16")]
        at = (offset + i * 3) % 9 if offset else 0
        buffer = torch.full((n + at + 9,), 1e30, dtype=dtype, device=DEV)
        buffer[at:at + n] = torch.randn(n, device=DEV, generator=gen).to(dtype) * (0.01 + i % 5)
        out.append(buffer[at:at + n])
    return out


def exact_norm(g):
    return math.sqrt(math.fsum(float(t.double().square().sum()) for t in g))


def clipped(g, norm, max_norm, dtype):
    """the formula in fp32 with numpy's roundings"""
    with np.errstate(all="ignore"):
        c = np.float32(max_norm) / (np.float32(norm) + np.float32(1e-6))
        c = np.float32(1.0) if c >= 1 else c
        return torch.from_numpy(np.asarray(c * g.float().cpu().numpy(), np.float32).reshape(-1)).to(dtype)


def same(a, b):
    return torch.equal(torch.nan_to_num(a.float(), nan=123.0), torch.nan_to_num(b.float(), nan=123.0)) and torch.equal(torch.isnan(a), torch.isnan(b))


@pytest.mark.parametrize("types", ["f32", "bf16", "mixed"])
@pytest.mark.parametrize("name", sorted(LISTS))
def test_norm(name, types):
    ws, norm = ss.new_grad_norm_workspace(), torch.full((1,), 9.0, device=DEV)
    for offset in (0, 1, 5):
        g = gradients(LISTS[name], types, offset=offset)
        want = exact_norm(g)
        got = [float(ss.grad_norm(g, norm, ws)) for _ in range(3)]
        assert abs(got[0] - want) <= NORM * want, (got[0], want)
        assert got[0] == got[1] == got[2]
    assert not ws[:1].any()


@pytest.mark.parametrize("types,out_type", [("f32", "f32"), ("bf16", "f32"), ("mixed", "f32"), ("mixed", "bf16"), ("f32", "bf16"), ("bf16", "bf16")])
@pytest.mark.parametrize("name", sorted(LISTS))
def test_clip_into_one_vector(name, types, out_type):
    dtype = torch.float32 if out_type == "f32" else torch.bfloat16
    ws, norm = ss.new_grad_norm_workspace(), torch.empty(1, device=DEV)
    lengths = LISTS[name]
    for offset in (0, 1):
        g = gradients(lengths, types, offset=offset)
        before = [t.clone() for t in g]
        ss.grad_norm(g, norm, ws)
        for max_norm in (0.25 * float(norm), 2 * float(norm) + 1.0, 0.0):
            buffer = torch.full((sum(lengths) + 16,), 77.0, dtype=dtype, device=DEV)
            flat = buffer[offset:offset + sum(lengths)]
            ss.grad_clip(g, norm, max_norm, list(flat.split(lengths)) if lengths else [])
            want = [clipped(t, float(norm), max_norm, dtype) for t in g]
            assert same(flat.cpu(), torch.cat(want) if want else torch.empty(0, dtype=dtype))
            assert bool((buffer[:offset] == 77.0).all()) and bool((buffer[offset + sum(lengths):] == 77.0).all())
        assert all(torch.equal(a, b) for a, b in zip(before, g))


@pytest.mark.parametrize("types", ["f32", "bf16", "mixed"])
@pytest.mark.parametrize("name", sorted(LISTS))
def test_clip_in_place(name, types):
    ws, norm = ss.new_grad_norm_workspace(), torch.empty(1, device=DEV)
    for offset in (0, 2):
        g = gradients(LISTS[name], types, offset=offset)
        ss.grad_norm(g, norm, ws)
        for max_norm in (4 * float(norm) + 1.0, 0.5 * float(norm)):      # nothing to do first
            want = [clipped(t, float(norm), max_norm, t.dtype) for t in g]
            ss.grad_clip(g, norm, max_norm)
            assert all(same(t.cpu(), w) for t, w in zip(g, want))


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_what_is_not_finite_follows_the_formula(bad):
    ws, norm = ss.new_grad_norm_workspace(), torch.empty(1, device=DEV)
    g = gradients([5000, 3, 70_000], "mixed")
    g[2][69_999] = bad
    ss.grad_norm(g, norm, ws)
    assert math.isnan(float(norm)) if math.isnan(bad) else float(norm) == math.inf
    want = [clipped(t, float(norm), 1.0, t.dtype) for t in g]
    out = [torch.empty_like(t) for t in g]
    ss.grad_clip(g, norm, 1.0, out)
    assert all(same(t.cpu(), w) for t, w in zip(out, want))
    ss.grad_clip(g, norm, 1.0)
    assert all(same(t.cpu(), w) for t, w in zip(g, want))
    # the workspace is ready again
    assert float(ss.grad_norm([torch.full((4,), 2.0, device=DEV)], norm, ws)) == 4.0


def test_ends_of_the_range():
    ws, norm = ss.new_grad_norm_workspace(), torch.empty(1, device=DEV)
    # squares beyond and below fp32
    for value in (1e30, 3e-30, 2.0 ** -149):
        g = [torch.full((9,), value, device=DEV)]
        assert abs(float(ss.grad_norm(g, norm, ws)) - 3 * float(np.float32(value))) <= 3 * value * 2.0 ** -23
    # a norm beyond fp32 is infinite
    assert float(ss.grad_norm([torch.full((100,), 3e38, device=DEV)], norm, ws)) == math.inf
    # a norm of zero clips by 1
    g = [torch.zeros(50, device=DEV)]
    ss.grad_norm(g, norm, ws)
    assert float(norm) == 0.0 and not ss.grad_clip(g, norm, 1.0)[0].any()


def test_memory_orders():
    ws, norm = ss.new_grad_norm_workspace(), torch.empty(1, device=DEV)
    w = torch.randn(8, 16, 3, 3, device=DEV).to(memory_format=torch.channels_last)
    t = torch.randn(40, 30, device=DEV).t()
    want = exact_norm([w, t])
    assert abs(float(ss.grad_norm([w, t], norm, ws)) - want) <= NORM * want
    expect = [clipped(v.contiguous(), float(norm), 1.0, v.dtype).view(v.shape) for v in (w, t)]
    out = [torch.empty_like(w), torch.empty_like(t)]
    ss.grad_clip([w, t], norm, 1.0, out)
    assert all(same(o.cpu(), e) for o, e in zip(out, expect))
    ss.grad_clip([w, t], norm, 1.0)
    assert all(same(o.cpu(), e) for o, e in zip((w, t), expect))
    with pytest.raises(TypeError, match=r"out\[0\] must have g's memory order"):
        ss.grad_clip([w], norm, 1.0, [torch.empty(w.numel(), device=DEV)])
    with pytest.raises(TypeError, match=r"g\[0\] must be dense"):
        ss.grad_norm([torch.randn(8, 8, device=DEV)[:, ::2]], norm, ws)
    # rows of a stacked tensor, which exist for the call alone
    stack = torch.randn(6, 1000, device=DEV)
    assert abs(float(ss.grad_norm(stack, norm, ws)) - exact_norm([stack])) <= NORM * exact_norm([stack])
    assert abs(float(ss.grad_norm((v for v in (w, t)), norm, ws)) - exact_norm([w, t])) <= NORM * exact_norm([w, t])


def test_tensors_that_are_only_read_may_coincide():
    ws, norm = ss.new_grad_norm_workspace(), torch.empty(1, device=DEV)
    g = torch.randn(1000, device=DEV)
    want = exact_norm([g, g, g[10:]])
    assert abs(float(ss.grad_norm([g, g, g[10:]], norm, ws)) - want) <= NORM * want
    out = torch.empty(2000, device=DEV)
    ss.grad_clip([g, g], norm, 1.0, [out[:1000], out[1000:]])
    assert torch.equal(out[:1000], out[1000:])


def test_overlaps_of_what_is_written_are_refused():
    ws, norm = ss.new_grad_norm_workspace(), torch.ones(8, device=DEV)
    g = torch.randn(4000, device=DEV)
    keep = g.clone()
    a, b = g[:2000], g[2000:]
    for grads, out in (([a, a], None), ([a, g[1000:3000]], None), ([a], [g[4:2004]]), ([a, b], [b, a]), ([b, a], [a, torch.empty(2000, device=DEV)])):
        with pytest.raises(ss.SignSGDError, match="SS_ERR_ARG"):
            ss.grad_clip(grads, norm, 1.0, out)
    with pytest.raises(ss.SignSGDError, match="SS_ERR_ARG"):
        ss.grad_clip([norm[4:]], norm, 1.0, [norm[:4]])
    with pytest.raises(ss.SignSGDError, match="SS_ERR_ARG"):
        ss.grad_norm([norm], norm, ws)
    with pytest.raises(ss.SignSGDError, match="SS_ERR_ARG"):
        ss.grad_norm([ws.view(torch.float32)[4:9]], norm, ws)
    assert torch.equal(g, keep)


def test_streams_and_graphs():
    ws, norm = ss.new_grad_norm_workspace(), torch.empty(1, device=DEV)
    lengths = [1000 + 77 * i for i in range(300)]
    g = gradients(lengths, "mixed")
    flat = torch.empty(sum(lengths), device=DEV)
    out = list(flat.split(lengths))

    def calls(stream=None):
        ss.grad_norm(g, norm, ws, stream=stream)
        ss.grad_clip(g, norm, 1.0, out, stream=stream)

    calls()
    torch.cuda.synchronize()
    want, want_flat = norm.clone(), flat.clone()
    side = torch.cuda.Stream()
    flat.zero_()
    torch.cuda.synchronize()
    calls(side)
    side.synchronize()
    assert torch.equal(norm, want) and torch.equal(flat, want_flat)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for k in range(3):
        for t in g:
            t.mul_(1.5)
        flat.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got, got_flat = norm.clone(), flat.clone()
        calls()
        torch.cuda.synchronize()
        assert torch.equal(norm, got) and torch.equal(flat, got_flat)


def test_offsets_beyond_32_bits():
    ws, norm = ss.new_grad_norm_workspace(), torch.empty(1, device=DEV)
    n = (1 << 32) + 12_345                       # elements, and bytes twice over
    g = [torch.zeros(n, dtype=torch.bfloat16, device=DEV), torch.full((3,), 4.0, device=DEV)]
    g[0][-1] = 3.0
    g[0][(1 << 31) + 7] = 12.0
    want = math.sqrt(9 + 144 + 48)
    assert abs(float(ss.grad_norm(g, norm, ws)) - want) <= NORM * want
    flat = torch.full((n + 3,), 7.0, dtype=torch.bfloat16, device=DEV)
    ss.grad_clip(g, norm, 1.0, [flat[:n], flat[n:]])
    assert same(flat[-4:].cpu(), torch.cat([clipped(g[0][-1:], float(norm), 1.0, torch.bfloat16), clipped(g[1], float(norm), 1.0, torch.bfloat16)]))
    assert same(flat[(1 << 31) + 7:(1 << 31) + 8].cpu(), clipped(g[0][(1 << 31) + 7:(1 << 31) + 8], float(norm), 1.0, torch.bfloat16))
    assert int(torch.count_nonzero(flat)) == 5


@pytest.mark.parametrize("nbytes", [(1 << 28) - 64, 1 << 28, (1 << 28) + 64, (1 << 30) - 64, 1 << 30, (1 << 30) + 64])
def test_norm_around_the_sizes_where_its_launch_changes(nbytes):
    ws, norm = ss.new_grad_norm_workspace(), torch.empty(1, device=DEV)
    for dtype, parts in ((torch.bfloat16, 1), (torch.float32, 3), (torch.bfloat16, 300)):
        n = nbytes // (2 if dtype == torch.bfloat16 else 4)
        flat = torch.randn(n, device=DEV).to(dtype)
        g = list(flat.split([n - 1001 * (parts - 1)] + [1001] * (parts - 1)))
        want = math.sqrt(sum(float(t.double().square().sum()) for t in flat.split(1 << 26)))
        assert abs(float(ss.grad_norm(g, norm, ws)) - want) <= NORM * want
