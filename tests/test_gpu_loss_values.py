"""Values of the loss and its gradient that bounds over whole matrices would hide, on the GPU, on operands whose products add up exactly."""
import pytest
import torch

import loss_plain as plain
import paper_1802_04434_amd as ss
from test_gpu_loss import DEV, NAN, both, case, check, scratch_for, sliced

pytestmark = pytest.mark.gpu


def confident(T, V, base):
    """h, w, target and z with z[t, target[t]] = base^2, the largest of its row by 8 to 16: whole sixteenths, which bf16 and every fp32 sum hold"""
    kinds = 7
    gen = torch.Generator().manual_seed(T * 31 + V)
    gap = torch.randint(128, 257, (kinds, V), generator=gen).float() / 16
    likely = torch.randint(0, V, (kinds,), generator=gen)
    gap[torch.arange(kinds), likely] = 0
    kind = torch.arange(T) % kinds
    h, w = torch.zeros(T, 1 + kinds), torch.zeros(V, 1 + kinds)
    h[:, 0], w[:, 0], w[:, 1:] = base, base, -gap.t()
    h[torch.arange(T), 1 + kind] = 1
    h, w = h.bfloat16(), w.bfloat16()
    z = h.double() @ w.double().t()
    assert torch.equal(z, (base * base - gap.double())[kind])
    return h, w, likely[kind], z


@pytest.mark.parametrize("base", [32.0, 128.0])
@pytest.mark.parametrize("T,V", [(1, 300), (40, 300), (7, 9000), (1100, 1000)])
def test_a_confident_rows_loss_does_not_go_by_the_size_of_its_logits(T, V, base):
    """z is exact, so that top - z[target] is 0 and the loss is log(sum of exp(z - top)), a sum of 1 and what is small.  A term e^-g is off by the rounding of g log2(e), g <= 16,
    by half a step of each of log2(e) and the product, and by two steps of the function: (2 x 16 + 4) U32 of itself; an addition by U32 of a sum below 1 + tail, and on the way of any
    term there are at most 128 of a lane, 2 between lanes, 8 + 1 for each group of eight parts, and 8 levels.  The logarithm of x near 1 is off by two steps of itself; lse by its rounding too."""
    h, w, target, z = confident(T, V, base)
    loss, lse = torch.full((T,), NAN, device=DEV), torch.full((T,), NAN, device=DEV)
    ss.cross_entropy(h.to(DEV), w.to(DEV), target.to(DEV), loss, lse, scratch_for(T, V, h.shape[1]))
    tail = (z - base * base).exp().sum(1) - 1
    want = torch.log1p(tail)
    groups = -(-V // 32 // 8) + 1           # parts of 32 columns at the least
    off = plain.U32 * (36 * tail + (1 + tail) * (128 + 2 + 9 * groups + 8) + 4 * want)
    assert (off < 0.4 * base * base * 2 ** -24).all() or base < 100        # a step of lse would show
    assert ((loss.cpu().double() - want).abs() <= off).all(), float(((loss.cpu().double() - want).abs() / off).max())
    assert ((lse.cpu().double() - (base * base + want)).abs() <= off + plain.U32 * (base * base + want)).all()


# several pieces of the vocabulary: of D, of copied weights, one that divides and one that does not; few rows, and many with a narrow head
@pytest.mark.parametrize("T,V,K,pad", [(4096, 40_000, 64, 0), (4096, 40_000, 72, 3), (40, 30_003, 4096, 0), (40, 30_003, 4096, 1), (1, 20_000, 8200, 1), (2000, 70_001, 136, 8)])
def test_pieces_stay_in_their_scratch(T, V, K, pad):
    gen = torch.Generator(device=DEV).manual_seed(T + V + K + pad)
    h = sliced(torch.randn(T, K, generator=gen, device=DEV).bfloat16(), pad, pad % 2)
    w = sliced((torch.randn(V, K, generator=gen, device=DEV) * 2 / K ** 0.5).bfloat16(), pad, pad % 2)
    target = torch.randint(0, V, (T,), generator=gen, device=DEV)
    target[T // 2] = -1 if T > 1 else V - 1
    dloss = torch.randn(T, generator=gen, device=DEV)
    wanted = ss.new_cross_entropy_scratch(T, V, K).numel()
    memory = torch.full((wanted + (1 << 20),), 0xA5, dtype=torch.uint8, device=DEV)
    got = both(h, w, target, dloss, memory[:wanted])
    assert (memory[wanted:] == 0xA5).all()
    check(got, plain.softmax_loss(h, w, target, dloss), (target >= 0).cpu())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_gradients_into_rows_far_apart(dtype):
    """of every sequence's last token, and of a head whose rows lie in a larger buffer: beyond 2^21 elements, in all beyond 4 GiB"""
    T, V, K, length, width = 19, 300, 200, 1024, 4096
    h, w, target, dloss = (x.to(DEV) for x in case(T, V, K))
    scratch = scratch_for(T, V, K)
    want = both(h, w, target, dloss, scratch, dtype, dtype)
    hidden = torch.full((T, length, width), NAN, dtype=dtype, device=DEV)
    dh = hidden[:, -1, 4:4 + K]
    rows = torch.full((V * ((1 << 23) + 5),), NAN, dtype=dtype, device=DEV)
    dw = rows.as_strided((V, K), ((1 << 23) + 5, 1))
    assert dh.stride(0) == 1 << 22 and dw.stride(0) * V * dw.element_size() > 1 << 32
    ss.cross_entropy_grad(h, w, target, want["lse"], dloss, dh, dw, scratch)
    assert torch.equal(dh, want["dh"]) and torch.equal(dw, want["dw"])
    assert torch.isnan(hidden[:, :-1]).all() and torch.isnan(hidden[:, -1, :4]).all() and torch.isnan(hidden[:, -1, 4 + K:]).all()
    for at in (0, 1, V - 1):        # around a row nothing is written
        assert torch.isnan(rows[at * dw.stride(0) + K:(at + 1) * dw.stride(0)]).all()


def test_rows_too_far_apart_to_be_read_are_refused_by_name():
    T, V, K = 3, 20, 64
    h, w, target, dloss = (x.to(DEV) for x in case(T, V, K))
    loss, lse, scratch = torch.empty(T, device=DEV), torch.empty(T, device=DEV), scratch_for(T, V, K)
    buffer = torch.zeros(V * ((1 << 21) + 1), dtype=torch.bfloat16, device=DEV)
    apart = lambda x, n: buffer.as_strided(x.shape, (n, 1)).copy_(x)  # noqa: E731
    for name, tensors in (("h", (apart(h, (1 << 21) + 1), w)), ("w", (h, apart(w, (1 << 21) + 1)))):
        for call in (lambda: ss.cross_entropy(*tensors, target, loss, lse, scratch), lambda: ss.cross_entropy_grad(*tensors, target, lse, dloss, torch.empty_like(h), torch.empty_like(w), scratch)):
            with pytest.raises(TypeError, match="%s must have its rows 2097152 elements apart at most, got 2097153" % name):
                call()
    # at the limit, in place and copied
    want = both(h, w, target, dloss, scratch)
    for offset in (0, 1):
        at = buffer[offset:].as_strided(w.shape, (1 << 21, 1), offset).copy_(w)
        got = both(h, at, target, dloss, scratch)
        assert all(torch.equal(got[name], want[name]) for name in want)


# few rows against many tokens, and many rows, whose D comes in two pieces of the vocabulary
LIKELY = [(1, 70_001, 64), (2, 30_003, 200), (2000, 70_001, 136), (70, 9001, 520)]


def likely_tokens(T, V, K):
    """h, w, target, dloss, and the tokens that have all of the probability but a hundredth, each about as much as the others: the last nine, and some on both sides of tiles and pieces"""
    gen = torch.Generator().manual_seed(T + V + K)
    pieces = -(-V // ((1 << 27) // (-(-T // 64) * 64) // 256 * 256))
    edge = -(-V // pieces // 256) * 256 if pieces > 1 else 4096
    hot = torch.tensor([0, 63, 64, 255, 256, edge - 1, edge, *range(V - 9, V)])
    h, w = torch.randn(T, K, generator=gen) / (4 * K ** 0.5), torch.randn(V, K, generator=gen)
    h[:, 0], w[:, 0] = 16, 0
    w[hot, 0] = 1                                    # e^16 times as likely: 8.9e6 to 70001 times at most e^(1/2)
    target = torch.randint(1, 60, (T,), generator=gen)
    return h.bfloat16(), w.bfloat16(), target, torch.rand(T, generator=gen) + 0.5, hot


@pytest.mark.parametrize("T,V,K", LIKELY)
def test_no_likely_token_is_left_out_of_a_gradient(T, V, K):
    h, w, target, dloss, _ = (x.to(DEV) for x in likely_tokens(T, V, K))
    for pad in (0, 1):
        got = both(sliced(h, pad, pad), sliced(w, pad, pad), target, dloss, scratch_for(T, V, K), torch.float32, torch.float32)
        check(got, plain.softmax_loss(h, w, target, dloss))


def test_logits_of_minus_infinity():
    """beside finite ones: probability zero, and an infinite loss where it is the target's; nothing else in a row: lse is -infinity, the loss no number, and 0 where there is no target"""
    T, V, K = 66, 200, 64
    h, w, target, _ = case(T, V, K, masked=0)
    h[:, 0], w[:, 0] = 1, float("-inf")
    h[3, 1:] = 0
    target[3], target[5], target[7] = 4, -1, 150
    loss, lse = torch.empty(T, device=DEV), torch.empty(T, device=DEV)
    ss.cross_entropy(h.to(DEV), w.to(DEV), target.to(DEV), loss, lse, scratch_for(T, V, K))
    there = (target >= 0).to(DEV)
    assert (lse == float("-inf")).all() and torch.isnan(loss[there]).all() and loss[5] == 0
    w[4, 0] = 2                                            # all but one token
    ss.cross_entropy(h.to(DEV), w.to(DEV), target.to(DEV), loss, lse, scratch_for(T, V, K))
    hit = (target == 4).to(DEV)
    assert torch.isfinite(lse).all() and lse[3] == 2 and (loss[hit] == 0).all() and loss[5] == 0 and (loss[there & ~hit] == float("inf")).all()
