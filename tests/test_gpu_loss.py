"""The loss over a vocabulary and its gradient on the GPU against their definition in 64 bits, within the bounds of their
roundings (loss_plain), at the sizes, masks and layouts where they can go wrong."""
import pytest
import torch

import loss_plain as plain
import paper_1802_04434_amd as ss

pytestmark = pytest.mark.gpu
DEV = "cuda"
NAN = float("nan")
# rows, vocabulary, width: one of each to several tiles, both sides of 8, 32, 64, 128 and 256
SIZES = [(1, 1, 1), (1, 2, 64), (1, 1000, 8), (2, 63, 7), (3, 64, 64), (5, 65, 63), (31, 255, 65), (33, 257, 128), (63, 127, 96), (64, 128, 64),
         (65, 129, 72), (100, 33, 200), (127, 513, 130), (128, 1000, 256), (129, 2049, 40), (257, 300, 520), (300, 700, 192), (513, 96, 320)]

# every tile size, several pieces of the vocabulary (also of copied weights), sums in parts; compared with 64 bits on the GPU
LARGE = [(1, 70_001, 64), (2, 30_000, 200), (40, 257, 8192), (1500, 4100, 256), (2600, 5000, 320), (5000, 9000, 1000), (33_000, 9000, 72), (3, 5000, 60_001)]


def sliced(x, pad, offset):
    """x as a slice of a buffer of NaN: rows `pad` further apart than they are long, the first `offset` elements in"""
    rows, cols = x.shape
    buffer = torch.full((offset + rows * (cols + pad),), NAN, dtype=x.dtype, device=DEV)
    view = buffer[offset:].view(rows, cols + pad)[:, :cols]
    view.copy_(x)
    return view


def case(T, V, K, seed=0, masked=0.25):
    gen = torch.Generator().manual_seed(seed * 7919 + T * 31 + V * 7 + K)
    h = torch.randn(T, K, generator=gen).bfloat16()
    w = (torch.randn(V, K, generator=gen) * 2 / K ** 0.5).bfloat16()
    target = torch.randint(0, V, (T,), generator=gen)
    target[torch.rand(T, generator=gen) < masked] = -1
    dloss = torch.randn(T, generator=gen)
    return h, w, target, dloss


def scratch_for(T, V, K):
    s = ss.new_cross_entropy_scratch(T, V, K)
    return s.fill_(0xFF)            # NaN, whatever it is read as


def both(h, w, target, dloss, scratch, dh_type=torch.bfloat16, dw_type=torch.bfloat16, pad=0, offset=0, stream=None):
    T, K = h.shape
    loss, lse = torch.full((T,), NAN, device=DEV), torch.full((T,), NAN, device=DEV)
    dh, dw = sliced(torch.zeros(T, K, dtype=dh_type), pad, offset), sliced(torch.zeros(w.shape, dtype=dw_type), pad, offset)
    ss.cross_entropy(h, w, target, loss, lse, scratch, stream=stream)
    ss.cross_entropy_grad(h, w, target, lse, dloss, dh, dw, scratch, stream=stream)
    return {"loss": loss, "lse": lse, "dh": dh, "dw": dw}


def check(got, want, rows=None):
    for name, (value, bound) in want.items():
        g, value, bound = got[name].cpu(), value.cpu(), bound.cpu()
        half = {torch.float32: plain.U32, torch.bfloat16: plain.U16}[g.dtype]
        bound = bound + 2 * half * value.abs() + 1e-30
        off = (g.double() - value).abs()
        if name in ("loss", "lse") and rows is not None:
            off, bound = off[rows], bound[rows]
        assert torch.isfinite(off).all() and (off <= bound).all(), "%s off by %.3g of its bound" % (name, float((off / bound).max()))


@pytest.mark.parametrize("T,V,K", SIZES)
def test_loss_and_gradients(T, V, K):
    h, w, target, dloss = case(T, V, K)
    want = plain.softmax_loss(h, w, target, dloss)
    there = target >= 0
    # rows at any multiple of 2, of 16 and of 4 bytes
    for pad, offset in ((0, 0), (3, 1), (8, 8), (2 - K % 2, 2)):
        got = both(sliced(h, pad, offset), sliced(w, pad, offset), target.to(DEV), dloss.to(DEV), scratch_for(T, V, K), pad=pad, offset=offset)
        check(got, want, there)
        assert (got["loss"][~there.to(DEV)] == 0).all() and (got["dh"][~there.to(DEV)] == 0).all()
        for name in ("dh", "dw"):       # between the rows nothing is written
            t = got[name]
            around = t.as_strided((t.shape[0] - 1, pad), (t.stride(0), 1), t.storage_offset() + t.shape[1]) if pad and t.shape[0] > 1 else None
            assert around is None or torch.isnan(around).all(), name


@pytest.mark.parametrize("T,V,K", LARGE)
def test_large_sizes(T, V, K):
    gen = torch.Generator(device=DEV).manual_seed(T + V + K)
    h = torch.randn(T, K, generator=gen, device=DEV).bfloat16()
    w = (torch.randn(V, K, generator=gen, device=DEV) * 2 / K ** 0.5).bfloat16()
    target = torch.randint(0, V, (T,), generator=gen, device=DEV)
    target[torch.rand(T, generator=gen, device=DEV) < 0.2] = -1
    target[0] = V - 1
    dloss = torch.randn(T, generator=gen, device=DEV)
    got = both(h, w, target, dloss, scratch_for(T, V, K))
    check(got, plain.softmax_loss(h, w, target, dloss), (target >= 0).cpu())


@pytest.mark.parametrize("K", [1152, 1151])
def test_weights_beyond_4_gib(K):
    """and the gradients' rows at their end, which tiles find at offsets of more than 32 bits; read in place, and copied"""
    T, V = 3, 1_900_003
    gen = torch.Generator(device=DEV).manual_seed(K)
    w = torch.empty(V, K, dtype=torch.bfloat16, device=DEV).normal_(0, K ** -0.5, generator=gen)
    h = torch.randn(T, K, generator=gen, device=DEV).bfloat16()
    target, dloss = torch.tensor([V - 1, -1, 7], device=DEV), torch.tensor([1.0, 5.0, -0.5], device=DEV)
    assert w.numel() * 2 > 1 << 32
    dw = torch.full_like(w, NAN)
    loss, lse, dh, scratch = torch.empty(T, device=DEV), torch.empty(T, device=DEV), torch.empty_like(h), scratch_for(T, V, K)
    ss.cross_entropy(h, w, target, loss, lse, scratch)
    ss.cross_entropy_grad(h, w, target, lse, dloss, dh, dw, scratch)
    # in bands, by the same formulas
    h64 = h.double()
    z = torch.cat([band.double() @ h64.t() for band in w.split(1 << 17)]).t()
    want = torch.logsumexp(z, 1)
    ez = 2 * plain.U32 * K * float(h64.abs().amax() * w.abs().amax()) * K
    assert ((lse.double() - want).abs() <= ez + 2 * plain.U32 * (V / 32 + 100)).all()
    assert ((loss.double() - (want - z.gather(1, target.clamp(min=0)[:, None])[:, 0])).abs() <= 2 * ez + 2 * plain.U32 * (V / 32 + 200))[[0, 2]].all() and loss[1] == 0
    d = (z - want[:, None]).exp()
    d[[0, 2], target[[0, 2]]] -= 1
    d *= torch.where(target >= 0, dloss, 0.0).double()[:, None]
    size = 2 * plain.U16 + 2 * ez + 2 * plain.U32 * (V / 32 + 300)      # D's rounding, the result's, and what z and lse are off by, relative to the terms
    for at in (0, V // 2, V - 1000):
        part = d[:, at:at + 1000]
        off = (dw[at:at + 1000].double() - part.t() @ h64).abs()
        assert (off <= size * (part.abs().t() @ h64.abs()) + 1e-30).all(), at
    assert torch.isfinite(dw.amax()) and torch.isfinite(dw.amin())
    terms = sum(part.abs() @ band.double().abs() for part, band in zip(d.split(1 << 17, 1), w.split(1 << 17)))
    value = sum(part @ band.double() for part, band in zip(d.split(1 << 17, 1), w.split(1 << 17)))
    assert ((dh.double() - value).abs() <= size * terms + 1e-30).all() and (dh[1] == 0).all()


@pytest.mark.parametrize("dh_type", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("dw_type", [torch.float32, torch.bfloat16])
def test_types_of_gradients(dh_type, dw_type):
    h, w, target, dloss = case(70, 300, 136)
    got = both(h.to(DEV), w.to(DEV), target.to(DEV), dloss.to(DEV), scratch_for(70, 300, 136), dh_type, dw_type)
    check(got, plain.softmax_loss(h, w, target, dloss), target >= 0)


def test_either_gradient_alone_and_rows_of_weight_one():
    h, w, target, _ = case(90, 500, 128)
    want = plain.softmax_loss(h, w, target)
    hd, wd, td, scratch = h.to(DEV), w.to(DEV), target.to(DEV), scratch_for(90, 500, 128)
    full = both(hd, wd, td, None, scratch)
    check(full, want, target >= 0)
    dh, dw = torch.full_like(hd, NAN), torch.full_like(wd, NAN)
    ss.cross_entropy_grad(hd, wd, td, full["lse"], None, dh, None, scratch)
    ss.cross_entropy_grad(hd, wd, td, full["lse"], None, None, dw, scratch)
    assert torch.equal(dh, full["dh"]) and torch.equal(dw, full["dw"])


def test_gradient_against_differences():
    """of the loss itself, in 64 bits: what the formula of the gradient has to agree with"""
    T, V, K = 9, 70, 24
    h, w, target, dloss = case(T, V, K, seed=3)
    got = both(h.to(DEV), w.to(DEV), target.to(DEV), dloss.to(DEV), scratch_for(T, V, K), torch.float32, torch.float32)

    def total(h64, w64):
        z = h64 @ w64.t()
        each = torch.logsumexp(z, 1) - z.gather(1, target.clamp(min=0)[:, None])[:, 0]
        return float((torch.where(target >= 0, each, 0.0) * dloss.double()).sum())

    bounds = plain.softmax_loss(h, w, target, dloss)
    gen = torch.Generator().manual_seed(5)
    step = 1e-5
    for name, at in (("dh", h), ("dw", w)):
        direction = torch.randn(at.shape, generator=gen).double()
        move = lambda s: total(*[x.double() + s * direction if x is at else x.double() for x in (h, w)])  # noqa: E731
        slope = (move(step) - move(-step)) / (2 * step)
        found = float((got[name].cpu().double() * direction).sum())
        # the kernel's bound, and the differences' own: third derivatives times step^2 and the loss's rounding over the step
        allowed = float((bounds[name][1] * direction.abs()).sum()) + 1e-7
        assert abs(found - slope) <= allowed, (name, found, slope, allowed)


@pytest.mark.parametrize("masked", ["all", "none", "first", "last", "but one"])
def test_rows_without_a_target(masked):
    T, V, K = 67, 200, 80
    h, w, target, dloss = case(T, V, K, masked=0)
    if masked == "all":
        target[:] = -100
    elif masked == "but one":
        target[:40], target[41:] = -1, -2 ** 62
    elif masked != "none":
        target[0 if masked == "first" else -1] = -1
    hd = h.to(DEV)
    for garbage in (NAN, float("inf"), torch.finfo(torch.bfloat16).min):     # a padded batch's rows may hold anything
        hd[(target < 0).to(DEV)] = garbage
        got = both(hd, w.to(DEV), target.to(DEV), dloss.to(DEV), scratch_for(T, V, K))
        check(got, plain.softmax_loss(h, w, target, dloss), target >= 0)
        assert (got["loss"].cpu()[target < 0] == 0).all() and (got["dh"].cpu()[target < 0] == 0).all()


def test_targets_that_are_no_token():
    h, w, target, dloss = case(70, 130, 64, masked=0)
    target[3], target[69] = 130, 2 ** 62
    got = both(h.to(DEV), w.to(DEV), target.to(DEV), dloss.to(DEV), scratch_for(70, 130, 64))
    bad = torch.zeros(70, dtype=torch.bool)
    bad[[3, 69]] = True
    assert torch.equal(torch.isnan(got["loss"]).cpu(), bad) and torch.isfinite(got["lse"]).all()
    assert torch.equal(torch.isnan(got["dh"]).all(1).cpu(), bad) and torch.isnan(got["dw"]).all()


def test_infinities_and_nan():
    T, V, K = 40, 150, 64
    h, w, target, dloss = case(T, V, K, masked=0)
    h[:, 0], w[:, 0] = 1, 0
    w[7, 0] = float("-inf")                                # one token's probability is zero
    target[target == 7] = 8
    lowest = torch.finfo(torch.bfloat16).min
    w[9, 0] = lowest
    target[target == 9] = 8
    h[5, 1] = NAN                                          # one row
    keep = torch.arange(T) != 5
    keep_v = (torch.arange(V) != 7) & (torch.arange(V) != 9)
    loss, lse = torch.empty(T, device=DEV), torch.empty(T, device=DEV)
    ss.cross_entropy(h.to(DEV), w.to(DEV), target.to(DEV), loss, lse, scratch_for(T, V, K))
    renumber = torch.cumsum(keep_v, 0) - 1
    want = plain.softmax_loss(h[keep], w[keep_v], renumber[target[keep]])
    # two columns more change nothing: exp(-inf) and exp of the lowest bf16 are zero
    check({"loss": loss.cpu()[keep], "lse": lse.cpu()[keep]}, {k: want[k] for k in ("loss", "lse")})
    assert torch.isnan(loss[5]) and torch.isnan(lse[5])
    w[3, 0] = float("inf")
    ss.cross_entropy(h.to(DEV), w.to(DEV), target.to(DEV), loss, lse, scratch_for(T, V, K))
    assert torch.isnan(loss).all()


def test_large_logits_do_not_overflow():
    T, V, K = 33, 90, 64
    h, w, target, dloss = case(T, V, K)
    h, w = (h * 60).bfloat16(), (w * 40).bfloat16()
    got = both(h.to(DEV), w.to(DEV), target.to(DEV), dloss.to(DEV), scratch_for(T, V, K))
    check(got, plain.softmax_loss(h, w, target, dloss), target >= 0)


def test_weights_of_rows():
    """from the smallest to large, of either sign and zero"""
    T, V, K = 50, 333, 64
    h, w, target, dloss = case(T, V, K, masked=0)
    for scale in (1e-30, 1e-6, 1.0, 1e6):
        d = dloss * scale
        d[4] = 0
        got = both(h.to(DEV), w.to(DEV), target.to(DEV), d.to(DEV), scratch_for(T, V, K))
        check(got, plain.softmax_loss(h, w, target, d))
    got = both(h.to(DEV), w.to(DEV), target.to(DEV), torch.zeros(T, device=DEV), scratch_for(T, V, K))
    assert (got["dh"] == 0).all() and (got["dw"] == 0).all()


def test_no_rows():
    scratch = ss.new_cross_entropy_scratch(0, 50, 64)
    empty, w = torch.empty(0, 64, dtype=torch.bfloat16, device=DEV), torch.randn(50, 64, device=DEV).bfloat16()
    none, target = torch.empty(0, device=DEV), torch.empty(0, dtype=torch.int64, device=DEV)
    for dtype, pad in ((torch.bfloat16, 0), (torch.float32, 3)):
        dw = sliced(torch.ones(50, 64, dtype=dtype), pad, 0)
        ss.cross_entropy(empty, w, target, none, none, scratch)
        ss.cross_entropy_grad(empty, w, target, none, None, empty, dw, scratch)
        assert (dw == 0).all()


def test_same_bits_on_another_stream_and_in_a_replayed_graph():
    T, V, K = 200, 1500, 192
    h, w, target, dloss = (x.to(DEV) for x in case(T, V, K))
    scratch = scratch_for(T, V, K)
    want = both(h, w, target, dloss, scratch)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = both(h, w, target, dloss, scratch)
    torch.cuda.current_stream().wait_stream(side)
    named = both(h, w, target, dloss, scratch, stream=torch.cuda.current_stream())
    for name in want:
        assert torch.equal(want[name], again[name]) and torch.equal(want[name], named[name]), name
    loss, lse, dh, dw = (torch.full_like(want[k], NAN) for k in ("loss", "lse", "dh", "dw"))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ss.cross_entropy(h, w, target, loss, lse, scratch)
        ss.cross_entropy_grad(h, w, target, lse, dloss, dh, dw, scratch)
    for seed in range(4):
        h2, w2, target2, dloss2 = case(T, V, K, seed=seed)
        h.copy_(h2), w.copy_(w2), target.copy_(target2), dloss.copy_(dloss2)
        eager = both(h, w, target, dloss, scratch.fill_(seed * 85))
        for t in (loss, lse, dh, dw):
            t.fill_(NAN)
        graph.replay()
        torch.cuda.synchronize()
        for name, t in (("loss", loss), ("lse", lse), ("dh", dh), ("dw", dw)):
            assert torch.equal(t, eager[name]), (seed, name)


def test_refusals():
    h, w, target, dloss = (x.to(DEV) for x in case(10, 20, 64))
    loss, lse, scratch = torch.empty(10, device=DEV), torch.empty(10, device=DEV), ss.new_cross_entropy_scratch(10, 20, 64)
    for bad, what in (((h.float(), w), "h must be bfloat16"), ((h, w.float()), "w must be bfloat16"), ((h, w[:, :63]), "w must have h's 64 columns"),
                      ((h.t(), w), "side by side"), ((h[0], w), "two dimensions"), ((h.cpu(), w), "h must live in device memory"), ((h, w.half()), "w has dtype")):
        with pytest.raises(TypeError, match=what):
            ss.cross_entropy(*bad, target, loss, lse, scratch)
    for args, what in (((target[:9], loss, lse, scratch), "target must be contiguous"), ((target.int(), loss, lse, scratch), "target has dtype"),
                       ((target, torch.empty(11, device=DEV), lse, scratch), "loss must have h's 10 rows"), ((target, loss, lse.double(), scratch), "lse has dtype"),
                       ((target, loss, lse, scratch.int()), "scratch has dtype"), ((target, loss, lse, scratch.cpu()), "scratch must live")):
        with pytest.raises(TypeError, match=what):
            ss.cross_entropy(h, w, *args)
    with pytest.raises(ss.SignSGDError, match="ss_cross_entropy returned SS_ERR_ARG"):
        ss.cross_entropy(h, w, target, loss, lse, scratch[:-256])
    with pytest.raises(ss.SignSGDError, match="SS_ERR_ARG"):
        ss.cross_entropy(h, w, target, loss, loss, scratch)
    dh, dw = torch.empty_like(h), torch.empty_like(w)
    with pytest.raises(TypeError, match="dh must be 10 x 64, got 9 x 64"):
        ss.cross_entropy_grad(h, w, target, lse, dloss, dh[:9], dw, scratch)
    with pytest.raises(ss.SignSGDError, match="ss_cross_entropy_grad returned SS_ERR_NULL"):
        ss.cross_entropy_grad(h, w, target, lse, dloss, None, None, scratch)
    with pytest.raises(ss.SignSGDError, match="SS_ERR_ARG"):
        ss.cross_entropy_grad(h, w, target, lse, dloss, h, dw, scratch)
