"""The two ends of a training step over matrices, as measurable cases: the cross entropy over a large
vocabulary with its gradient, and the update that is orthogonalised before it is taken.

A case is one pass through the public calls of `paper_1802_04434_amd` (`own`) or through the plain
form of the same operators in elementary torch operations of 32 bits.  Sizes are generic.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
COEFFICIENTS = (3.4445, -4.7750, 2.0315)
STEPS = 5
BETA = 0.95


def listed():
    return [
        # how likely the one next token is, while answering: latency, and the bandwidth of the head's weights
        {"name": "loss_one_token", "kind": "loss", "tokens": 1, "vocab": 32_000, "width": 2048, "pad": 0, "masked": 0.0},
        # a short text is scored; slices of wider buffers, nothing a multiple of a tile
        {"name": "loss_ragged", "kind": "loss", "tokens": 301, "vocab": 10_007, "width": 520, "pad": 3, "masked": 0.2},
        # evaluation of a long batch under a large vocabulary
        {"name": "loss_long", "kind": "loss", "tokens": 8192, "vocab": 128_000, "width": 4096, "pad": 0, "masked": 0.05},
        # a small model's training pass: loss, then both gradients; a third of the rows is padding
        {"name": "train_small", "kind": "train", "tokens": 64, "vocab": 5003, "width": 256, "pad": 0, "masked": 0.33},
        # an ordinary training pass
        {"name": "train_ordinary", "kind": "train", "tokens": 4096, "vocab": 32_000, "width": 2048, "pad": 0, "masked": 0.05},
        # a long batch under a large vocabulary
        {"name": "train_large", "kind": "train", "tokens": 8192, "vocab": 128_000, "width": 4096, "pad": 0, "masked": 0.05},
        # one small matrix: latency
        {"name": "orthogonalize_tiny", "kind": "orthogonalize", "count": 1, "rows": 64, "cols": 64, "dtype": "f32", "pad": 0},
        # odd sizes, a slice of a wider buffer
        {"name": "orthogonalize_ragged", "kind": "orthogonalize", "count": 1, "rows": 257, "cols": 1000, "dtype": "f32", "pad": 3},
        # the same matrix of many layers at once
        {"name": "orthogonalize_stack", "kind": "orthogonalize", "count": 24, "rows": 512, "cols": 2048, "dtype": "bf16", "pad": 0},
        # the largest square matrix
        {"name": "orthogonalize_large", "kind": "orthogonalize", "count": 1, "rows": 8192, "cols": 8192, "dtype": "bf16", "pad": 0},
        # a tall, small matrix's whole step: momentum, update, parameters
        {"name": "step_tall", "kind": "step", "count": 1, "rows": 1000, "cols": 120, "dtype": "f32", "pad": 0, "ahead": True},
        # an ordinary layer's whole step
        {"name": "step_square", "kind": "step", "count": 1, "rows": 4096, "cols": 4096, "dtype": "bf16", "pad": 0, "ahead": False},
    ]


def _size(rng, lo, hi):
    """spread over the logarithm, every third one a multiple of 64"""
    v = int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))
    v = min(max(v, lo), hi)
    return max(64, v // 64 * 64) if v >= 64 and rng.random() < 0.35 else v


def draw(rng):
    kind = rng.choice(["loss", "train", "train", "orthogonalize", "orthogonalize", "step"])
    if kind in ("loss", "train"):
        return {"kind": kind, "tokens": _size(rng, 1, 8192), "vocab": _size(rng, 500, 128_000), "width": _size(rng, 32, 4096),
                "pad": rng.choice([0, 0, 0, 8, 3]), "masked": rng.choice([0.0, 0.05, 0.3])}
    rows, cols = _size(rng, 16, 8192), _size(rng, 16, 8192)
    low, high = min(rows, cols), max(rows, cols)
    most = min(48, (1 << 39) // (low * low * high), (1 << 27) // (rows * cols))     # no more work than the largest listed case
    return {"kind": kind, "count": _size(rng, 1, most) if most > 1 and rng.random() < 0.5 else 1, "rows": rows, "cols": cols,
            "dtype": rng.choice(["f32", "bf16"]), "pad": rng.choice([0, 0, 0, 8, 3]), **({"ahead": rng.random() < 0.5} if kind == "step" else {})}


def work(case):
    if case["kind"] in ("loss", "train"):
        t, v, k = case["tokens"], case["vocab"], case["width"]
        if case["kind"] == "loss":
            return {"bytes": 2 * k * (t + v) + 16 * t, "flops": 2 * t * v * k}
        # one product for the logits, one for each gradient
        return {"bytes": 4 * k * (t + v) + 20 * t, "flops": 6 * t * v * k}
    n, elements = case["count"], case["count"] * case["rows"] * case["cols"]
    low, high = min(case["rows"], case["cols"]), max(case["rows"], case["cols"])
    element = 2 if case["dtype"] == "bf16" else 4
    # two symmetric products, of which half is enough, and a whole one
    flops = n * STEPS * (3 * low * low * high + low ** 3)
    return {"bytes": elements * (element + (2 if case["kind"] == "orthogonalize" else 16)), "flops": flops}


# ------------------------------------------------------------------ inputs ----

def _generator(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed((seed * 1_000_003 + sum(int(v * 100) * (i + 7) for i, v in enumerate(case.values()) if isinstance(v, (int, float)))) % (1 << 62))
    return gen


def _head(case, gen):
    """last hidden states, whose columns differ in size, and a head whose frequent tokens have larger rows; targets follow the frequencies"""
    t, v, k, pad = case["tokens"], case["vocab"], case["width"], case["pad"]
    h = torch.randn(t, k + pad, device="cuda", generator=gen)
    loud = torch.rand(k + pad, device="cuda", generator=gen) < 0.03
    h.mul_(torch.where(loud, 6.0, 1.0))
    w = torch.randn(v, k + pad, device="cuda", generator=gen)
    w.mul_(1.5 / k ** 0.5)
    often = torch.rand(t, device="cuda", generator=gen).pow_(3)
    target = (often * v).long().clamp_(0, v - 1)
    masked = torch.rand(t, device="cuda", generator=gen) < case["masked"]
    if t > 1:
        masked[0], masked[-1] = False, case["masked"] > 0
    return {"h": h.to(torch.bfloat16)[:, :k], "w": w.to(torch.bfloat16)[:, :k], "target": torch.where(masked, -1, target)}


def _gradient(case, gen, dtype, scale, pad):
    """count x rows x cols, as gradients and momentum are: a few strong directions over much that is weak"""
    n, r, c = case["count"], case["rows"], case["cols"]
    rank = max(1, min(r, c) // 16)
    out = torch.randn(n, r, c + pad, device="cuda", generator=gen).mul_(0.3)
    left = torch.randn(n, r, rank, device="cuda", generator=gen).mul_(rank ** -0.5)
    right = torch.randn(n, rank, c + pad, device="cuda", generator=gen)
    for i in range(n):
        out[i].addmm_(left[i], right[i])
    return out.mul_(scale).to(dtype)[:, :, :c]


def prepare(case, seed):
    gen, kind = _generator(case, seed), case["kind"]
    s = {"case": case}
    if kind in ("loss", "train"):
        s |= _head(case, gen)
        t, v, k = case["tokens"], case["vocab"], case["width"]
        s["loss"], s["lse"] = torch.empty(t, device="cuda"), torch.empty(t, device="cuda")
        if kind == "train":
            # the mean over the rows that have a target
            there = s["target"] >= 0
            s["dloss"] = torch.where(there, 1.0 / there.sum().clamp(min=1), 0.0).float()
            s["dh"], s["dw"] = torch.empty(t, k, dtype=torch.bfloat16, device="cuda"), torch.empty(v, k, dtype=torch.bfloat16, device="cuda")
        return s
    n, r, c = case["count"], case["rows"], case["cols"]
    s["g"] = _gradient(case, gen, DTYPES[case["dtype"]], 1e-3, case["pad"])
    if kind == "orthogonalize":
        s["out"] = torch.empty(n, r, c, dtype=torch.bfloat16, device="cuda")
        return s
    s["m"] = _gradient(case, gen, torch.float32, 7e-4, 0).contiguous()
    s["x"] = torch.randn(n, r, c, device="cuda", generator=gen).mul_(0.03)
    s["delta"] = 3e-4 * 0.2 * max(r, c) ** 0.5      # so that an update's entries are of one size, whatever the matrix's
    return s


# -------------------------------------------------------------------- pass ----

def _plain_logits(s):
    return torch.matmul(s["h"].float(), s["w"].float().t())


def _plain_loss(s, z):
    top = z.amax(1, keepdim=True)
    lse = (top + (z - top).exp_().sum(1, keepdim=True).log()).view(-1)
    picked = z.gather(1, s["target"].clamp(min=0).view(-1, 1)).view(-1)
    return torch.where(s["target"] >= 0, lse - picked, 0.0), lse


def _plain_orthogonalized(u):
    a, b, c = COEFFICIENTS
    u = u.float()
    tall = u.shape[1] > u.shape[2]
    x = u.transpose(1, 2).contiguous() if tall else u
    norm = x.double().square().sum((1, 2), keepdim=True).sqrt()
    x = (x / norm).float()
    for _ in range(STEPS):
        p = torch.bmm(x, x.transpose(1, 2).contiguous())
        x = a * x + torch.bmm(b * p + c * torch.bmm(p, p), x)
    return x.transpose(1, 2) if tall else x


def _plain(s):
    kind = s["case"]["kind"]
    if kind == "orthogonalize":
        return {"out": _plain_orthogonalized(s["g"]).to(torch.bfloat16)}
    if kind == "step":
        g, m, x = s["g"].float(), s["m"], s["x"]
        m = BETA * m + (1 - BETA) * g
        u = BETA * m + (1 - BETA) * g if s["case"]["ahead"] else m
        s["m"], s["x"] = m, x - s["delta"] * _plain_orthogonalized(u)
        return {"m": s["m"], "x": s["x"]}
    z = _plain_logits(s)
    loss, lse = _plain_loss(s, z)
    if kind == "loss":
        return {"loss": loss, "lse": lse}
    d = z.sub_(lse.view(-1, 1)).exp_()
    rows = torch.arange(d.shape[0], device=d.device)
    at = s["target"].clamp(min=0)
    d[rows, at] = d[rows, at] - 1
    d.mul_(torch.where(s["target"] >= 0, s["dloss"], 0.0).view(-1, 1))
    dh = torch.matmul(d, s["w"].float()).to(torch.bfloat16)
    dw = torch.matmul(d.t(), s["h"].float()).to(torch.bfloat16)
    return {"loss": loss, "lse": lse, "dh": dh, "dw": dw}


def _own(s):
    import paper_1802_04434_amd as ss
    case = s["case"]
    kind = case["kind"]
    if kind in ("loss", "train"):
        if "scratch" not in s:      # kept by the program, for every batch of this size
            s["scratch"] = ss.new_cross_entropy_scratch(case["tokens"], case["vocab"], case["width"])
        ss.cross_entropy(s["h"], s["w"], s["target"], s["loss"], s["lse"], s["scratch"])
        if kind == "loss":
            return {"loss": s["loss"], "lse": s["lse"]}
        ss.cross_entropy_grad(s["h"], s["w"], s["target"], s["lse"], s["dloss"], s["dh"], s["dw"], s["scratch"])
        return {"loss": s["loss"], "lse": s["lse"], "dh": s["dh"], "dw": s["dw"]}
    if "scratch" not in s:
        s["scratch"] = ss.new_orthogonalize_scratch(case["rows"], case["cols"], case["count"])
    if kind == "orthogonalize":
        return {"out": ss.orthogonalize(s["g"], s["out"], s["scratch"], steps=STEPS)}
    ss.orthogonal_step(s["g"], s["m"], BETA, s["delta"], s["x"], s["scratch"], ahead=case["ahead"], steps=STEPS)
    return {"m": s["m"], "x": s["x"]}


def run(state):
    return _own(state) if own else _plain(state)


# ----------------------------------------------------------- in 64 bits ----

def _exact_orthogonalized(u):
    """by the polynomial's own form: X (a + b X'X + c (X'X)^2), on the shorter side, one matrix at a time"""
    a, b, c = COEFFICIENTS
    out = torch.empty(u.shape, dtype=torch.float64, device=u.device)
    for i in range(u.shape[0]):
        x = u[i].double()
        flat = x.shape[0] < x.shape[1]
        if flat:
            x = x.t().contiguous()                  # rows x the shorter side
        x = x / torch.linalg.vector_norm(x)
        eye = torch.eye(x.shape[1], dtype=torch.float64, device=u.device)
        for _ in range(STEPS):
            p = x.t().contiguous() @ x
            x = x @ (a * eye + p @ (b * eye + c * p))
        out[i] = x.t() if flat else x
    return out


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "orthogonalize":
        return {"out": _exact_orthogonalized(s["g"])}
    if kind == "step":
        g, m = s["g"].double(), s["m"].double()
        m = m + (1 - BETA) * (g - m)
        return {"m": m, "x": s["x"].double() - s["delta"] * _exact_orthogonalized(m + (1 - BETA) * (g - m) if case["ahead"] else m)}
    h, w, target = s["h"], s["w"].double(), s["target"]
    wt = w.t().contiguous()
    loss, lse, dh, dw = [], [], [], None
    for at in range(0, case["tokens"], 1024):       # a band of rows at a time, for the memory's sake
        x, to = h[at:at + 1024].double(), target[at:at + 1024]
        z = x @ wt
        there = to >= 0
        log_p = torch.log_softmax(z, 1)
        hit = torch.nn.functional.one_hot(to.clamp(min=0), case["vocab"]) if kind == "train" else None
        nll = -log_p.gather(1, to.clamp(min=0).view(-1, 1)).view(-1)
        loss.append(torch.where(there, nll, 0.0))
        lse.append(torch.logsumexp(z, 1))
        if kind == "train":
            weight = torch.where(there, s["dloss"][at:at + 1024].double(), 0.0)
            d = (log_p.exp_() - hit) * weight.view(-1, 1)
            dh.append(d @ w)
            part = d.t().contiguous() @ x
            dw = part if dw is None else dw + part
    if kind == "loss":
        return {"loss": torch.cat(loss), "lse": torch.cat(lse)}
    return {"loss": torch.cat(loss), "lse": torch.cat(lse), "dh": torch.cat(dh), "dw": dw}
