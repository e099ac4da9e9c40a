"""The loss over a vocabulary and orthogonalised updates from their definitions in 64 bits, with the bounds that the kernels'
roundings have: operands of products rounded to 16 bits by at most half a step, sums in fp32."""
import math

import torch

U32, U16, H16 = 2.0 ** -24, 2.0 ** -8, 2.0 ** -11       # half a step of fp32, bf16 and fp16, relative
A, B, C = 3.4445, -4.7750, 2.0315


def softmax_loss(h, w, target, dloss=None):
    """loss, lse, dh, dw of bf16 h and w in 64 bits, and how far each may be off (before the gradients' own rounding)"""
    there = target >= 0
    h64 = torch.where(there[:, None], h.double(), 0.0)
    w64 = w.double()
    K, V = h.shape[1], w.shape[0]
    weight = torch.where(there, 1.0 if dloss is None else dloss.double(), 0.0)
    z = h64 @ w64.t()
    lse = torch.logsumexp(z, 1)
    picked = z.gather(1, target.clamp(0, V - 1)[:, None])[:, 0]
    loss = torch.where(there, lse - picked, 0.0)
    # K exact products added in fp32, whatever the order
    ez = 2 * U32 * K * (h64.abs() @ w64.abs().t())
    # exp(z - top): the difference and its product with log2(e) are rounded, so is the function; the terms' errors weigh as their share p, and
    # the sum of p |log p| is at most log V; 32 T terms of a lane, then the parts
    log_v = math.log(V)
    e_lse = ez.amax(1) + 2 * U32 * (2 * log_v + 8 + 80 + V / 32) + 2 * U32 * lse.abs()
    e_loss = torch.where(there, e_lse + ez.gather(1, target.clamp(0, V - 1)[:, None])[:, 0] + U32 * (lse - picked).abs(), 0.0)
    p = (z - lse[:, None]).exp()
    d = p.clone()
    d[torch.arange(len(d), device=d.device), target.clamp(0, V - 1)] -= 1.0
    d *= weight[:, None]
    ep = p * (ez + e_lse[:, None] + 4 * U32 * ((z - lse[:, None]).abs() + 4))
    ed = ep * weight.abs()[:, None] + (U16 + 8 * U32) * d.abs()
    edh = ed @ w64.abs() + 2 * U32 * (V + 64) * (d.abs() @ w64.abs())
    edw = ed.t() @ h64.abs() + 2 * U32 * (len(d) + 64) * (d.abs().t() @ h64.abs())
    return {"loss": (loss, e_loss), "lse": (lse, e_lse), "dh": (d @ w64, edh), "dw": (d.t() @ h64, edw)}


def polynomial(s):
    return A * s + B * s ** 3 + C * s ** 5


def orthogonalized(g, steps=5):
    """of one matrix, in 64 bits"""
    x = g.double()
    x = x.t() if x.shape[0] > x.shape[1] else x
    norm = x.norm()
    x = x / norm if norm > 0 else x
    for _ in range(steps):
        p = x @ x.t()
        x = A * x + (B * p + C * p @ p) @ x
    return x.t() if g.shape[0] > g.shape[1] else x


def rounded_steps(g, steps, gen):
    """the steps with what the kernel rounds to fp16 off by anything up to half a step, each entry by its own draw"""
    x = g.double()
    tall = x.shape[0] > x.shape[1]
    x = x.t() if tall else x
    x = x / x.norm()
    off = lambda t, h: t * (1 + h * (2 * torch.rand(t.shape, generator=gen, dtype=torch.float64, device=t.device) - 1))  # noqa: E731
    for k in range(steps):
        mu = {1: 2.0, 2: 0.8}.get(steps - k, 0.0)
        hi = off(x, H16)
        p = off(hi @ hi.t(), H16)
        b = off(B * p + C * p @ p + mu * torch.eye(len(p), dtype=torch.float64, device=p.device), H16)
        x = off((A - mu) * x + b @ hi, H16 ** 2)
    return x.t() if tall else x


def orthogonal_bound(g, steps=5):
    """How far the result may be off in the Frobenius norm.  To first order it is a sum over the roundings, each off by up to half a step and each on its own,
    so that its size is that of the same sum over random draws as large as a rounding can be (a rounding's own is smaller by a factor between 1 and 2).  Over many
    entries that size hardly varies: three times the largest of four draws; over few, six times the largest of eight, where all of them could add up:
    15 roundings of an entry, of equal weight, are off by (3 x 15)^1/2 = 6.7 deviations at most, a draw of eight by one at least.  Sums in fp32 over
    k terms are off by k^1/2 2^-24, a hundredth of that."""
    want = orthogonalized(g, steps)
    gen = torch.Generator(device=g.device).manual_seed(g.shape[0] * 8191 + g.shape[1])
    few = g.numel() < 256
    return (6 if few else 3) * max(float((rounded_steps(g, steps, gen) - want).norm()) for _ in range(8 if few else 4))
