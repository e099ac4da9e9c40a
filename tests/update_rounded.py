"""Orthogonalised updates with every rounding that the kernels make, in 64 bits: what a result is off by is then only what the order of fp32 sums leaves open,
and whatever else is lost shows, second halves of operands among it."""
import torch

from loss_plain import A, B, C, H16, U16, U32

SCALE = 4096.0


def halves(v):
    """what an fp16 holds of v, and of what that leaves"""
    hi = v.half().double()
    return hi, (v - hi).half().double()


def twofold_steps(shorter, fp32):
    """how many of the last steps of a matrix that is worked on in tiles multiply 22 bits"""
    return 0 if not fp32 or shorter >= 1024 else 1 if shorter >= 512 else 2 if shorter >= 256 else 3


def rounded_to(shape, fp32, tiles, steps):
    """of each step, whether it multiplies 22 bits: matrices taken whole or in slices do in every one"""
    if not tiles:
        return [True] * steps
    shorter = -(-min(shape) // 64) * 64
    return [k + twofold_steps(shorter, fp32) >= steps for k in range(steps)]


class Sums:
    """products of pairs of halves: exact, or each sum off by what fp32 may leave of it.  An addition rounds the sum so far by two units U32 at most, k of them by (k)^1/2 times that;
    the sum so far is no larger than the last one and twice the size of a walk of its terms."""

    def __init__(self, gen=None):
        self.gen = gen
        self.largest = 0.0      # entry of X that was multiplied by an operand of 11 bits

    def draw(self, like):
        return 2 * torch.rand(like.shape, generator=self.gen, dtype=torch.float64, device=like.device) - 1

    def of(self, a, b, twofold, lost=""):
        """a b of halves scaled by SCALE, unscaled once; `lost`: products left out"""
        s = a[0] @ b[0]
        if twofold:
            s = s + (0 if "ab_lo" in lost else a[0] @ b[1]) + (0 if "a_lo_b" in lost else a[1] @ b[0])
        if self.gen is not None:
            k = a[0].shape[1] * (3 if twofold else 1)
            walk = (a[0].square() @ b[0].square()).sqrt()
            s = s + 2 * k ** 0.5 * U32 * (s.abs() + 2 * walk) * self.draw(s)
        return s / SCALE

    def near(self, v, roundings=3):
        """v after that many roundings to fp32"""
        return v if self.gen is None else v * (1 + roundings * U32 * self.draw(v))


def update(g, steps=5, fp32=True, tiles=True, sums=None, lost=""):
    """g as the kernels orthogonalise it, before the result's own rounding.  tiles: whether in products of tiles.  lost: for tests of the tests, what a mistake would leave out."""
    sums = Sums() if sums is None else sums
    x = g.double()
    tall = x.shape[0] > x.shape[1]
    x = x.t() if tall else x
    x = sums.near(x * (SCALE / x.norm()))
    hi, lo = halves(x)
    if "x_lo" in lost:
        lo = lo * 0
    eye = torch.eye(len(x), dtype=torch.float64, device=x.device)
    for k, twofold in enumerate(rounded_to(g.shape, fp32, tiles, steps)):
        if not twofold:
            sums.largest = max(sums.largest, float((hi + lo).abs().max()) / SCALE)
        twofold = twofold and "twofold" not in lost
        mu = {1: 2.0, 2: 0.8}.get(steps - k, 0.0)
        a = halves(sums.near(sums.of((hi, lo), (hi.t(), lo.t()), twofold, lost)))
        whole = a[0] + a[1] if twofold else a[0]
        b = halves(sums.near(B * whole + C * sums.of(a, a, twofold, lost) + mu * SCALE * eye))
        x = sums.near((A - mu) * (hi + lo) + sums.of(b, (hi, lo), twofold, lost))
        if k + 1 < steps or not tiles:
            hi, lo = halves(x)
            if "x_lo" in lost:
                lo = lo * 0
            x = hi + lo
    x = x / SCALE
    return x.t() if tall else x


HALF = {torch.float32: U32, torch.bfloat16: U16}        # half a step of the result's own type, relative


def update_spread(g, want, result, steps=5, tiles=True):
    """How far a result may be from update() in the Frobenius norm before its own rounding: three times the largest of four draws of what sums in fp32 leave open; over few entries six
    times the largest of eight (see loss_plain.orthogonal_bound)."""
    few = g.numel() < 256
    gen = torch.Generator(device=g.device).manual_seed(g.shape[0] * 8191 + g.shape[1])
    return (6 if few else 3) * max(float((update(g, steps, result == torch.float32, tiles, Sums(gen)) - want).norm()) for _ in range(8 if few else 4))


def flipped(largest):
    """How far an entry may be off by what four draws seldom hold: a large entry of A or B, one in a row, that lies between two fp16 and goes the other way, a step, 2 H16, of itself.  It moves an entry
    of the result by that times an entry of X.  |B + mu| <= 2.9, and a step of A_ii makes (|b| - 2 c A) A <= 1.6 of one in B, for A_ii <= 1.44 (X's singular values are 1.2 at most)."""
    return 2 * H16 * (2.9 + 1.6) * largest
