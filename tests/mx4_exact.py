"""MX4 operands whose products add up exactly in fp32, in whatever order: a lost, doubled or misplaced block shows in the result's bits,
however long the sum.

Values are E2M1 codes times 2^-1, 1 or 2 (1 alone where the sums are longer than LONG), so products are multiples of 2^-4 (2^-2).
While the magnitudes of a sum's products stay below 2^24 of these units, every partial sum is an fp32."""
import torch

BOOK = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
LONG = 60_000


def operand(seed, rows, cols, device="cpu"):
    """data, scales (as the library lays them out) and the values in 64 bits.  Every block has a magnitude of 4 or 6, so that quantising
    the values along the rows gives these codes again."""
    gen = torch.Generator(device=device)
    gen.manual_seed(seed * 1_000_003 + rows * 1009 + cols)
    groups = -(-cols // 128)
    code = torch.randint(0, 16, (rows, groups * 4, 32), generator=gen, dtype=torch.uint8, device=device)
    for_block = torch.tensor([max(0, min(32, cols - 32 * k)) for k in range(groups * 4)], device=device)        # columns that each block has
    at = (torch.rand(rows, groups * 4, 1, generator=gen, device=device) * for_block[:, None]).long().clamp_(max=31)
    code.scatter_(2, at, (torch.randint(6, 8, at.shape, generator=gen, device=device) + 8 * torch.randint(0, 2, at.shape, generator=gen, device=device)).to(torch.uint8))
    code = code.view(rows, -1)
    code[:, cols:] = 0
    e = torch.randint(-1, 2, (rows, groups * 4), generator=gen, device=device) * int(cols <= LONG)
    e[:, for_block == 0] = 0
    book = torch.tensor([*BOOK, *(-v for v in BOOK)], dtype=torch.float64, device=device)
    values = (book[code.long()].view(rows, -1, 32) * torch.exp2(e.double())[..., None]).view(rows, -1)[:, :cols].contiguous()
    data = code[:, 0::2] | (code[:, 1::2] << 4)
    scales = (e + 127).to(torch.uint8).view(rows, groups, 4).permute(1, 0, 2).contiguous()
    return data.contiguous(), scales, values


def product(x, w):
    """x w^T, after a look at whether every order of the additions is exact in fp32"""
    unit = 2.0 ** -4 if x.shape[1] <= LONG else 2.0 ** -2
    assert float((x.abs() @ w.abs().t()).max()) / unit < 2 ** 24
    return x @ w.t()
