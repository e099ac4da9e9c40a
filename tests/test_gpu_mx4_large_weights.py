"""A few rows against weights whose scales are 4 GiB and more, 64 GiB of codes with them: to the bit, on values whose sums are exact in fp32."""
import pytest
import torch

import paper_1802_04434_amd as ss

pytestmark = pytest.mark.gpu
DEV = "cuda"


# 2^30 scales of four, of which 32 bits say 0 bytes; more, with rows and columns that fill no tile, group or step
@pytest.mark.parametrize("N,K", [(1 << 20, 1 << 17), ((1 << 20) + 5, (1 << 17) + 300)])
def test_scales_beyond_32_bits(N, K):
    w = ss.new_mx4(N, K)
    groups = w.scales.shape[0]
    assert N * groups >= 1 << 30
    w.data.fill_(0x22)                               # ones
    w.data[:, K // 2:] = 0
    gen = torch.Generator(device=DEV)
    gen.manual_seed(N)
    sums = torch.zeros(N, dtype=torch.int64, device=DEV)
    for g in range(groups):                          # each block of 32 counts once or twice
        w.scales[g].random_(127, 129, generator=gen)
        columns = torch.tensor([min(max(K - g * 128 - 32 * b, 0), 32) for b in range(4)], device=DEV)
        sums += ((w.scales[g].to(torch.int32) - 126) * columns).sum(1)
    for T in (1, 16, 17):
        powers = torch.exp2(torch.arange(T, device=DEV) - 8.0)
        x = powers[:, None].expand(T, K).contiguous()
        a = ss.new_mx4(T, K)
        ss.mx4_quantize(x, a)
        want = (powers.double()[:, None] * sums.double()).float()
        assert torch.equal(ss.mx4_matmul(a, w, torch.empty(T, N, device=DEV)), want)
        assert torch.equal(ss.mx4_matmul(w, a, torch.empty(N, T, device=DEV)), want.t())
        for dtype in (torch.float32, torch.bfloat16) if T <= 16 else ():
            assert torch.equal(ss.mx4_linear(x.to(dtype), w, torch.empty(T, N, device=DEV)), want)
