"""Products and single tokens with long sums, to the bit: on operands that add up exactly in fp32 the result is the one number, however the
sum is cut into steps, passes, waves and parts."""
import ctypes

import pytest
import torch

import mx4_exact as exact
import paper_1802_04434_amd as ss

pytestmark = pytest.mark.gpu
DEV = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}

# tiles of each size in one part and in several, sums that end one column into a block, a group and a step, edge strips, few rows or columns
PRODUCTS = [(64, 64, 20_000), (64, 64, 20_001), (15, 33, 70_000), (17, 64, 300_000), (300, 1000, 3000), (300, 1000, 2817), (513, 129, 1500), (385, 383, 10_000), (256, 256, 65_536),
            (1024, 1024, 16_000), (2052, 4099, 16_000), (2050, 4100, 1000), (4099, 2048, 8193), (1, 64, 20_000), (64, 1, 20_033), (7, 16_384, 8192), (1, 1000, 10_241), (16, 2000, 9000), (2000, 16, 9001),
            (3, 700, 33_000), (16, 16, 32_768), (5, 700, 16_500), (1, 4096, 4001), (130, 20, 300_001), (512, 2048, 262_145)]
# on both sides of the columns of x that a block holds, of 512 columns a step, and of waves that share rows or do not
LINEARS = [(300, 4096), (300, 4097), (300, 10_240), (300, 10_241), (64, 16_500), (40, 32_800), (4097, 32_801), (20_000, 10_000), (17_000, 10_300), (9000, 20_600), (33, 70_000),
           (300, 12_289), (1000, 513), (5000, 11_000), (20_000, 4095), (1, 300_001)]


def matrix(seed, rows, cols):
    data, scales, values = exact.operand(seed, rows, cols, DEV)
    return ss.Mx4(data, scales, rows, cols), values


@pytest.mark.parametrize("M,N,K", PRODUCTS)
def test_products(M, N, K):
    a, x = matrix(1, M, K)
    b, w = matrix(2, N, K)
    want = exact.product(x, w).float()
    L, stream = ss.load_library(), torch.cuda.current_stream().cuda_stream
    vp, sz = ctypes.c_void_p, ctypes.c_size_t
    for dtype in DTYPES.values():
        assert torch.equal(ss.mx4_matmul(a, b, torch.full((M, N), 77.0, dtype=dtype, device=DEV)), want.to(dtype))
        # without memory for partial sums
        out = torch.full((M, N), 77.0, dtype=dtype, device=DEV)
        assert L.ss_mx4_matmul(a.data.data_ptr(), a.scales.data_ptr(), b.data.data_ptr(), b.scales.data_ptr(), sz(M), sz(N), sz(K), vp(out.data_ptr()),
                               int(dtype == torch.bfloat16), sz(N), None, sz(0), vp(stream)) == 0
        assert torch.equal(out, want.to(dtype))


@pytest.mark.parametrize("N,K", LINEARS)
def test_linears(N, K):
    q, w = matrix(3, N, K)
    for T in (1, 2, 5, 16):
        x = matrix(4 + T, T, K)[1]
        want = exact.product(x, w).float()
        for xdt in DTYPES.values():
            for odt in DTYPES.values():
                assert torch.equal(ss.mx4_linear(x.to(xdt), q, torch.full((T, N), 77.0, dtype=odt, device=DEV)), want.to(odt))
