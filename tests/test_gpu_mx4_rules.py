"""MX4 matrices on the GPU on both sides of the rules on size: products cut into tiles of each size, edge strips and parts of
their sums, a few rows with waves that share or do not, matrices that are read with another cache policy."""
import pytest
import torch

import paper_1802_04434_amd as ss
from test_gpu_mx4 import DEV, DTYPES

pytestmark = pytest.mark.gpu

PRODUCTS = [(1, 64, 20_000), (40, 4096, 4096), (64, 16_384, 100), (255, 256, 8192), (256, 257, 520), (300, 1000, 3000), (385, 383, 10_000), (512, 512, 512), (1000, 1031, 777),
            (1024, 1024, 16_000), (1153, 2177, 640), (2048, 2048, 300), (2049, 2049, 2048), (2050, 4100, 1000), (4096, 4096, 129), (4099, 8192, 256), (4097, 4098, 700), (2052, 4099, 16_000), (2084, 4130, 8192),
            (1, 1, 8192), (16, 17, 600), (17, 16, 600), (5, 700, 70), (700, 5, 4097), (7, 16_384, 8192), (32_768, 3, 4096), (16, 2000, 9000), (15, 33, 70_000)]
LINEARS = [(700, 4096), (6000, 3000), (9000, 4097), (12_288, 1000), (12_289, 4096), (16_384, 8192), (16_383, 8192), (24_576, 700), (32_768, 4096), (32_767, 4096),
           (40_000, 9000), (4097, 32_800), (300, 10_240), (300, 10_241), (20_000, 10_000), (5000, 4096), (33_000, 600)]
MATRICES = [(8192, 8191), (8192, 8192), (4096, 8192), (4096, 8191), (8320, 8300)]


def operand(seed, rows, cols):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    x = torch.randn(rows, cols, device=DEV, generator=gen) * torch.exp2(torch.randint(-6, 7, (rows, 1), device=DEV, generator=gen).float())
    q = ss.new_mx4(rows, cols)
    ss.mx4_quantize(x, q)
    return q, ss.mx4_dequantize(q, x).double()


def check(got, x, w, dtype):
    """each of at most K additions is off by 2^-23 of the magnitudes' sum, which the double product is by 2^-50; then one rounding,
    which keeps the order of numbers"""
    want, bound = x @ w.t(), x.abs() @ w.abs().t() * x.shape[1] * (2.0 ** -23 + 2.0 ** -50)
    low, high = (v.float().to(DTYPES[dtype]).double() for v in (want - bound, want + bound))
    got = got.double()
    assert bool(((low <= got) & (got <= high)).all()), float((got - want).abs().max())


@pytest.mark.parametrize("M,N,K", PRODUCTS)
def test_products(M, N, K):
    a, x = operand(M + K, M, K)
    b, w = operand(3 * N + K, N, K)
    for dtype, pad in (("f32", 0), ("bf16", 5)):
        out = torch.full((M, N + pad), 77.0, dtype=DTYPES[dtype], device=DEV)
        ss.mx4_matmul(a, b, out[:, :N])
        check(out[:, :N], x, w, dtype)
        assert bool((out[:, N:] == 77.0).all())


@pytest.mark.parametrize("N,K", LINEARS)
def test_linears(N, K):
    w, values = operand(N + K, N, K)
    for T, xdt, odt in ((1, "bf16", "bf16"), (16, "f32", "f32"), (5, "bf16", "f32"), (12, "f32", "bf16")):
        x = torch.randn(T, K, device=DEV).to(DTYPES[xdt])
        q = ss.new_mx4(T, K)
        ss.mx4_quantize(x, q)
        want = ss.mx4_dequantize(q, torch.empty(T, K, device=DEV)).double()
        out = torch.full((T, N + 3), 77.0, dtype=DTYPES[odt], device=DEV)
        ss.mx4_linear(x, w, out[:, :N])
        check(out[:, :N], want, values, odt)
        assert bool((out[:, N:] == 77.0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", MATRICES)
def test_quantisation_of_a_whole_is_that_of_its_parts(rows, cols, dtype):
    x = torch.randn(rows, cols, device=DEV).to(DTYPES[dtype])
    q, qt, only_q, only_t = ss.new_mx4(rows, cols), ss.new_mx4(cols, rows), ss.new_mx4(rows, cols), ss.new_mx4(cols, rows)
    ss.mx4_quantize(x, q, qt)
    ss.mx4_quantize(x, only_q)
    ss.mx4_quantize(x, None, only_t)
    for one, other in ((q, only_q), (qt, only_t)):
        assert torch.equal(one.data, other.data) and torch.equal(one.scales, other.scales)
    for a, b in ((0, 300), (rows - 513, rows)):
        part = ss.new_mx4(b - a, cols)
        ss.mx4_quantize(x[a:b], part)
        assert torch.equal(part.data, q.data[a:b]) and torch.equal(part.scales, q.scales[:, a:b])
    for a, b in ((0, 300), (cols - 513, cols)):
        part = ss.new_mx4(b - a, rows)
        ss.mx4_quantize(x[:, a:b], None, part)
        assert torch.equal(part.data, qt.data[a:b]) and torch.equal(part.scales, qt.scales[:, a:b])
