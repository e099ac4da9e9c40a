"""Which kernels the operators on gradients and on MX4 matrices launch, without a GPU: every one that the library holds is reached,
and the sizes in test_gpu_mx4_rules stand on both sides of every rule."""
import os
import re
import subprocess
import sys

import pytest

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import test_gpu_mx4_rules as gpu  # noqa: E402
from test_gradients_mx4_host import BF16, F32, OK, Calls  # noqa: E402
from test_launch_limits import shim  # noqa: E402,F401
from test_launch_rules import Rules  # noqa: E402


class Kernels(Calls, Rules):
    def of(self, call, *args, **how):
        assert call(*args, **how)[0] == OK, (args, how)
        return self.kernels()


def numbers(symbol):
    """a kernel's template parameters that are numbers or truth values"""
    return tuple(int(v) for v in re.findall(r"L[ib](\d+)E", symbol))


def check_every_kernel_is_reached(k):
    seen = set()
    for n in (100, 1 << 26, (1 << 28) - 1, 1 << 28, 1 << 29):
        for dt in (F32, BF16):
            seen.update(k.of(k.norm, [n], [dt]))
            for odt in (F32, BF16):
                seen.update(k.of(k.clip, [n], [dt], odt=[odt]))
    for rows, cols in ((100, 100), (8192, 8192)):
        for dt in (F32, BF16):
            for want in ((1, 1, 0, 0), (0, 0, 1, 1), (1, 1, 1, 1)):
                seen.update(k.of(k.quantize, rows, cols, dt, want=want))
            seen.update(k.of(k.dequantize, rows, cols, dt))
    for M, N, K in gpu.PRODUCTS:
        for dt in (F32, BF16):
            seen.update(k.of(k.matmul, M, N, K, dt))
    for N, K in ((100, 100), (64, 8192), (100_000, 4096), (16_384, 16_384)):
        for xdt in (F32, BF16):
            for odt in (F32, BF16):
                seen.update(k.of(k.linear, 3, N, K, xdt, odt))
    held = subprocess.run(["nm", "-D", "--defined-only", k.lib._name], capture_output=True, text=True, check=True).stdout
    held = {t.split()[-1] for t in held.splitlines() if t.split()[1] in "VD" and re.match("_ZN(3mx4|5grads)", t.split()[-1])}
    assert held and held == seen, sorted(held ^ seen)


def check_gpu_tests_reach_both_sides(k):
    tiles, parts, splits = set(), set(), set()
    for M, N, K in gpu.PRODUCTS:
        got = k.of(k.matmul, M, N, K)
        products = [s for s in got if "join" not in s]
        tiles.update(numbers(s)[1] if "matmul_tiles" in s else "few" for s in products)
        parts.add(len(products))
        splits.add(len(got) > len(products))
    assert tiles == {1, 2, 4, "few"} and parts == {1, 2, 3} and splits == {False, True}, (tiles, parts, splits)
    shapes = {numbers(s)[1:] for N, K in gpu.LINEARS for s in k.of(k.linear, 1, N, K)}
    assert len(shapes) == 4 and {s[0] for s in shapes} == {0, 1} and len({s[1:] for s in shapes}) == 2, shapes       # cache policies, columns at a time
    sharers = {round(8 * k.linear(1, N, K)[1][0][0] / -(-N // 16)) for N, K in gpu.LINEARS}       # waves to the same rows, of a block's eight
    assert sharers == {1, 2, 4, 8}, sharers
    for dt in (F32, BF16):
        once = {numbers(s)[-1] for rows, cols in gpu.MATRICES for s in k.of(k.quantize, rows, cols, dt)}
        assert once == {0, 1}, once


CHECKS = {f.__name__: f for f in (check_every_kernel_is_reached, check_gpu_tests_reach_both_sides)}


@pytest.mark.parametrize("name", sorted(CHECKS))
def test_rules(shim, name):  # noqa: F811
    r = subprocess.run([sys.executable, os.path.abspath(__file__), shim, name], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr


if __name__ == "__main__":
    CHECKS[sys.argv[2]](Kernels(sys.argv[1]))
