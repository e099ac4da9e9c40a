"""The exact sums' sizes reach tiles of each size in one part and in several, edge strips, few rows from codes, and every number of waves that
share rows with one pass over the columns and with more.  Without a GPU."""
import os
import subprocess
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import test_gpu_mx4_exact_sums as gpu  # noqa: E402
from test_gradients_mx4_host import BF16, F32  # noqa: E402
from test_gradients_mx4_rules import Kernels, numbers  # noqa: E402
from test_launch_limits import shim  # noqa: E402,F401


def check(k):
    whole, cut, parts, few = set(), set(), set(), set()
    for M, N, K in gpu.PRODUCTS:
        for lend in (True, False):
            got = k.of(k.matmul, M, N, K, lend=lend)
            tiles = [numbers(s)[1] for s in got if "matmul_tiles" in s]
            few.update(numbers(s)[2:] for s in got if "linear" in s)
            parts.add(len([s for s in got if "join" not in s]))
            (cut if any("join" in s for s in got) else whole).update(tiles)
    assert whole == {1, 2, 4} and cut == {1, 2, 4} and parts >= {1, 2, 3} and len(few) == 2, (whole, cut, parts, few)
    seen = set()
    for N, K in gpu.LINEARS:
        for xdt in (F32, BF16):
            steps, in_lds = -(-K // 512), numbers(k.of(k.linear, 1, N, K, xdt)[0])[2]
            sharers = round(8 * k.linear(1, N, K, xdt)[1][0][0] / -(-N // 16))
            seen.add((sharers, steps > in_lds // sharers * sharers))
    assert seen >= {(1, False), (1, True), (2, False), (2, True), (4, True), (8, False), (8, True)}, seen


def test_reach(shim):  # noqa: F811
    r = subprocess.run([sys.executable, os.path.abspath(__file__), shim], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr


if __name__ == "__main__":
    check(Kernels(sys.argv[1]))
