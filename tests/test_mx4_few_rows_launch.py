"""A few rows against weights of any size are one launch, as the header says, whichever way their waves share rows.  Without a GPU."""
import os
import subprocess
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from test_gradients_mx4_host import BF16, F32, OK, Calls  # noqa: E402
from test_launch_limits import shim, threads  # noqa: E402,F401


def check(c):
    for T, K in ((1, 64), (16, 600), (3, 5000)):
        for N in (1, 15, 2049, 16_384, 16_385, 40_000, (1 << 27) - 17, 1 << 27):
            for xdt in (F32, BF16):
                rc, got = c.linear(T, N, K, xdt)
                assert rc == OK and len(got) == 1 and 0 < threads(got[0]) < 1 << 32, (T, N, K, rc, got)
                # a block has eight waves of 16 rows, or two, four or eight of them share the same rows
                per = N / got[0][0]
                assert per <= 128 and got[0][0] in [-(-N // rows) for rows in (16, 32, 64, 128)], (T, N, K, got)


def test_one_launch(shim):  # noqa: F811
    r = subprocess.run([sys.executable, os.path.abspath(__file__), shim], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr


if __name__ == "__main__":
    check(Calls(sys.argv[1]))
