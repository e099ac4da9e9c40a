"""How far apart rows and matrices may be, without a GPU: what is read of the loss's operands by offsets of 32 bits, what is written by 64, and nothing
whose bytes pass 64 bits.  The recorder of test_launch_limits stands in for the runtime's launch call."""
import os
import subprocess
import sys

import pytest

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from test_launch_limits import shim  # noqa: E402,F401
from test_loss_orthogonal_host import ARG, BF16, F32, OK, Calls  # noqa: E402


def check_rows_that_are_read(c):
    good = c.buffer(1 << 40)
    for call in (c.loss, c.grad):
        for name in ("ldh", "ldw"):
            assert call(5, 6, 64, **{name: 1 << 21})[0] == OK
            assert call(5, 6, 64, **{name: (1 << 21) + 1}) == (ARG, [])
            assert call(5, 6, 64, **{name: (1 << 64) - 1, name[2]: good}) == (ARG, [])


def check_rows_that_are_written(c):
    good = c.buffer(1 << 50)
    for name, rows in (("lddh", 5), ("lddw", 6)):
        for dtype in (F32, BF16):
            most = (1 << 40) // (rows - 1)
            for ld in ((1 << 21) + 1, 1 << 22, 1 << 36, most):
                assert c.grad(5, 6, 64, **{name: ld, name[2:]: good, name[2:] + "dt": dtype})[0] == OK, (name, ld)
            for ld in (63, most + 1, 1 << 62, (1 << 64) - 1):
                assert c.grad(5, 6, 64, **{name: ld, name[2:]: good, name[2:] + "dt": dtype}) == (ARG, []), (name, ld)
    # a row by itself has no distance
    assert c.grad(1, 6, 64, lddh=1 << 62, dh=good)[0] == OK
    # a written row that lies over another buffer is still found
    assert c.grad(5, 6, 64, lddh=1 << 30, dh=good, h=good + (1 << 32)) == (ARG, [])


def check_matrices(c):
    good = c.buffer(1 << 50)
    for call, name in ((c.orthogonalize, "out"), (c.step, "x")):
        assert call(3, 5, 6, ld=1 << 36, apart=1 << 39, g=good)[0] == OK
        # 2^14 + 1 matrices 2^48 elements apart: their last byte is 2^64 + 4 from the first, which a sum of 64 bits takes for 4
        for count, ld, apart in (((1 << 14) + 1, 1, 1 << 48), (3, 1, (1 << 39) + 1), (3, 1, 1 << 62), (3, 1, (1 << 64) - 1)):
            assert call(count, 1, 1, ld=ld, apart=apart, g=good, **{name: good + (1 << 30)}) == (ARG, []), (count, apart)
        for ld in ((1 << 40) // 4 + 1, 1 << 61, (1 << 64) - 1):
            assert call(1, 5, 6, ld=ld, apart=0, g=good) == (ARG, []), ld
        assert call(1, 1, 6, ld=1 << 61, apart=1 << 61, g=good)[0] == OK           # one row of one matrix has no distance
        assert call(3, 5, 6, ld=1 << 30, apart=1 << 34, g=good, **{name: good + (1 << 33)}) == (ARG, [])


CHECKS = {f.__name__: f for f in (check_rows_that_are_read, check_rows_that_are_written, check_matrices)}


@pytest.mark.parametrize("name", sorted(CHECKS))
def test_without_a_gpu(shim, name):  # noqa: F811
    r = subprocess.run([sys.executable, os.path.abspath(__file__), shim, name], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr


if __name__ == "__main__":
    CHECKS[sys.argv[2]](Calls(sys.argv[1]))
