"""What the operators on lists of gradients and on MX4 matrices refuse, before anything is launched, and what they launch, without a
GPU: the runtime's launch call is replaced by the recorder of test_launch_limits."""
import ctypes
import os
import re
import subprocess
import sys

import pytest

from test_launch_limits import Recorder, shim, threads  # noqa: F401

OK, NULL, ALIGN, DTYPE, ARG = 0, -1, -3, -4, -5
F32, BF16 = 0, 1
vp, sz, f32 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_float


class Calls(Recorder):
    """the new entry points with made-up addresses"""

    def __init__(self, path):
        super().__init__(path)
        for name in ("ss_grad_norm_workspace_bytes", "ss_mx4_padded", "ss_mx4_data_bytes", "ss_mx4_scale_bytes", "ss_mx4_matmul_scratch_bytes"):
            getattr(self.lib, name).restype = sz

    def anew(self):
        self.shim.record_anew(-1)

    def lists(self, lengths, types=None, at=None):
        types = types or [F32] * len(lengths)
        at = at or [self.buffer(4 * n) for n in lengths]
        return self.table(at), (ctypes.c_int * len(lengths))(*types), (sz * len(lengths))(*lengths), sz(len(lengths))

    def norm(self, lengths, types=None, at=None, norm=None, ws=None):
        self.anew()
        return self.lib.ss_grad_norm(*self.lists(lengths, types, at), vp(norm if norm is not None else self.buffer(4)),
                                     vp(ws if ws is not None else self.buffer(8192)), None), self.launches()

    def clip(self, lengths, types=None, at=None, out=None, odt=None, norm=None, max_norm=1.0):
        self.anew()
        g, t, n, count = self.lists(lengths, types, at)
        if out is None:
            flat = self.buffer(4 * sum(lengths))
            out = [flat + 4 * sum(lengths[:i]) for i in range(len(lengths))]
        odt = (ctypes.c_int * len(lengths))(*(odt or [F32] * len(lengths)))
        return self.lib.ss_grad_clip(g, t, n, count, vp(norm if norm is not None else self.buffer(4)), f32(max_norm), self.table(out), odt,
                                     None), self.launches()

    def quantize(self, rows, cols, dt=F32, ld=None, want=(1, 1, 1, 1), x=None, **at):
        self.anew()
        p = [vp(at.get(k, self.buffer(getattr(self.lib, f)(sz(r), sz(c)) + 16))) if w else None for w, k, f, r, c in
             zip(want, ("data", "scales", "data_t", "scales_t"), ("ss_mx4_data_bytes", "ss_mx4_scale_bytes") * 2, (rows, rows, cols, cols), (cols, cols, rows, rows))]
        x = self.buffer(4 * rows * (ld or cols) + 4) if x is None else x
        return self.lib.ss_mx4_quantize(vp(x), dt, sz(rows), sz(cols), sz(cols if ld is None else ld), *p, None), self.launches()

    def dequantize(self, rows, cols, dt=F32, ld=None, data=None, scales=None, out=None):
        self.anew()
        pick = lambda p, n: vp(self.buffer(n) if p is None else p)  # noqa: E731
        return self.lib.ss_mx4_dequantize(pick(data, rows * (cols + 128)), pick(scales, rows * (cols + 128) // 8), sz(rows), sz(cols), pick(out, 4 * rows * (ld or cols) + 4),
                                          dt, sz(cols if ld is None else ld), None), self.launches()

    def matmul(self, M, N, K, dt=F32, ld=None, lend=True, **at):
        self.anew()
        pick = lambda k, n: vp(at[k] if k in at else self.buffer(n + 16))  # noqa: E731
        wanted = self.lib.ss_mx4_matmul_scratch_bytes(sz(M), sz(N), sz(K)) if lend else 0
        s = pick("scratch", wanted) if wanted or "scratch" in at else None
        return self.lib.ss_mx4_matmul(pick("a", M * (K + 128)), pick("sa", M * (K + 128)), pick("b", N * (K + 128)), pick("sb", N * (K + 128)), sz(M), sz(N), sz(K),
                                      pick("out", 4 * M * (ld or N) + 4), dt, sz(N if ld is None else ld), s, sz(wanted), None), self.launches()

    def linear(self, T, N, K, xdt=F32, odt=F32, ldx=None, ldo=None, **at):
        self.anew()
        pick = lambda k, n: vp(at[k] if k in at else self.buffer(n + 16))  # noqa: E731
        return self.lib.ss_mx4_linear(pick("x", 4 * T * (ldx or K) + 4), xdt, sz(T), sz(K if ldx is None else ldx), pick("w", N * (K + 128)), pick("sw", N * (K + 128)),
                                      sz(N), sz(K), pick("out", 4 * T * (ldo or N) + 4), odt, sz(N if ldo is None else ldo), None), self.launches()


def check_lists_are_refused(c):
    good = c.buffer(1 << 20)
    for call in (c.norm, c.clip):
        assert call([10, 0, 3])[0] == OK and call([])[0] == OK
        assert call([10, 3], at=[good, 0]) == (NULL, []) and call([10, 0], at=[good, 0])[0] == OK
        assert call([10], types=[2]) == (DTYPE, []) and call([10], types=[-1]) == (DTYPE, [])
        assert call([10], at=[good + 2]) == (ALIGN, []) and call([10], types=[BF16], at=[good + 1]) == (ALIGN, [])
        assert call([10], at=[good + 4])[0] == OK and call([10], types=[BF16], at=[good + 2])[0] == OK
        assert call([10], norm=0) == (NULL, []) and call([10], norm=good + 4096 + 8) == (ALIGN, [])
        for n in ([1 << 41], [(1 << 40)] * 5, [(1 << 64) - 1], [1 << 62, 1 << 62]):
            assert call(n, at=[good] * len(n), **({"out": [good] * len(n)} if call == c.clip else {})) == (ARG, []), n
    assert c.norm([10], ws=0) == (NULL, []) and c.norm([10], ws=good + 8) == (ALIGN, [])
    assert c.norm([10], at=[good], norm=good + 32) == (ARG, []) and c.norm([10], at=[good], norm=good + 48)[0] == OK
    assert c.norm([10], at=[good], ws=good + 32) == (ARG, []) and c.norm([10], ws=good, norm=good + 64) == (ARG, [])
    for bad in (-1.0, float("nan"), float("inf")):
        assert c.clip([10], max_norm=bad) == (ARG, [])
    assert c.clip([10], at=[good], out=[good])[0] == OK
    for at, out in (([good], [good + 4]), ([good], [good + 36]), ([good + 400, good], [good, good + 400]), ([good, good], [good, good]),
                    ([good + 4096, good + 8192], [good, good + 16]), ([good, good + 8192], [good + 12288, good + 20])):
        assert c.clip([10] * len(at), at=at, out=out) == (ARG, []), (at, out)
    assert c.clip([10], at=[good], out=[good], odt=[BF16]) == (ARG, [])          # another type is no clip in place
    assert c.clip([10], at=[good], out=[good + 40])[0] == OK
    assert c.clip([10], out=[good], norm=good + 32) == (ARG, []) and c.clip([10], at=[good + 4096], out=[0]) == (NULL, [])
    assert c.clip([10], odt=[7]) == (DTYPE, [])


def check_how_lists_are_launched(c):
    header = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "signsgd.h")).read()
    for call, name in ((c.norm, "NORM"), (c.clip, "CLIP")):
        per = int(re.search(r"SS_GRAD_%s_PER_LAUNCH (\d+)" % name, header).group(1))
        for n, launches in ((0, 1 if call == c.norm else 0), (1, 1), (per, 1), (per + 1, 2), (5 * per, 5)):
            for lengths in ([100] * n, [0, 100, 0] * n):
                rc, got = call(lengths)
                assert rc == OK and len(got) == launches and all(0 < threads(t) < 1 << 32 for t in got), (name, n)
    assert c.norm([0] * 1000)[0] == OK and c.clip([0] * 1000) == (OK, [])
    # a tensor of a quarter of the card's memory and more, and many of them
    for lengths, types in (([1 << 36], [F32]), ([(1 << 37) - 3], [BF16]), ([(1 << 34) + 1] * 9, [BF16] * 9)):
        rc, got = c.norm(lengths, types)
        assert rc == OK and len(got) == 1 and got[0][0] <= 256
        rc, got = c.clip(lengths, types)
        assert rc == OK and all(0 < threads(t) < 1 << 32 for t in got)


def check_matrices_are_refused(c):
    good = c.buffer(1 << 30)
    assert c.quantize(5, 100)[0] == OK and c.quantize(5, 100, BF16)[0] == OK and c.quantize(0, 100) == (OK, []) and c.quantize(100, 0) == (OK, [])
    for dt in (2, -1):
        assert c.quantize(5, 100, dt) == (DTYPE, []) and c.dequantize(5, 100, dt) == (DTYPE, []) and c.matmul(5, 6, 100, dt) == (DTYPE, [])
        assert c.linear(5, 6, 100, dt) == (DTYPE, []) and c.linear(5, 6, 100, F32, dt) == (DTYPE, [])
    for want in ((1, 0, 0, 0), (0, 1, 1, 1), (1, 1, 0, 1), (0, 0, 0, 0)):
        assert c.quantize(5, 100, want=want) == (NULL, [])
    assert c.quantize(5, 100, x=0) == (NULL, [])
    assert c.quantize(5, 100, ld=99) == (ARG, []) and c.quantize(5, 100, ld=1 << 41) == (ARG, [])
    assert c.quantize((1 << 27) + 1, 1, x=good) == (ARG, []) and c.quantize(1, (1 << 27) + 1, x=good) == (ARG, []) and c.quantize(1 << 20, 1 << 20, x=good) == (ARG, [])
    assert c.quantize(5, 100, x=good + 2) == (ALIGN, []) and c.quantize(5, 100, BF16, x=good + 2)[0] == OK and c.quantize(5, 100, BF16, x=good + 1) == (ALIGN, [])
    for name in ("data", "scales", "data_t", "scales_t"):
        assert c.quantize(5, 100, **{name: good + 8}) == (ALIGN, [])
        assert c.quantize(5, 100, x=good, **{name: good + 1600}) == (ARG, []), name
    assert c.quantize(5, 100, data=good, data_t=good + 64) == (ARG, [])
    assert c.dequantize(5, 100, data=0) == (NULL, []) and c.dequantize(5, 100, scales=0) == (NULL, []) and c.dequantize(5, 100, out=0) == (NULL, [])
    assert c.dequantize(5, 100, data=good + 8) == (ALIGN, []) and c.dequantize(5, 100, scales=good + 4) == (ALIGN, []) and c.dequantize(5, 100, out=good + 2) == (ALIGN, [])
    assert c.dequantize(5, 100, ld=99) == (ARG, []) and c.dequantize(5, 100, data=good, out=good + 64) == (ARG, []) and c.dequantize(0, 5) == (OK, [])
    for name in ("a", "sa", "b", "sb", "out"):
        assert c.matmul(5, 6, 100, **{name: 0}) == (NULL, [])
        assert c.matmul(5, 6, 100, **{name: good + (8 if name != "out" else 2)}) == (ALIGN, [])
    assert c.matmul(5, 6, 100, scratch=good + 8) == (ALIGN, [])
    assert c.matmul(5, 6, 100, a=good, b=good)[0] == OK                         # read only: a product with itself
    for name in ("a", "sa", "b", "sb"):
        assert c.matmul(5, 6, 100, out=good + 16, **{name: good}) == (ARG, [])
    assert c.matmul(5, 6, 100, ld=5) == (ARG, []) and c.matmul(5, 6, (1 << 24) + 1, a=good) == (ARG, []) and c.matmul(1 << 18, 1 << 18, 100, out=good) == (ARG, [])
    assert c.matmul(0, 6, 100) == (OK, []) and c.matmul(5, 0, 100) == (OK, []) and len(c.matmul(5, 6, 0)[1]) == 1
    for name in ("x", "w", "sw", "out"):
        assert c.linear(5, 6, 100, **{name: 0}) == (NULL, [])
        assert c.linear(5, 6, 100, **{name: good + (8 if name[-1] == "w" else 2)}) == (ALIGN, [])
    assert c.linear(17, 6, 100) == (ARG, []) and c.linear(16, 6, 100)[0] == OK and c.linear(0, 6, 100) == (OK, []) and c.linear(5, 0, 100) == (OK, [])
    assert c.linear(5, 6, 100, ldx=99) == (ARG, []) and c.linear(5, 6, 100, ldo=5) == (ARG, []) and c.linear(5, 6, 100, x=good, out=good + 4) == (ARG, [])


def check_sizes_of_matrices(c):
    L = c.lib
    for cols, padded in ((0, 0), (1, 128), (128, 128), (129, 256), (4096, 4096)):
        assert L.ss_mx4_padded(sz(cols)) == padded
        assert L.ss_mx4_data_bytes(sz(7), sz(cols)) == 7 * padded // 2 and L.ss_mx4_scale_bytes(sz(7), sz(cols)) == 7 * padded // 32
    assert L.ss_grad_norm_workspace_bytes() <= 8192 and L.ss_grad_norm_workspace_bytes() % 8 == 0


def check_large_matrices_are_launched(c):
    for rows, cols in ((1 << 27, 128), (1 << 27, 1), (1, 1 << 27), (128, 1 << 27), (1 << 17, 1 << 17), ((1 << 27) - 1, 127), (3, (1 << 27) - 5)):
        for dt in (F32, BF16):
            for want in ((1, 1, 0, 0), (0, 0, 1, 1), (1, 1, 1, 1)):
                rc, got = c.quantize(rows, cols, dt, want=want)
                assert rc == OK and len(got) == 1 and 0 < threads(got[0]) < 1 << 32, (rows, cols, dt, want, rc)
            rc, got = c.dequantize(rows, cols, dt)
            assert rc == OK and len(got) == 1 and 0 < threads(got[0]) < 1 << 32, (rows, cols, dt, rc)
    for M, N, K in ((1 << 27, 128, 128), (1 << 27, 1, 64), (1, 1 << 27, 64), (1 << 17, 1 << 17, 512), (16, 16, 1 << 24), (128, 1 << 27, 64)):
        for lend in (True, False):
            rc, got = c.matmul(M, N, K, BF16, lend=lend)
            assert rc == OK and got and all(0 < threads(t) < 1 << 32 for t in got), (M, N, K, rc)
    for T, N, K in ((16, 1 << 27, 128), (1, 1 << 27, 64), (16, 5, 1 << 27)):
        rc, got = c.linear(T, N, K)
        assert rc == OK and got and all(0 < threads(t) < 1 << 32 for t in got), (T, N, K, rc)


CHECKS = {f.__name__: f for f in (check_lists_are_refused, check_how_lists_are_launched, check_matrices_are_refused, check_sizes_of_matrices,
                                  check_large_matrices_are_launched)}


@pytest.mark.parametrize("name", sorted(CHECKS))
def test_without_a_gpu(shim, name):  # noqa: F811
    r = subprocess.run([sys.executable, os.path.abspath(__file__), shim, name], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr


def test_the_binding_refuses_what_is_no_device_tensor():
    import torch

    import paper_1802_04434_amd as ss
    host, norm, ws = torch.zeros(64), torch.zeros(1), torch.zeros(1024, dtype=torch.int64)
    q = ss.new_mx4(8, 64, device="cpu")
    assert q.data.shape == (8, 64) and q.scales.shape == (1, 8, 4)
    with pytest.raises(TypeError, match="norm must live in device memory"):
        ss.grad_norm([host], norm, ws)
    with pytest.raises(TypeError, match="norm must live in device memory"):
        ss.grad_clip([host], norm, 1.0)
    with pytest.raises(TypeError, match="x must live in device memory"):
        ss.mx4_quantize(host.view(8, 8), q)
    with pytest.raises(TypeError, match="q.data must live in device memory"):
        ss.mx4_dequantize(q, host.view(8, 8))
    with pytest.raises(TypeError, match="a must be an Mx4, got Tensor"):
        ss.mx4_matmul(host, q, host.view(8, 8))
    with pytest.raises(TypeError, match="x must be a tensor"):
        ss.mx4_linear([1.0], q, host)


if __name__ == "__main__":
    CHECKS[sys.argv[2]](Calls(sys.argv[1]))
