"""What the loss over a vocabulary and orthogonalised updates refuse before anything is launched, what they launch, that every kernel is reached, and
that the GPU tests' sizes stand on both sides of every rule, without a GPU: the runtime's launch call is replaced by the recorder of test_launch_limits."""
import ctypes
import os
import re
import subprocess
import sys

import pytest

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import test_gpu_loss as gpu_loss  # noqa: E402
import test_gpu_orthogonal as gpu_orthogonal  # noqa: E402
from test_launch_limits import shim, threads  # noqa: E402,F401
from test_launch_rules import Rules  # noqa: E402

OK, NULL, ALIGN, DTYPE, ARG = 0, -1, -3, -4, -5
F32, BF16 = 0, 1
vp, sz, f32 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_float


class Calls(Rules):
    """the entry points with made-up addresses"""

    def __init__(self, path):
        super().__init__(path)
        for name in ("ss_cross_entropy_scratch_bytes", "ss_orthogonalize_scratch_bytes"):
            getattr(self.lib, name).restype = sz

    def scratch(self, at, name, *sizes):
        wanted = getattr(self.lib, name)(*map(sz, sizes))
        given = at.get("bytes", wanted)
        return vp(at["scratch"] if "scratch" in at else self.buffer(wanted + 16)), sz(given)

    def loss(self, T, V, K, dt=BF16, ldh=None, ldw=None, **at):
        self.shim.record_anew(-1)
        pick = lambda k, n: vp(at[k] if k in at else self.buffer(n + 16))  # noqa: E731
        ldh, ldw = K if ldh is None else ldh, K if ldw is None else ldw
        return self.lib.ss_cross_entropy(pick("h", 2 * T * ldh), dt, sz(T), sz(ldh), pick("w", 2 * V * ldw), sz(V), sz(K), sz(ldw), pick("target", 8 * T), pick("loss", 4 * T),
                                         pick("lse", 4 * T), *self.scratch(at, "ss_cross_entropy_scratch_bytes", T, V, K), None), self.launches()

    def grad(self, T, V, K, dt=BF16, ldh=None, ldw=None, dhdt=BF16, dwdt=BF16, lddh=None, lddw=None, **at):
        self.shim.record_anew(-1)
        pick = lambda k, n: vp(at[k] if k in at else self.buffer(n + 16))  # noqa: E731
        ldh, ldw, lddh, lddw = (K if x is None else x for x in (ldh, ldw, lddh, lddw))
        return self.lib.ss_cross_entropy_grad(pick("h", 2 * T * ldh), dt, sz(T), sz(ldh), pick("w", 2 * V * ldw), sz(V), sz(K), sz(ldw), pick("target", 8 * T), pick("lse", 4 * T),
                                              pick("dloss", 4 * T), pick("dh", 4 * T * lddh), dhdt, sz(lddh), pick("dw", 4 * V * lddw), dwdt, sz(lddw),
                                              *self.scratch(at, "ss_cross_entropy_scratch_bytes", T, V, K), None), self.launches()

    def orthogonalize(self, count, rows, cols, gdt=F32, odt=BF16, ld=None, apart=None, ldo=None, aparto=None, steps=5, **at):
        self.shim.record_anew(-1)
        ld, ldo = cols if ld is None else ld, cols if ldo is None else ldo
        apart, aparto = rows * ld if apart is None else apart, rows * ldo if aparto is None else aparto
        pick = lambda k, n: vp(at[k] if k in at else self.buffer(n + 16))  # noqa: E731
        return self.lib.ss_orthogonalize(pick("g", 4 * count * apart), gdt, sz(count), sz(rows), sz(cols), sz(ld), sz(apart), steps, pick("out", 4 * count * aparto), odt, sz(ldo),
                                         sz(aparto), *self.scratch(at, "ss_orthogonalize_scratch_bytes", count, rows, cols), None), self.launches()

    def step(self, count, rows, cols, gdt=F32, ld=None, apart=None, steps=5, beta=0.9, delta=0.1, ahead=0, **at):
        self.shim.record_anew(-1)
        ld = cols if ld is None else ld
        apart, n = rows * ld if apart is None else apart, 4 * count * rows * cols
        pick = lambda k, n: vp(at[k] if k in at else self.buffer(n + 16))  # noqa: E731
        return self.lib.ss_orthogonal_step(pick("g", 4 * count * apart), gdt, sz(count), sz(rows), sz(cols), sz(ld), sz(apart), pick("m", n), f32(beta), ahead, steps, f32(delta),
                                           pick("x", n), *self.scratch(at, "ss_orthogonalize_scratch_bytes", count, rows, cols), None), self.launches()

    def of(self, call, *args, **how):
        rc, launches = call(*args, **how)
        assert rc == OK and all(0 < threads(t) < 1 << 32 for t in launches), (args, how, rc)
        return self.kernels()


def check_the_loss_is_refused(c):
    good = c.buffer(1 << 30)
    for call in (c.loss, c.grad):
        assert call(5, 6, 100)[0] == OK and call(5, 6, 64)[0] == OK
        assert call(5, 6, 100, dt=F32) == (DTYPE, []) and call(5, 6, 100, dt=2) == (DTYPE, [])
        assert call(5, 0, 100, scratch=good, bytes=1 << 20) == (ARG, []) and call(5, 6, 0, scratch=good, bytes=1 << 20) == (ARG, [])
        for sizes in (((1 << 24) + 1, 6, 8), (1 << 24, 6, 1100), (5, (1 << 24) + 1, 8), (5, 6, (1 << 20) + 1), ((1 << 64) - 1, 6, 8), (5, (1 << 64) - 1, 8)):
            at = {k: good for k in ("h", "w", "target", "loss", "lse", "dloss", "dh", "dw")}
            assert call(*sizes, ldh=max(8, min(sizes[2], 1 << 20)), ldw=max(8, min(sizes[2], 1 << 20)), **at) == (ARG, []), sizes
        assert call(5, 6, 100, ldh=99) == (ARG, []) and call(5, 6, 100, ldw=99) == (ARG, []) and call(5, 6, 100, ldh=1 << 22, h=good) == (ARG, [])
        for name in ("h", "w", "target", "lse"):
            assert call(5, 6, 100, **{name: 0}) == (NULL, []), name
            assert call(5, 6, 100, **{name: good + 1}) == (ALIGN, []), name
        assert call(5, 6, 100, h=good + 2)[0] == OK and call(5, 6, 100, w=good + 2)[0] == OK and call(5, 6, 100, target=good + 4) == (ALIGN, [])
        assert call(5, 6, 100, scratch=0) == (NULL, []) and call(5, 6, 100, scratch=good + 8) == (ALIGN, [])
        assert call(5, 6, 100, scratch=good, bytes=c.lib.ss_cross_entropy_scratch_bytes(sz(5), sz(6), sz(100)) - 1) == (ARG, [])
        assert call(5, 6, 100, h=good, w=good)[0] == OK                    # both are only read
        for name in ("h", "w", "target"):
            assert call(5, 6, 100, scratch=good + 16, **{name: good}) == (ARG, []), name
    assert c.loss(5, 6, 100, loss=good, lse=good + 16) == (ARG, []) and c.loss(5, 6, 100, loss=good, lse=good + 20)[0] == OK
    assert c.loss(5, 6, 100, loss=0) == (NULL, []) and c.loss(5, 6, 100, h=good, loss=good + 900) == (ARG, [])
    assert c.loss(0, 6, 100) == (OK, []) and c.lib.ss_cross_entropy_scratch_bytes(sz(0), sz(6), sz(100)) == 0
    for a, b in (("h", "dh"), ("w", "dw"), ("dh", "dw"), ("lse", "dh"), ("dloss", "dw"), ("target", "dh")):
        assert c.grad(5, 6, 100, **{a: good, b: good + 16}) == (ARG, []), (a, b)
    assert c.grad(5, 6, 100, dh=0)[0] == OK and c.grad(5, 6, 100, dw=0)[0] == OK and c.grad(5, 6, 100, dh=0, dw=0) == (NULL, []) and c.grad(5, 6, 100, dloss=0)[0] == OK
    for name in ("dhdt", "dwdt"):
        assert c.grad(5, 6, 100, **{name: 2}) == (DTYPE, []) and c.grad(5, 6, 100, **{name: F32})[0] == OK
    assert c.grad(5, 6, 100, lddh=99) == (ARG, []) and c.grad(5, 6, 100, lddw=99) == (ARG, []) and c.grad(5, 6, 100, dh=good + 1) == (ALIGN, [])
    assert c.grad(5, 6, 100, dw=good + 2, dwdt=F32) == (ALIGN, []) and c.grad(5, 6, 100, dloss=good + 2) == (ALIGN, [])
    assert len(c.grad(0, 6, 100)[1]) == 1 and c.grad(0, 6, 100, dw=0) == (OK, [])       # the gradient of no rows is zero


def check_updates_are_refused(c):
    good = c.buffer(1 << 30)
    for call in (c.orthogonalize, c.step):
        for rows, cols in ((5, 6), (300, 400)):
            assert call(2, rows, cols)[0] == OK and call(2, rows, cols, gdt=BF16)[0] == OK and call(2, rows, cols, gdt=2) == (DTYPE, [])
            for steps in (0, -1, 101):
                assert call(2, rows, cols, steps=steps) == (ARG, [])
            assert call(2, rows, cols, ld=cols - 1) == (ARG, []) and call(2, rows, cols, apart=rows * cols - 1) == (ARG, []) and call(1, rows, cols, apart=0)[0] == OK
            for name in ("g", "out") if call == c.orthogonalize else ("g", "m", "x"):
                assert call(2, rows, cols, **{name: 0}) == (NULL, []), name
                assert call(2, rows, cols, **{name: good + 1}) == (ALIGN, []), name
                assert call(2, rows, cols, scratch=good + 16, **{name: good}) == (ARG, []), name
            assert call(2, rows, cols, scratch=0) == (NULL, []) and call(2, rows, cols, scratch=good + 8) == (ALIGN, [])
            assert call(2, rows, cols, scratch=good, bytes=c.lib.ss_orthogonalize_scratch_bytes(sz(2), sz(rows), sz(cols)) - 1) == (ARG, [])
        for sizes in ((65536, 1, 1), (1, (1 << 20) + 1, 1), (1, 1, (1 << 20) + 1), (1, (1 << 15) + 1, (1 << 15) + 1), (65535, 4096, 4096), ((1 << 64) - 1,) * 3):
            at = {k: good for k in ("g", "out", "m", "x")}
            assert call(*sizes, apart=1, scratch=good, bytes=1 << 20, **at) == (ARG, []), sizes
            assert c.lib.ss_orthogonalize_scratch_bytes(*map(sz, sizes)) == 0
        for empty in ((0, 5, 6), (2, 0, 6), (2, 5, 0)):
            assert call(*empty) == (OK, []) and c.lib.ss_orthogonalize_scratch_bytes(*map(sz, empty)) == 0
    assert c.orthogonalize(2, 5, 6, odt=2) == (DTYPE, []) and c.orthogonalize(2, 5, 6, ldo=5) == (ARG, []) and c.orthogonalize(2, 5, 6, g=good, out=good + 16) == (ARG, [])
    assert c.orthogonalize(2, 5, 6, g=good, out=good) == (ARG, [])
    for how in ({"beta": float("nan")}, {"beta": float("inf")}, {"delta": float("nan")}, {"delta": float("inf")}, {"ahead": 2}, {"ahead": -1}):
        assert c.step(2, 5, 6, **how) == (ARG, []), how
    for a, b in (("g", "m"), ("g", "x"), ("m", "x")):
        assert c.step(2, 5, 6, **{a: good, b: good + 16}) == (ARG, []), (a, b)


def check_large_sizes_are_launched(c):
    for T, V, K in ((1 << 24, 64, 8), (64, 1 << 24, 8), (64, 64, 1 << 20), (1 << 20, 1 << 19, 64), (1, 1 << 24, 1 << 12), (1 << 24, 1 << 20, 1)):
        c.of(c.loss, T, V, K)
        if T * V <= 1 << 39:
            c.of(c.grad, T, V, K)
    for count, rows, cols in ((65535, 1, 1), (65535, 64, 64), (1, 1 << 20, 1), (1, 64, 1 << 20), (1, 1 << 15, 1 << 15), (1, 1 << 13, 1 << 20), (2000, 1024, 1024), (65535, 96, 800)):
        for call in (c.orthogonalize, c.step):
            c.of(call, count, rows, cols)


def kind(symbol):
    """kernel, its ends, and its template parameters that are numbers or truth values"""
    return re.search(r"_ZN\d+\w+?(\d+)([a-z_]+_kernel)", symbol).group(2), re.findall(r"\d+([A-Z][a-z]+End)", symbol), tuple(int(v) for v in re.findall(r"L[ibj](\d+)E", symbol))


# what each kind of call meets: more than the GPU tests', for the sizes that these would take long with
LARGE_LOSSES = [(8192, 128000, 4096), (8192, 128000, 4008), (900, 20000, 1002), (8192, 8192, 8192), (4096, 32000, 2048), (2048, 2048, 2048), (300, 700, 192), (4096, 4096, 64), (64, 64, 64), (16, 256, 8192), (1024, 1024, 8192)]
LARGE_MATRICES = [(1, 8192, 8192), (1, 4096, 4096), (1, 2048, 2048), (1, 1024, 1024), (1, 512, 4096), (1, 4096, 512), (24, 512, 2048), (24, 2048, 512), (1, 20, 30), (1, 30, 800), (1, 90, 90), (1, 250, 80), (1, 100, 30), (1, 60, 300), (1, 130, 8192), (1, 128, 100_000), (1, 100_000, 128), (300, 150, 250), (300, 250, 150), (1, 8192, 130), (8, 4096, 8192),
                  (8, 8192, 4096), (1, 32768, 2048), (1, 2048, 32768)]


def check_every_kernel_is_reached(c):
    seen = set()
    for T, V, K in gpu_loss.SIZES + gpu_loss.LARGE + LARGE_LOSSES:
        seen.update(c.of(c.loss, T, V, K))
        seen.update(c.of(c.grad, T, V, K))
    seen.update(c.of(c.grad, 0, 5, 6))
    for count, rows, cols in [(1, *s) for s in gpu_orthogonal.SHAPES + gpu_orthogonal.LARGE] + LARGE_MATRICES:
        seen.update(c.of(c.orthogonalize, count, rows, cols))
        seen.update(c.of(c.step, count, rows, cols))
    held = subprocess.run(["nm", "-D", "--defined-only", c.lib._name], capture_output=True, text=True, check=True).stdout
    held = {t.split()[-1] for t in held.splitlines() if t.split()[1] in "VD" and re.match("_ZN(7product|4loss|10orthogonal)", t.split()[-1])}
    assert held and held == seen, sorted(held ^ seen)


def check_gpu_tests_reach_both_sides(c):
    sizes, tiles, joins = gpu_loss.SIZES + gpu_loss.LARGE, {}, set()
    pieces, ragged, few = set(), set(), set()
    for T, V, K in sizes:
        got = [kind(s) for call in (c.loss, c.grad) for s in c.of(call, T, V, K)]
        for name, ends, numbers in got:
            if name == "tiles_kernel":
                tiles.setdefault(ends[0], set()).add(numbers[2])
                few.add(ends[0] + str(numbers[-1]))
                ragged.update({ends[0] + str(numbers[3])} if len(numbers) > 4 else ())
        joins.add(any(name == "join_kernel" for name, _, _ in got))
        pieces.add(min(2, sum(ends == ["SoftmaxEnd"] for _, ends, _ in got)))
    assert tiles == {"StatsEnd": {1, 2, 4}, "SoftmaxEnd": {1, 2, 4}, "GradientEnd": {1, 2, 4}}, tiles
    assert joins == {False, True} and pieces == {1, 2} and ragged == {"StatsEnd0", "StatsEnd1", "SoftmaxEnd0", "SoftmaxEnd1"} and few == {"StatsEnd0", "SoftmaxEnd0", "SoftmaxEnd1", "GradientEnd0", "GradientEnd1"}, (joins, pieces, ragged, few)
    tiles, whole, slices, halves, joins, short, few = {}, set(), set(), set(), set(), set(), set()
    for rows, cols in gpu_orthogonal.SHAPES + gpu_orthogonal.LARGE:
        for call, how in ((c.orthogonalize, {"odt": BF16}), (c.orthogonalize, {"odt": F32}), (c.step, {})):
            got = [kind(s) for s in c.of(call, 1, rows, cols, **how)]
            grids = [t[0] for t in call(1, rows, cols, **how)[1]]
            for (name, ends, numbers), grid in zip(got, grids):
                if name in ("whole_kernel", "slice_kernel"):
                    (whole if name == "whole_kernel" else slices).add(numbers[0])
                elif name == "tiles_kernel":
                    tiles.setdefault(ends[0], set()).add(numbers[2])
                    few.add(numbers[-1])
                    side = -(-min(rows, cols) // (64 * numbers[2]))
                    if ends[0] != "UpdateEnd" and side > 1:
                        halves.add(grid < side * side)
            joins.add(any(name == "join_kernel" for name, _, _ in got))
            if min(rows, cols) <= 128 and max(rows, cols) > 320:
                short.add(any(name == "slice_kernel" for name, _, _ in got))
    assert few == {0, 1}, few
    assert whole == slices == {32, 64, 96, 128} and short == {True, False} and halves == {False, True} and joins == {False, True}, (whole, slices, short, halves, joins)
    assert all(t >= {1, 2} for t in tiles.values()) and len(tiles) == 3, tiles
    shorter = [min(s) for s in gpu_orthogonal.SHAPES + gpu_orthogonal.LARGE if min(s) > 128]
    assert any(s < 256 for s in shorter) and any(256 <= s < 512 for s in shorter) and any(512 <= s < 1024 for s in shorter) and any(s >= 1024 for s in shorter)


CHECKS = {f.__name__: f for f in (check_the_loss_is_refused, check_updates_are_refused, check_large_sizes_are_launched, check_every_kernel_is_reached, check_gpu_tests_reach_both_sides)}


@pytest.mark.parametrize("name", sorted(CHECKS))
def test_without_a_gpu(shim, name):  # noqa: F811
    r = subprocess.run([sys.executable, os.path.abspath(__file__), shim, name], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr


def test_the_binding_refuses_what_is_no_device_tensor():
    import torch

    import paper_1802_04434_amd as ss
    h, w, target, f = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(9, 64, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int64), torch.zeros(4)
    scratch = ss.new_cross_entropy_scratch(4, 9, 64, device="cpu")
    assert scratch.dtype == torch.uint8 and scratch.numel() == ss.load_library().ss_cross_entropy_scratch_bytes(4, 9, 64) > 0
    with pytest.raises(TypeError, match="h must live in device memory"):
        ss.cross_entropy(h, w, target, f, f, scratch)
    with pytest.raises(TypeError, match="h must live in device memory"):
        ss.cross_entropy_grad(h, w, target, f, None, h, w, scratch)
    with pytest.raises(TypeError, match="h must be a tensor"):
        ss.cross_entropy([1.0], w, target, f, f, scratch)
    scratch = ss.new_orthogonalize_scratch(4, 64, device="cpu")
    with pytest.raises(TypeError, match="g must live in device memory"):
        ss.orthogonalize(h, h, scratch)
    with pytest.raises(TypeError, match="g must live in device memory"):
        ss.orthogonal_step(h, f, 0.9, 0.1, f, scratch)


if __name__ == "__main__":
    CHECKS[sys.argv[2]](Calls(sys.argv[1]))
