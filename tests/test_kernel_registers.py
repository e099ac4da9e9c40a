"""Registers of the built kernels that share a compute unit by eight blocks, from the notes that the compiler leaves in the library's code objects."""
import os
import re
import struct
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
READELF = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin", "llvm-readelf")
MAGIC = b"__CLANG_OFFLOAD_BUNDLE__"


def code_objects(data):
    """the gfx950 entries of the bundles, one of each source file"""
    at = data.find(MAGIC)
    while at >= 0:
        count, = struct.unpack_from("<Q", data, at + len(MAGIC))
        p = at + len(MAGIC) + 8
        for _ in range(count):
            start, size, length = struct.unpack_from("<QQQ", data, p)
            if data[p + 24:p + 24 + length].endswith(b"gfx950"):
                yield data[at + start:at + start + size]
            p += 24 + length
        at = data.find(MAGIC, p)


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    if not os.path.exists(READELF):
        pytest.skip("no llvm-readelf")
    with open(os.path.join(ROOT, "paper_1802_04434_amd", "libsignsgd.so"), "rb") as f:
        objects = list(code_objects(f.read()))
    found, at = {}, tmp_path_factory.mktemp("objects") / "code"
    for o in objects:
        at.write_bytes(o)
        notes = subprocess.run([READELF, "--notes", str(at)], capture_output=True, text=True, check=True).stdout
        for kernel in notes.split("- .agpr_count:")[1:]:
            fields = dict(re.findall(r"\.(\w+): +(\S+)", kernel))
            found[fields["name"]] = {k: int(fields[k]) for k in ("vgpr_count", "vgpr_spill_count", "group_segment_fixed_size")}
    return found


def test_kernels_of_a_few_steps_leave_room_for_eight_blocks(kernels):
    """of 256 threads on a compute unit: an eighth of a lane's 512 registers and of 160 KB of LDS, and nothing spilled"""
    short = {n: k for n, k in kernels.items() if "tiles_kernel" in n and "Lb1EEEvNS_9TilesArgs" in n}
    ends = {re.search(r"\d([A-Z][a-z]+End)(ILb[01])?", n).group(0)[1:] for n in short}
    assert ends == {"SoftmaxEndILb0", "SoftmaxEndILb1", "GradientEnd", "SquareEnd", "PolynomialEnd", "UpdateEnd"}, ends
    for name, k in short.items():
        assert k["vgpr_count"] <= 64 and k["vgpr_spill_count"] == 0 and 8 * k["group_segment_fixed_size"] <= 160 << 10, (name, k)


def test_no_product_keeps_sums_in_memory(kernels):
    tiles = {n: k for n, k in kernels.items() if "tiles_kernel" in n}
    assert len(tiles) > 20 and not [n for n, k in tiles.items() if k["vgpr_spill_count"]]
