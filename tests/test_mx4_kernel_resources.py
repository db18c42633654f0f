"""Registers and LDS of the microscaled products' tiles: two waves of a SIMD
share its registers, and a tile that holds more of either runs alone or spills."""
import os
import re
import shutil
import subprocess

import pytest

import paper_2109_12497_amd as uq

READELF = shutil.which("llvm-readelf") or "/opt/rocm/llvm/bin/llvm-readelf"


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """{mangled name: (vector registers, LDS bytes, scratch bytes)} of the 4-bit kernels."""
    if not os.path.exists(READELF):
        pytest.skip("llvm-readelf is not installed")
    blob = open(uq.LIB_PATH, "rb").read()
    out, tmp = {}, tmp_path_factory.mktemp("co")
    for n, m in enumerate(re.finditer(b"\x7fELF", blob)):
        at = m.start()
        if int.from_bytes(blob[at + 18:at + 20], "little") != 224:  # EM_AMDGPU
            continue
        f = tmp / f"{n}.co"
        f.write_bytes(blob[at:])
        notes = subprocess.run([READELF, "--notes", str(f)], capture_output=True, text=True, check=True).stdout
        for block in notes.split("- .agpr_count:")[1:]:
            name = re.search(r"\.name:\s+(\S+)", block).group(1)
            if "k_mx4" in name:
                field = lambda key: int(re.search(rf"\.{key}:\s+(\d+)", block).group(1))  # noqa: E731
                out[name] = (int(block.split()[0]) + field("vgpr_count"), field("group_segment_fixed_size"),
                             field("private_segment_fixed_size"))
    assert out, "no 4-bit kernels found in libuq.so"
    return out


def test_no_kernel_uses_scratch(kernels):
    assert not {n: r for n, r in kernels.items() if r[2]}


# <type, waves down, across, fragments down, across, stages>: waves on a SIMD
# where the tile is alone on its compute unit or, of 81,920 bytes, twice there
@pytest.mark.parametrize("tile,lds", [("Li2ELi4ELi4ELi2ELi2E", 163840), ("Li2ELi4ELi2ELi1ELi4E", 163840),
                                      ("Li2ELi2ELi2ELi2ELi2E", 81920), ("Li2ELi2ELi1ELi2ELi4E", 163840)])
def test_tiles_fit_their_compute_unit(kernels, tile, lds):
    of = {n: r for n, r in kernels.items() if re.search(rf"k_mx4_tilesILi\dE{tile}EEvNS", n)}
    assert len(of) == 3
    assert all(r[0] <= 256 and r[1] <= lds for r in of.values()), of
