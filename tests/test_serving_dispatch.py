"""The decode's number of workgroups, on the host (tests/serving_dispatch.cpp compiled
host-only against the library's own header), against what the built kernels leave
room for on a compute unit."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2503_16428_amd import build as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")
LLVM = os.path.join(ROCM, "llvm", "bin")
CUS, LDS, LANE_REGISTERS, SIMDS = 256, 160 * 1024, 512, 4


@pytest.fixture(scope="module")
def workers(tmp_path_factory):
    hipcc = os.path.join(ROCM, "bin", "hipcc")
    if not os.path.exists(hipcc):
        pytest.skip("hipcc not available")
    exe = tmp_path_factory.mktemp("serving") / "serving_dispatch"
    subprocess.run([hipcc, "-x", "hip", "--cuda-host-only", "-O1", "-std=c++17",
                    "-I", os.path.join(ROOT, "include"),
                    "-I", os.path.join(ROOT, "paper_2503_16428_amd", "csrc"),
                    os.path.join(ROOT, "tests", "serving_dispatch.cpp"), "-o", str(exe)],
                   check=True, capture_output=True)

    def ask(rows, two_tiles):
        out = subprocess.run([str(exe)], input=f"workers {rows} {int(two_tiles)}", check=True,
                             capture_output=True, text=True, timeout=60).stdout
        return int(out)
    return ask


@pytest.fixture(scope="module")
def resident(tmp_path_factory):
    """Workgroups that a compute unit holds of the decode kernels that share out work, least of
    both cache types: {two_tiles: number}, by local memory and registers."""
    if not os.path.exists(os.path.join(LLVM, "llvm-objdump")):
        pytest.skip("llvm-objdump not available")
    tmp = tmp_path_factory.mktemp("kernels")
    shutil.copy(B.LIB, tmp / "lib.so")
    subprocess.run([os.path.join(LLVM, "llvm-objdump"), "--offloading", "lib.so"], cwd=tmp,
                   check=True, capture_output=True)
    least = {}
    for f in sorted(tmp.glob("*gfx950*")):
        notes = subprocess.run([os.path.join(LLVM, "llvm-readelf"), "--notes", str(f)], check=True,
                               capture_output=True, text=True).stdout
        for k in notes.split("- .agpr_count:")[1:]:
            name = re.search(r"\.name: +(\S+)", k)[1]
            tiles = re.search(r"decode_kernelILb[01]ELi([12])ELb0E", name)
            if not tiles:
                continue
            lds, vgprs = (int(re.search(rf"\.{n}: +(\d+)", k)[1])
                          for n in ("group_segment_fixed_size", "vgpr_count"))
            waves = LANE_REGISTERS // (-(-vgprs // 8) * 8)  # of a SIMD; a workgroup has one on each
            two = tiles[1] == "2"
            least[two] = min(least.get(two, 99), LDS // lds, waves)
    assert set(least) == {False, True}
    return least


@pytest.mark.parametrize("two_tiles", [False, True])
@pytest.mark.parametrize("rows", [1, 8, 511, 512, 600, 1024, 1 << 20])
def test_every_workgroup_of_a_decode_is_resident(workers, resident, rows, two_tiles):
    n = workers(rows, two_tiles)
    assert n % CUS == 0 and 2 * CUS <= n <= resident[two_tiles] * CUS


def test_many_rows_of_one_tile_have_three_a_unit(workers):
    assert [workers(r, False) for r in (511, 512)] == [512, 768]
