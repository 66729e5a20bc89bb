"""Places in the paged cache, on the host (tests/serve_check.cpp compiled
host-only against the library's own header): whatever a table, a length or a
start holds, a place lies inside the pool or is none."""
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
EDGES = [-2**31, -2**31 + 1, -1, 0, 1, 2, 15, 16, 17, 2**24, 2**31 - 2, 2**31 - 1]


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    hipcc = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "bin", "hipcc")
    if not os.path.exists(hipcc):
        pytest.skip("hipcc not available")
    exe = tmp_path_factory.mktemp("serve") / "serve_check"
    cmd = [hipcc, "-x", "hip", "--cuda-host-only", "-O1", "-std=c++17",
           "-I", os.path.join(ROOT, "include"),
           "-I", os.path.join(ROOT, "paper_2503_16428_amd", "csrc"),
           os.path.join(ROOT, "tests", "serve_check.cpp"), "-o", str(exe)]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr

    def run(lines):
        out = subprocess.run([str(exe)], input="\n".join(lines), capture_output=True, text=True,
                             timeout=60, check=True).stdout.split()
        assert len(out) == len(lines)
        return [int(x) for x in out]
    return run


def test_rows_lie_in_the_pool_or_are_none(ask):
    asked = [(e, pages, hkv, hkv - 1, shift, (1 << shift) - 1) for e in EDGES
             for pages in (1, 17, 2**31 - 1) for hkv in (1, 8) for shift in (4, 8)]
    got = ask(["row " + " ".join(map(str, a)) for a in asked])
    for (e, pages, hkv, h, shift, slot), r in zip(asked, got):
        want = ((e * hkv + h) << shift) + slot if 0 <= e < pages else -1
        assert r == want
        assert -1 <= r < (pages * hkv) << shift


def test_columns_and_lengths(ask):
    rng = random.Random(3)
    starts = EDGES + [rng.randrange(-2**31, 2**31) for _ in range(50)]
    asked = [(s + t, shift, n) for s in starts for t in (0, 1, 2**28) for shift in (4, 7)
             for n in (1, 5, 2**22)]
    got = ask(["column " + " ".join(map(str, a)) for a in asked])
    assert got == [t >> s if 0 <= t < n << s else -1 for t, s, n in asked]
    asked = [(n, c) for n in EDGES for c in (16, 2**30)]
    assert ask([f"len {n} {c}" for n, c in asked]) == [min(max(n, 0), c) for n, c in asked]
