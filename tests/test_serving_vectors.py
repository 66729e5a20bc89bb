"""Whether an output lies apart from its input in one buffer, on the host
(tests/serving_vectors.cpp compiled host-only against the library's own header)
against every pair of vectors."""
import itertools
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
D = 128


@pytest.fixture(scope="module")
def meet(tmp_path_factory):
    hipcc = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "bin", "hipcc")
    if not os.path.exists(hipcc):
        pytest.skip("hipcc not available")
    exe = tmp_path_factory.mktemp("vectors") / "serving_vectors"
    subprocess.run([hipcc, "-x", "hip", "--cuda-host-only", "-O1", "-std=c++17",
                    "-I", os.path.join(ROOT, "include"),
                    "-I", os.path.join(ROOT, "paper_2503_16428_amd", "csrc"),
                    os.path.join(ROOT, "tests", "serving_vectors.cpp"), "-o", str(exe)],
                   check=True, capture_output=True)

    def ask(cases):
        lines = "\n".join(" ".join(map(str, (a, *s, *n))) for a, s, n in cases)
        out = subprocess.run([str(exe)], input=lines, check=True, capture_output=True, text=True,
                             timeout=60).stdout.split()
        assert len(out) == len(cases)
        return [x == "1" for x in out]
    return ask


def really(apart, strides, sizes):
    steps = [[i * s for i in range(-n + 1, n)] for s, n in zip(strides, sizes)]
    return any(abs(apart - sum(t)) < D for t in itertools.product(*steps))


def test_every_distance(meet):
    rng = random.Random(7)
    cases = []
    for _ in range(60):
        sizes = [rng.choice([1, 1, 2, 3, 5]) for _ in range(3)]
        order, strides, span = rng.sample(range(3), 3), [0] * 3, D
        for i in order:  # nested, in any order of the dimensions
            if sizes[i] > 1:
                strides[i] = span + 8 * rng.choice([0, 0, 1, 16, 40])
                span += strides[i] * (sizes[i] - 1)
        most = span + 300
        cases += [(8 * a, strides, sizes) for a in range(-most // 8, most // 8 + 1,
                                                         max(1, most // 4000))]
    got = meet(cases)
    assert got == [really(*c) for c in cases]
    assert any(got) and not all(got)


def test_slices_of_a_projection(meet):
    """[batch, tokens, 12 heads, 128]: the first 4 heads and others beside and over them."""
    strides, sizes = (9 * 12 * D, D, 12 * D), (2, 4, 9)
    got = meet([(h * D, strides, sizes) for h in (-12, -8, -4, -3, 0, 1, 3, 4, 8, 9, 12)])
    assert got == [True, False, False, True, True, True, True, False, False, True, True]
    far = 1 << 40
    assert meet([(far, (far, 4 * D, D), (3, 4, 4)), (3 * far, (far, 4 * D, D), (3, 4, 4))]) == \
        [True, False]
