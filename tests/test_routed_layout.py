"""Sizes of the routed calls' workspace, by the functions of routed.h themselves: compiled for
the host and compared with groups laid out one by one."""
import os
import shutil
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CODE = """
#include "routed.h"
#include <cstdio>
int main() {
  long long R, groups, widest, N;
  while (std::scanf("%lld %lld %lld %lld", &R, &groups, &widest, &N) == 4) {
    const long long P = pmlpk::rt_places(R, groups);
    std::printf("%lld %lld\\n", P, (long long)pmlpk::rt_hidden(R, P, widest, N));
  }
}
"""


@pytest.fixture(scope="module")
def sizes(tmp_path_factory):
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    if not shutil.which("g++") or not os.path.exists(os.path.join(rocm, "include", "hip", "hip_runtime.h")):
        pytest.skip("needs g++ and the HIP headers")
    folder = tmp_path_factory.mktemp("layout")
    source, program = str(folder / "sizes.cpp"), str(folder / "sizes")
    with open(source, "w") as f:
        f.write(CODE)
    subprocess.run(["g++", "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(rocm, "include"),
                    "-I", os.path.join(ROOT, "include"),
                    "-I", os.path.join(ROOT, "paper_2206_08369_amd", "csrc"), source, "-o", program],
                   check=True, timeout=120)

    def ask(rows):
        text = "".join("%d %d %d %d\n" % tuple(r) for r in rows)
        out = subprocess.run([program], input=text, capture_output=True, text=True, check=True).stdout
        return [tuple(map(int, l.split())) for l in out.splitlines()]

    return ask


def test_places_and_hidden_values_suffice(sizes):
    rng = np.random.default_rng(1)
    rows, used = [], []
    for _ in range(300):
        M, R = int(rng.integers(1, 40)), int(rng.integers(1, 500))
        hs = rng.integers(1, 9, M)
        hs[rng.integers(0, M)] = rng.integers(1, 2000)
        n = np.bincount(rng.choice(M, R, p=rng.dirichlet(np.full(M, 0.3))), minlength=M)
        padded = (n + 31) // 32 * 32
        rows.append((R, min(M, R), hs.max(), hs.sum()))
        used.append((padded.sum(), (padded * hs).sum()))
    for row, (places, hidden), (P, H) in zip(rows, used, sizes(rows)):
        assert places <= P and hidden <= H, row


def test_rows_of_places_are_aligned(sizes):
    """Output gradients by place are [O][P] floats, read four at a time."""
    rows = [(R, g, 1, 1) for R in range(1, 200) for g in (1, 2, 3, 7, 64) if g <= R]
    assert all(P % 32 == 0 for P, _ in sizes(rows))


def test_one_wide_model_does_not_widen_the_others_padding(sizes):
    # 5,999 models of 1 to 9 units and one of 1,000, 32,768 slots
    N = sum(1 + m % 9 for m in range(5999)) + 1000
    (P, H), = sizes([(32768, 6000, 1000, N)])
    assert H <= 1000 * 32768 + 31 * N
