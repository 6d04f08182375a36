"""Which kernel the sizes of tests/linear_kernels.py reach, by the rules as they are compiled (CPU only)."""
import os
import shutil
import subprocess

import pytest

import linear_kernels as sizes

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_12703_amd", "csrc")
MAIN = """
#include <cstdio>
#include "linear_plan.h"
int main() {
  int P, Q, K, direct, ckpt, few;
  while (scanf("%d %d %d %d %d %d", &P, &Q, &K, &direct, &ckpt, &few) == 6) {
    const ad::Plan r = ad::plan(P, Q, K, direct, ckpt);
    const ad::FewPlan f = ad::few_plan(P, Q, K);
    if (few && Q <= ad::kFewRows && ad::few_wins(f, r, P, K)) {
      printf("few%dx%d\\n", Q <= 16 ? 1 : 2, f.narrow ? 8 : 16);
      continue;
    }
    const char* tile = !direct ? "any" : r.deep ? "deep" : r.tile == 256 ? "256" : "128";
    const size_t need = r.S > 1 ? 4 * ad::part_floats(r) : 0;
    if ((need > 0) != (r.S > 1) || need > 4 * ad::plan_floats(ckpt, P, Q, K)) printf("workspace! ");
    printf("%s%c%d\\n", tile, r.S > 1 && r.whole > 0 ? '+' : '/', r.S);
  }
}
"""


@pytest.fixture(scope="module")
def choose(tmp_path_factory):
    cxx = shutil.which("g++") or shutil.which("clang++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    d = tmp_path_factory.mktemp("plan")
    (d / "plan.cpp").write_text(MAIN)
    subprocess.run([cxx, "-O1", "-std=c++17", "-I", CSRC, str(d / "plan.cpp"), "-o", str(d / "plan")], check=True)

    def run(cases):
        """cases: (P, Q, K, direct, from a checkpoint, forward without one) -> the kernel of each."""
        text = "\n".join(" ".join(str(int(v)) for v in c) for c in cases)
        return subprocess.run([str(d / "plan")], input=text, capture_output=True, text=True, check=True).stdout.split("\n")[:-1]

    return run


def test_tiles_of_256(choose):
    for table, kinds in ((sizes.TILES_256, (0,)), (sizes.WGRAD_256, (0, 1)), (sizes.WGRAD_256_BF16, (0,)),
                         (sizes.WGRAD_256_CKPT, (1,))):
        for ckpt in kinds:
            assert choose([(P, Q, K, 1, ckpt, 0) for P, Q, K, *_ in table]) == [t[-1] for t in table]
        assert all(P % 8 == 0 and pad % 8 == 0 and shift % 8 == 0 for P, _, _, pad, shift, _ in table)
    seen = {t[-1][:4] for t in sizes.TILES_256}
    assert {"256/", "256+"} <= seen


def test_tiles_of_128(choose):
    assert choose([(P, Q, K, 1, 0, 0) for P, Q, K, *_ in sizes.TILES_128]) == [t[-1] for t in sizes.TILES_128]
    assert all(P % 8 == 0 and K % 8 == 0 and pad % 8 == 0 for P, _, K, pad, *_ in sizes.TILES_128)


def test_few_rows(choose):
    assert choose([(n, rows, k, 1, 0, 1) for rows, n, k, *_ in sizes.FEW]) == [t[-1] for t in sizes.FEW]
    assert {"few1x8", "few1x16", "few2x8", "few2x16"} <= {t[-1] for t in sizes.FEW}


def test_any_alignment_in_parts(choose):
    assert choose([(n, rows, k, 0, 0, 0) for rows, n, k, *_ in sizes.ANY_FWD]) == [t[-1] for t in sizes.ANY_FWD]
    assert choose([(k, rows, n, 0, 0, 0) for rows, n, k, *_ in sizes.ANY_DGRAD]) == [t[-1] for t in sizes.ANY_DGRAD]
    for ckpt, table in ((0, sizes.ANY_WGRAD), (1, sizes.ANY_WGRAD_CKPT)):
        assert choose([(k, n, rows, 0, ckpt, 0) for rows, n, k, *_ in table]) == [t[-1] for t in table]


def test_numbers_of_steps(choose):
    for direct, ckpt in ((1, 0), (1, 1), (0, 0), (0, 1)):
        got = choose([(136, 40, K, direct, ckpt, 0) for K in sizes.STEPS])
        assert all(g.endswith("/1") for g in got[:7]) and all(int(g.split("/")[1]) > 1 for g in got[7:]), got
