"""What a query's window leaves visible, by the mask that the kernels apply to a tile, as compiled (CPU only, signed
arithmetic left to the compiler): windows are any integers, and keys outside the sequence are never seen."""
import os
import random
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_12703_amd", "csrc")
MAIN = """
#include <cstdio>
#include "attention_rows.h"
using namespace ad;
int main() {
  int nq, nk, i, causal, lo, hi, first;
  while (scanf("%d %d %d %d %d %d %d", &nq, &nk, &i, &causal, &lo, &hi, &first) == 7) {
    AttnBatch b{};
    const int cq[2] = {0, nq}, ck[2] = {0, nk};
    b.batch = 1; b.q_rows = b.q_max = nq; b.k_rows = b.k_max = nk; b.causal = causal;
    b.cu_q = cq; b.cu_k = ck;
    int window[2 * 64] = {};
    window[2 * i] = lo;
    window[2 * i + 1] = hi;
    b.window = window;
    const Mask m = mask_of(keys_of(b, span_of(b, 0), i), first);
    for (int e = 0; e < 128; ++e) putchar(shows(m, e) ? '1' : '0');
    putchar(10);
  }
}
"""
LOW, HIGH = -2 ** 31, 2 ** 31 - 1


@pytest.mark.parametrize("opt", ["-O0", "-O2"])
def test_a_tile_shows_what_the_window_says(opt, tmp_path):
    cxx = shutil.which("g++") or shutil.which("clang++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    (tmp_path / "mask.cpp").write_text(MAIN)
    subprocess.run([cxx, opt, "-std=c++17", "-I", CSRC, str(tmp_path / "mask.cpp"), "-o", str(tmp_path / "mask")], check=True)
    rng = random.Random(17)
    ends = [LOW, LOW + 1, -(1 << 30), -1, 0, 1, 5, 60, 127, 199, 200, 201, 1 << 30, HIGH - 1, HIGH]
    cases = [(200, 200, 7, 0, lo, hi, first) for lo in ends for hi in ends for first in (0, 68, 128, 256)]
    for _ in range(3000):
        nq, nk = rng.randint(1, 40), rng.randint(0, 300)
        end = lambda: rng.choice([rng.choice(ends), rng.randint(-3, 310)])  # noqa: E731
        cases.append((nq, nk, rng.randrange(nq), rng.randint(0, 1), end(), end(), rng.randint(0, 80) * 4))
    text = "\n".join(" ".join(map(str, c)) for c in cases)
    got = subprocess.run([str(tmp_path / "mask")], input=text, capture_output=True, text=True, check=True).stdout.split()
    assert len(got) == len(cases)
    for (nq, nk, i, causal, lo, hi, first), line in zip(cases, got):
        want = "".join("01"[lo <= j < hi and j < nk and not (causal and j > i + nk - nq)] for j in range(first, first + 128))
        assert line == want, (nq, nk, i, causal, lo, hi, first)
