"""How many tensors a launch of the optimizer takes, by the rule as it is compiled (CPU only: sizes alone), and the
largest tensor: a launch of 256 threads a workgroup takes under 2^24 workgroups."""
import ctypes
import os
import random
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_12703_amd", "csrc")
MAIN = """
#include <cstdio>
#include <vector>
#include "opt_launch.h"
int main() {
  int count;
  while (scanf("%d", &count) == 1) {
    std::vector<long long> size(count);
    for (auto& n : size) if (scanf("%lld", &n) != 1) return 1;
    for (int i = 0; i < count;) {
      int places[ad::kOptTensors], n;
      i = ad::opt_launch([&](int k) { return (int64_t)size[k]; }, count, i, places, n);
      for (int k = 0; k < n; ++k) printf("%d ", places[k]);
      if (n) printf("; ");
    }
    printf("\\n");
  }
}
"""
CHUNK, MOST = 8192, (1 << 37) - 8192
P = 0x100000            # an address that is never dereferenced


def test_a_launch_has_the_workgroups_that_it_may_have(tmp_path):
    cxx = shutil.which("g++") or shutil.which("clang++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    (tmp_path / "cut.cpp").write_text(MAIN)
    subprocess.run([cxx, "-O1", "-std=c++17", "-I", CSRC, str(tmp_path / "cut.cpp"), "-o", str(tmp_path / "cut")], check=True)
    rng = random.Random(3)
    lists = [[MOST], [MOST, 1], [1, MOST, 1], [MOST] * 3, [1 << 36, (1 << 36) - 8192], [1 << 36, 1 << 36], [0] * 50, [], [1] * 100,
             [0, 5, 0, 0, 7, 0]]
    for _ in range(500):
        lists.append([rng.choice([0, 1, rng.randint(1, 10 ** 6), int(2 ** rng.uniform(20, 37)) - CHUNK]) for _ in range(rng.randint(0, 120))])
    lists = [[min(n, MOST) for n in x] for x in lists]
    text = "\n".join(" ".join(map(str, [len(x)] + x)) for x in lists)
    lines = subprocess.run([str(tmp_path / "cut")], input=text, capture_output=True, text=True, check=True).stdout.split("\n")[:-1]
    assert len(lines) == len(lists)
    for sizes, line in zip(lists, lines):
        launches = [list(map(int, part.split())) for part in line.split(";")[:-1]]
        assert [i for x in launches for i in x] == [i for i, n in enumerate(sizes) if n]       # each once, in order
        groups = [[-(-sizes[i] // CHUNK) for i in x] for x in launches]
        assert all(sum(x) * 256 < 1 << 32 and len(x) <= 40 for x in groups)
        # and none ends before it is full
        assert all(sum(a) + b[0] > (1 << 24) - 1 or len(a) == 40 for a, b in zip(groups, groups[1:]))


def test_larger_tensors_are_refused():
    from paper_2608_12703_amd import ad
    n = ctypes.c_size_t()
    tensor = lambda size: (ad.OptTensor * 1)(ad.OptTensor(size, P, None, P, P, P, None, None, 0.0, 0, 0, 0))  # noqa: E731
    assert ad.LIB.ad_grad_norm_workspace_size(tensor(MOST), 1, ctypes.byref(n)) == 0 and n.value >= 8 * (MOST // CHUNK)
    args = ctypes.byref(ad.AdamwArgs(1e-3, 0.9, 0.999, 1e-8, 1, 0, None, None, None))
    for size in (MOST + 1, 1 << 38, 1 << 40):
        assert ad.LIB.ad_adamw(tensor(size), 1, args, None) == -2
        assert ad.LIB.ad_opt_state(tensor(size), 1, P, P, None) == -2
        assert ad.LIB.ad_grad_norm_workspace_size(tensor(size), 1, ctypes.byref(n)) == -2
        assert ad.LIB.ad_grad_norm(tensor(size), 1, 1.0, P, None, P, 1 << 62, None) == -2
