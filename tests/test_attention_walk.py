"""The tiles of queries that a workgroup of keys walks over for dk and dv, by the rule as it is compiled (CPU only): all
that see one of its keys, and none where its keys are padding."""
import os
import random
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_12703_amd", "csrc")
MAIN = """
#include <cstdio>
#include <vector>
#include "attention_rows.h"
using namespace ad;
template <int TQ>
void walk(const AttnBatch& b, const Span& s, const int* ranges, int g, int k0, int k1) {
  Walk<TQ, const int*> w(b, s, ranges, g, k0, k1);
  while (w.settle()) {
    printf("%d %d ", w.h, w.t);
    ++w.t;
  }
  printf(";");
}
int main() {
  int tq, heads, kv, oq, ow, nq, nk, causal, window;
  while (scanf("%d %d %d %d %d %d %d %d %d", &tq, &heads, &kv, &oq, &ow, &nq, &nk, &causal, &window) == 9) {
    AttnBatch b{};
    const int cq[2] = {0, oq}, ck[2] = {0, ow};
    b.batch = 1; b.heads = heads; b.kv_heads = kv; b.group = heads / kv; b.q_rows = b.q_max = oq; b.k_rows = b.k_max = ow;
    b.causal = causal; b.cu_q = cq; b.cu_k = ck; b.q_len = &nq; b.k_len = &nk;
    std::vector<int> w, ranges;
    if (window) {
      w.resize(2 * oq);
      for (int& x : w) if (scanf("%d", &x) != 1) return 1;
      b.window = w.data();
    }
    const Span s = span_of(b, 0);
    for (int u = 0; 32 * u < nq; ++u) {      // as the kernel of dq leaves them
      Range r = {0x7fffffff, 0, 0, 0x7fffffff};
      for (int i = 32 * u; i < nq && i < 32 * u + 32; ++i) {
        const Keys k = keys_of(b, s, i);
        if (k.lo < k.hi) { r.lo = smaller(r.lo, k.lo); r.hi = larger(r.hi, k.hi); }
        r.all_lo = larger(r.all_lo, k.lo); r.all_hi = smaller(r.all_hi, k.hi);
      }
      for (int x : {r.lo, r.hi, r.all_lo, r.all_hi}) ranges.push_back(x);
    }
    const int width = tq == 64 ? 128 : 32;
    for (int g = 0; g < kv; ++g)
      for (int k0 = 0; k0 < ow; k0 += width) {
        const int k1 = smaller(k0 + width, nk);
        if (tq == 64) walk<64>(b, s, ranges.data(), g, k0, k1);
        else walk<128>(b, s, ranges.data(), g, k0, k1);
      }
    printf("\\n");
  }
}
"""


def test_the_tiles_that_see_the_keys(tmp_path):
    cxx = shutil.which("g++") or shutil.which("clang++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    (tmp_path / "walk.cpp").write_text(MAIN)
    subprocess.run([cxx, "-O1", "-std=c++17", "-I", CSRC, str(tmp_path / "walk.cpp"), "-o", str(tmp_path / "walk")], check=True)
    rng = random.Random(23)
    cases, lines = [], []
    for _ in range(600):
        kv = rng.choice([1, 2])
        oq, ow = rng.choice([0, 1, 31, 33, 128, 130, rng.randint(1, 300)]), rng.choice([1, 32, 128, 129, 500, rng.randint(1, 400)])
        nq, nk = rng.choice([oq, 0, rng.randint(0, oq)]), rng.choice([ow, 0, 1, rng.randint(0, ow)])
        c = dict(tq=rng.choice([64, 128]), heads=kv * rng.choice([1, 3]), kv=kv, oq=oq, ow=ow, nq=nq, nk=nk, causal=rng.randint(0, 1))
        w = [rng.choice([-2 ** 31, 2 ** 31 - 1, rng.randint(-5, ow + 5), rng.randint(-5, ow + 5)]) for _ in range(2 * oq)]
        c["w"] = w if rng.random() < 0.5 else None
        cases.append(c)
        lines.append(" ".join(map(str, [*list(c.values())[:8], int(c["w"] is not None), *(c["w"] or [])])))
    said = subprocess.run([str(tmp_path / "walk")], input="\n".join(lines), capture_output=True, text=True, check=True).stdout.split("\n")
    padding = 0
    for c, line in zip(cases, said):
        tq, n, nq, nk = c["tq"], c["heads"] // c["kv"], c["nq"], c["nk"]
        width = 128 if tq == 64 else 32
        places = [(g, k0) for g in range(c["kv"]) for k0 in range(0, c["ow"], width)]
        walks = line.split(";")[:-1]
        assert len(walks) == len(places)
        ends = []
        for i in range(nq):
            lo, hi = (0, nk) if c["w"] is None else (max(c["w"][2 * i], 0), min(c["w"][2 * i + 1], nk))
            ends.append((lo, min(hi, i + nk - nq + 1) if c["causal"] else hi))
        for (g, k0), walk in zip(places, walks):
            v = list(map(int, walk.split()))
            steps = list(zip(v[::2], v[1::2]))
            k1 = min(k0 + width, nk)
            need = {i // tq for i, (lo, hi) in enumerate(ends) if max(lo, k0) < min(hi, k1)}
            assert steps == sorted(set(steps)) and {h for h, _ in steps} <= set(range(g * n, g * n + n))
            for h in range(g * n, g * n + n):
                tiles = [t for x, t in steps if x == h]
                assert need <= set(tiles) <= set(range(-(-nq // tq))), (c, g, k0)
            if k0 >= nk:
                padding += 1
                assert not steps, (c, g, k0)
    assert padding > 300
