"""The tables of an attention batch and its cut into workgroups, by the rules as they are compiled (CPU only): what a
table entry out of range does, that no row outside the matrices is ever named, and what the workspace has to hold."""
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
static int next() { int v; if (scanf("%d", &v) != 1) v = 0; return v; }
static std::vector<int> list(int n) { std::vector<int> v(n); for (int& x : v) x = next(); return v; }
int main() {
  char what;
  while (scanf(" %c", &what) == 1) {
    AttnBatch b{};
    b.batch = next(); b.heads = next(); b.kv_heads = next(); b.q_rows = next(); b.k_rows = next();
    b.q_max = next(); b.k_max = next(); b.causal = next();
    static const int some[2] = {0, 0};
    if (what == 'p') {
      if (next()) b.window = some;
      const FwdPlan p = fwd_plan(b);
      printf("%d %d %d %d %d %zu %zu %d\\n", p.few, p.tiles, p.splits, p.chunk, wide_rows(b, b.k_max, b.kv_heads, true),
             attn_fwd_bytes(b), attn_bwd_bytes(b), attn_fits(b));
      continue;
    }
    if (what == 'f') {
      printf("%d\\n", first_piece(b.q_rows, b.k_rows, b.batch));
      continue;
    }
    if (what == 'd') {
      int bad = 0;
      const uint64_t m = per(b.batch);
      for (uint64_t n = 0; n < (1 << 24); n += 1 + n / 4096)
        for (uint64_t k : {n / b.batch * b.batch, n / b.batch * b.batch + b.batch - 1, n})
          bad += k < (1 << 24) && (k * m) >> kPerShift != k / b.batch;
      printf("%d\\n", bad);
      continue;
    }
    const int padded = next(), window = next();
    const auto cq = list(b.batch + 1), ck = list(b.batch + 1);
    std::vector<int> ql, kl, w;
    if (padded) { ql = list(b.batch); kl = list(b.batch); b.q_len = ql.data(); b.k_len = kl.data(); }
    if (window) { w = list(2 * b.q_rows); b.window = w.data(); }
    b.cu_q = cq.data(); b.cu_k = ck.data();
    for (int i = 0; i < b.batch; ++i) {
      const Span s = span_of(b, i);
      printf("%d", s.ok);
      if (s.ok) {
        printf(" %d %d %d %d %d %d", s.q0, s.nq, s.oq, s.k0, s.nk, s.ow);
        for (int r = 0; r < s.nq; ++r) { const Keys k = keys_of(b, s, r); printf(" %d %d", k.lo, k.hi); }
      }
      printf(";");
    }
    printf("\\n");
  }
}
"""


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    cxx = shutil.which("g++") or shutil.which("clang++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    d = tmp_path_factory.mktemp("rows")
    (d / "rows.cpp").write_text(MAIN)
    subprocess.run([cxx, "-O1", "-fwrapv", "-std=c++17", "-I", CSRC, str(d / "rows.cpp"), "-o", str(d / "rows")], check=True)

    def run(lines):
        text = "\n".join(" ".join(map(str, x)) for x in lines)
        return subprocess.run([str(d / "rows")], input=text, capture_output=True, text=True, check=True).stdout.split("\n")[:-1]

    return run


def _case(rng):
    batch = rng.randint(1, 5)
    rows_q, rows_k = rng.randint(0, 40), rng.randint(0, 60)
    q_max, k_max = rng.choice([rows_q, rng.randint(0, 40)]), rng.choice([rows_k, rng.randint(0, 60)])

    def cu(rows):
        v = sorted(rng.randint(0, rows) for _ in range(batch + 1))
        for _ in range(rng.choice([0, 0, 1, 2])):
            v[rng.randrange(batch + 1)] = rng.choice([-1, rows + 1, 2 ** 31 - 1, -2 ** 31, rng.randint(0, rows)])
        return v

    cq, ck = cu(rows_q), cu(rows_k)
    padded, causal, window = rng.random() < 0.5, rng.random() < 0.5, rng.random() < 0.4
    lens = lambda v: [rng.choice([max(0, min(v[i + 1] - v[i], rng.randint(0, 60))), -1, 2 ** 31 - 1, rng.randint(0, 40)])  # noqa: E731
                      if rng.random() < 0.4 else max(0, min(v[i + 1] - v[i], 60)) for i in range(batch)]
    ql, kl = (lens(cq), lens(ck)) if padded else (None, None)
    w = [rng.choice([rng.randint(-5, 70), -2 ** 31, 2 ** 31 - 1]) for _ in range(2 * rows_q)] if window else None
    return dict(batch=batch, rows_q=rows_q, rows_k=rows_k, q_max=q_max, k_max=k_max, cq=cq, ck=ck, ql=ql, kl=kl, w=w, causal=causal)


def test_spans_stay_inside(ask):
    rng = random.Random(5)
    cases = [_case(rng) for _ in range(4000)]
    lines = [["t", c["batch"], 2, 1, c["rows_q"], c["rows_k"], c["q_max"], c["k_max"], int(c["causal"]), int(c["ql"] is not None),
              int(c["w"] is not None), *c["cq"], *c["ck"], *(c["ql"] or []), *(c["kl"] or []), *(c["w"] or [])] for c in cases]
    good = bad = 0
    for c, line in zip(cases, ask(lines)):
        for b, said in enumerate(line.split(";")[:-1]):
            v = list(map(int, said.split()))
            q0, q1, k0, k1 = c["cq"][b], c["cq"][b + 1], c["ck"][b], c["ck"][b + 1]
            nq, nk = (c["ql"][b], c["kl"][b]) if c["ql"] is not None else (q1 - q0, k1 - k0)
            ok = (0 <= q0 <= q1 <= c["rows_q"] and 0 <= k0 <= k1 <= c["rows_k"] and q1 - q0 <= c["q_max"]
                  and k1 - k0 <= c["k_max"] and 0 <= nq <= q1 - q0 and 0 <= nk <= k1 - k0)
            assert v[0] == int(ok)
            if not ok:
                bad += 1
                continue
            good += 1
            assert v[1:7] == [q0, nq, q1 - q0, k0, nk, k1 - k0]
            for i in range(nq):
                lo, hi = v[7 + 2 * i], v[8 + 2 * i]
                want = set(range(nk))
                if c["causal"]:
                    want = {j for j in want if j <= i + nk - nq}
                if c["w"] is not None:
                    a, e = c["w"][2 * (q0 + i)], c["w"][2 * (q0 + i) + 1]
                    want = {j for j in want if a <= j < e}
                assert set(range(lo, hi)) == want and lo >= 0 and hi <= nk
    assert good > 2000 and bad > 2000


def test_plans(ask):
    rng = random.Random(6)
    shapes = [(b, h, kv, q, k, w) for b, h, kv, q, k, w in (
        (1, 20, 20, 1, 1500, 0), (32, 20, 20, 1, 1500, 0), (32, 20, 20, 448, 1500, 0), (12, 20, 20, 128, 128, 0),
        (1, 1, 1, 1, 1 << 24, 0), (1, 12, 12, 5000, 5000, 0), (12, 20, 5, 131, 1500, 1), (65535, 1, 1, 1, 1, 0), (1, 1, 1, 0, 0, 0),
        (0, 1, 1, 4, 4, 0), (3, 2, 1, 33, 0, 0))]
    for _ in range(3000):
        kv = rng.choice([1, 2, 5, 20])
        shapes.append((rng.randint(0, 40), kv * rng.choice([1, 2, 4]), kv, int(2 ** rng.uniform(0, 14)), int(2 ** rng.uniform(0, 16)),
                       rng.randint(0, 1)))
    lines = [["p", b, h, kv, b * q, b * k, q, k, 0, w] for b, h, kv, q, k, w in shapes]
    kinds = set()
    for (b, h, kv, q, k, w), line in zip(shapes, ask(lines)):
        few, tiles, splits, chunk, wide_k, fwd, bwd, fits = map(int, line.split())
        assert fits == (b * h <= 65535 * 8)
        if not b or not q:
            assert fwd == 0
            continue
        assert tiles == -(-q // (32 if few else 128))
        assert 1 <= splits <= 64                       # (a wave joins them, a lane a part)
        if splits > 1:
            assert few and chunk % 128 == 0 and splits * chunk >= k and (splits - 1) * chunk < k
            assert b * h * tiles * splits <= 512 + b * h * tiles
        assert fwd == (4 * 66 * splits * h * b * q if splits > 1 else 0)
        # what 32 queries see together, behind a float for each row and head
        assert bwd >= 4 * h * b * q + 16 * b * -(-q // 32)
        kinds.add((few, splits > 1, wide_k))
    assert len(kinds) >= 5


def test_quotients(ask):
    divisors = [1, 2, 3, 5, 6, 7, 12, 20, 61, 127, 641, 1000, 4095, 6700, 16383, 16384]
    assert ask([["d", d, 1, 1, 0, 0, 0, 0, 0] for d in divisors]) == ["0"] * len(divisors)


def test_first_piece(ask):
    """Pieces of 32 keys in turn: they cover what is visible, and none begins where nothing is."""
    none = 2 ** 31 - 1
    cases = [(w, lo, hi) for lo, hi in ((none, 0), (0, 0), (0, 1), (31, 33), (32, 64), (1499, 1500), (none, none)) for w in range(8)]
    got = [int(x) for x in ask([["f", w, 1, 1, lo, hi, 0, 0, 0] for w, lo, hi in cases if hi < none])]
    for (w, lo, hi), at in zip(cases, got):
        assert at == (min(lo, hi) // 32 + w) * 32 and (lo < hi or at >= hi)
