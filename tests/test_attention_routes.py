"""Which way through the forward pass the batches of attention_routes reach, by the rule as it is compiled (CPU only)."""
import os
import shutil
import subprocess

import pytest

from attention_routes import ROUTES

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_12703_amd", "csrc")
MAIN = """
#include <cstdio>
#include "attention_rows.h"
using namespace ad;
int main() {
  AttnBatch b{};
  static const int some[2] = {};
  int window;
  while (scanf("%d %d %d %d %d %d %d", &b.batch, &b.heads, &b.kv_heads, &b.q_max, &b.k_max, &b.causal, &window) == 7) {
    b.window = window ? some : nullptr;
    const FwdPlan p = fwd_plan(b);
    if (p.keys) printf("keys\\n");
    else if (!p.few) printf("wide\\n");
    else printf("few%s %s\\n", p.splits > 1 ? " parts" : "", (p.splits > 1 ? p.chunk : b.k_max) > 128 ? "several" : "one");
  }
}
"""


def test_the_batches_reach_every_way(tmp_path):
    cxx = shutil.which("g++") or shutil.which("clang++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    (tmp_path / "way.cpp").write_text(MAIN)
    subprocess.run([cxx, "-O1", "-std=c++17", "-I", CSRC, str(tmp_path / "way.cpp"), "-o", str(tmp_path / "way")], check=True)
    text = "\n".join(" ".join(map(str, (len(a["ql"]), a.get("heads", 2), a.get("kv", 2), max(a["ql"]), max(a["kl"]),
                                        int(a.get("causal", False)), int("window" in a)))) for _, a in ROUTES.values())
    got = subprocess.run([str(tmp_path / "way")], input=text, capture_output=True, text=True, check=True).stdout.split("\n")[:-1]
    assert dict(zip(ROUTES, got)) == {name: way for name, (way, _) in ROUTES.items()}
    assert set(got) == {"keys", "few one", "few several", "few parts one", "few parts several", "wide"}
