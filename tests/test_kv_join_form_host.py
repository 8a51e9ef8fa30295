"""Which form of the join kernel a plan gets (paper_2609_33224_gb300/csrc/kv_plan.h): a warp an entry only where the entries
fill the GPU and have several rows each; with and without masked spans."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_33224_gb300", "csrc")

HARNESS = r"""
#include <cstdio>
#include "kv_plan.h"
using namespace pskv;
int main() {
  unsigned D, fmt, H, g, T, n;
  while (std::scanf("%u %u %u %u %u %u", &D, &fmt, &H, &g, &T, &n) == 6) {
    std::vector<ps_kv_span> sp(n);
    uint64_t blocks = 0;
    for (auto& s : sp) {
      unsigned a, b, c, d;
      if (std::scanf("%u %u %u %u", &a, &b, &c, &d) != 4) return 2;
      s = ps_kv_span{a, b, c, d, blocks};
      blocks += (c + 15) / 16;
    }
    Layout o;
    lay_out(PlanShape{152, D, (int)fmt, H, g}, T, sp.data(), n, &o);
    std::printf("%zu %u %u %d\n", o.join.size(), o.join_stride, o.join_parts,
                (int)join_by_entries((uint32_t)o.join.size(), o.join_stride, o.join_parts));
  }
}
"""


@pytest.fixture(scope="module")
def form(tmp_path_factory):
    d = tmp_path_factory.mktemp("join")
    src, exe = d / "p.cpp", d / "p"
    src.write_text(HARNESS)
    subprocess.run(["g++", "-std=c++17", "-O2", "-I", CSRC, "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)],
                   check=True)

    def run(H, g, requests, new, own, shared, kind=1):
        T = requests * new
        spans = ([(0, T, shared, 0)] if shared else []) + [(i * new, new, own + new, kind) for i in range(requests)]
        text = "128 0 %d %d %d %d\n" % (H, g, T, len(spans)) + "".join("%d %d %d %d\n" % s for s in spans)
        r = subprocess.run([str(exe)], input=text, capture_output=True, text=True, check=True)
        return [int(x) for x in r.stdout.split()]
    return run


@pytest.mark.parametrize("case", [(8, 8, 32, 16, 200, 4000), (8, 8, 1, 512, 2000, 0), (32, 2, 4, 200, 2000, 1000), (1, 64, 4, 200, 2000, 1000)])
def test_many_entries_of_several_rows(form, case):
    entries, stride, parts, by = form(*case)
    assert by and entries >= 2048 and stride > 1 and parts <= 8


@pytest.mark.parametrize("case", [
    # as many rows, but few entries of many rows each
    (1, 128, 10, 16, 100, 4000), (2, 64, 512, 1, 100, 2000), (8, 16, 10, 16, 100, 4000), (1, 128, 10, 16, 100, 4000, 2),
    # as many entries, but of one row each
    (32, 1, 60, 31, 400, 16384), (64, 1, 4, 200, 2000, 1000), (64, 1, 32, 16, 200, 4000, 2)])
def test_few_entries_and_entries_of_one_row(form, case):
    entries, stride, parts, by = form(*case)
    assert not by and entries * stride > 16384 and (entries < 2048 or stride == 1)
