"""The plan's join (paper_2609_33224_gb300/csrc/kv_plan.h): its kernel gets a row per (query, head), hardly more, also where
the heads of a group are cut by many tiles."""
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
    unsigned long long exact = 0, gaps = 0;
    unsigned most = 0;
    for (const JoinEntry& e : o.join) {
      exact += e.count;
      most = std::max<unsigned>(most, e.count);
      // an entry's heads share a key/value head
      if ((unsigned)e.head0 + e.count > H * g || e.head0 / g != (e.head0 + e.count - 1) / g) ++gaps;
    }
    std::printf("%llu %llu %u %u %llu\n", exact, join_rows(o), o.join_stride, most, gaps);
  }
}
"""


@pytest.fixture(scope="module")
def rows(tmp_path_factory):
    d = tmp_path_factory.mktemp("join")
    src, exe = d / "p.cpp", d / "p"
    src.write_text(HARNESS)
    subprocess.run(["g++", "-std=c++17", "-O2", "-I", CSRC, "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)],
                   check=True)

    def run(D, fmt, H, g, T, spans):
        text = "%d %d %d %d %d %d\n" % (D, fmt, H, g, T, len(spans)) + "".join("%d %d %d %d\n" % s for s in spans)
        r = subprocess.run([str(exe)], input=text, capture_output=True, text=True)
        assert r.returncode == 0
        return [int(x) for x in r.stdout.split()]
    return run


@pytest.mark.parametrize("H,g,T", [(1, 128, 64), (8, 8, 64), (2, 64, 40), (1, 4096, 300), (1, 65535, 17), (1, 33, 50)])
@pytest.mark.parametrize("empty", [0, 1])
def test_rows_of_the_join(rows, H, g, T, empty):
    """A shared span, a causal one per query; the last query may have neither."""
    n = T - empty
    exact, launched, stride, most, gaps = rows(64, 0, H, g, T, [(0, n, 64, 0)] + [(i, 1, 40, 1) for i in range(n)])
    assert exact == T * H * g and most <= stride and gaps == 0
    # a tile of 16 rows that a group's heads do not fill is cut once more
    cuts = 1 if g % 16 == 0 or g <= 16 else 1 + 16 * (g / 16 + 2) / g
    assert exact <= launched <= exact * max(cuts, 1) + 16


def test_more_rows_than_32_bits_hold_are_counted(rows):
    """One entry of many heads among many small ones: the product does not wrap."""
    exact, launched, *_ = rows(64, 0, 1, 65535, 40, [(0, 39, 64, 0)] + [(i, 1, 40, 1) for i in range(39)])
    # two cuts per 16 heads: the shared span's tiles and the query's own do not start together
    assert exact == 40 * 65535 and exact <= launched < 2.01 * exact
