"""Batches that reach the rarer forms of the attention kernels, by the plan's rules on 152 SMs
(paper_2609_33224_gb300/csrc/kv_plan.h): masked tile pieces that are split by the parity of their steps, and joins by entries.
A change of the rules' constants that loses a form is found here; the GPU's tests of the same batches compare results."""
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_33224_gb300", "csrc")


def requests(sizes, shared=0, kind=2):
    """(T, spans (first, queries, length, kind)) of requests (context, nodes), all on a shared prefix."""
    T, first = sum(n for _, n in sizes), 0
    spans = [(0, T, shared, 0)] if shared else []
    for own, n in sizes:
        spans.append((first, n, own + n, kind))
        first += n
    return T, spans


def _straddling(count, steps, n, seed):
    """Contexts whose `n` drafted tokens lie on both sides of a multiple of 128, about `steps` of them in."""
    rng = random.Random(seed)
    return [(128 * (steps + rng.randint(0, 4)) - rng.randint(1, n - 1), n) for _ in range(count)]


# name: (H, g, T, spans)
SPLIT = {
    "8x32_on_3000": (4, 8, *requests(_straddling(8, 23, 32, 1))),
    "8x16_on_8000": (8, 8, *requests(_straddling(8, 62, 16, 2))),
}
SPLIT_LONG = {"4x16_on_30000": (8, 8, *requests(_straddling(4, 234, 16, 3)))}
# name: (D, H, g, T, spans), and between how many parts its row of most parts has
ENTRIES = {
    "few_parts": ((128, 8, 8, *requests([(700, 29)] * 10, 9000)), 2, 4),
    "few_parts_causal": ((128, 8, 8, *requests([(2000, 300)], kind=1)), 2, 4),
    "several_parts": ((128, 8, 8, *requests([(300, 52)] * 5, 500)), 5, 8),
    "several_parts_64": ((64, 8, 8, *requests([(300, 52)] * 5, 500)), 5, 8),
}

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
    // split pieces with own tokens; those of them whose own tokens begin in an even, an odd step, and are in two steps
    unsigned split = 0, even = 0, odd = 0, both = 0;
    for (const Piece& p : o.tile_pieces) {
      const uint32_t end = std::min(p.end, p.key0 + p.nblocks * kTileKeys);
      if (!p.split || p.climit == kNoLimit || (uint32_t)p.climit >= end) continue;
      const uint32_t first = p.climit < (int32_t)p.key0 ? 0 : (p.climit - p.key0) / kTileKeys;
      ++split;
      ++(first & 1 ? odd : even);
      both += first != (end - 1 - p.key0) / kTileKeys;
    }
    std::printf("%u %u %u %u %d %u\n", split, even, odd, both,
                (int)join_by_entries((uint32_t)o.join.size(), o.join_stride, o.join_parts), o.join_parts);
  }
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("shapes")
    src, exe = d / "p.cpp", d / "p"
    src.write_text(HARNESS)
    subprocess.run(["g++", "-std=c++17", "-O2", "-I", CSRC, "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)],
                   check=True)

    def run(D, fmt, H, g, T, spans):
        text = "%d %d %d %d %d %d\n" % (D, fmt, H, g, T, len(spans)) + "".join("%d %d %d %d\n" % s for s in spans)
        r = subprocess.run([str(exe)], input=text, capture_output=True, text=True, check=True)
        return [int(x) for x in r.stdout.split()]
    return run


@pytest.mark.parametrize("fmt", [0, 1, 2])
@pytest.mark.parametrize("name", [*SPLIT, *SPLIT_LONG])
def test_masked_pieces_split_by_steps(plan, name, fmt):
    split, even, odd, both, *_ = plan(128, fmt, *{**SPLIT, **SPLIT_LONG}[name])
    assert split >= 4 and even and odd and both >= 2


@pytest.mark.parametrize("fmt", [0, 1, 2])
@pytest.mark.parametrize("name", list(ENTRIES))
def test_joins_by_entries(plan, name, fmt):
    (D, *shape), least, most = ENTRIES[name]
    *_, by, parts = plan(D, fmt, *shape)
    assert by and least <= parts <= most
