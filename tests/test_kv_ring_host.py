"""A warp that gives up waits for all of its copies under way, the one it gave up on too
(paper_2609_33224_gb300/csrc/kv_ring.h)."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_33224_gb300", "csrc")

HARNESS = r"""
#include <cstdio>
#include <utility>
#include <vector>
#include "kv_ring.h"
template <uint32_t S>
int run() {
  for (uint32_t total = 0; total < 4 * S; ++total)        // blocks of the worker
    for (uint32_t used = 0; used <= total; ++used) {      // those used when it gives up
      const uint32_t issued = used + S < total ? used + S : total;
      std::vector<std::pair<uint32_t, uint32_t>> got, want;
      for (uint32_t i = used; i < issued; ++i) want.push_back({i % S, i / S & 1u});
      pskv::drain_ring<S>(used % S, used / S & 1u, issued - used, [&](uint32_t s, uint32_t p) { got.push_back({s, p}); });
      if (got != want) { std::printf("%u stages, %u of %u\n", S, used, total); return 1; }
    }
  return 0;
}
int main() { return run<1>() | run<2>() | run<3>() | run<4>() | run<7>(); }
"""


def test_every_copy_under_way_is_waited_for(tmp_path):
    src, exe = tmp_path / "r.cpp", tmp_path / "r"
    src.write_text(HARNESS)
    subprocess.run(["g++", "-std=c++17", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout


def test_the_row_kernel_uses_it():
    with open(os.path.join(CSRC, "kv_rows.cu")) as f:
        text = f.read()
    assert text.count("drain_ring<kStages>(st, phase, in_flight,") == 1 and "while (--in_flight)" not in text


def test_the_tile_kernel_ends_its_long_wait():
    """The warp that zeroes partial steps waits long for each; the threads it waits for say that they have given up
    before their last arrival, and it asks after each wait, before it goes on."""
    with open(os.path.join(CSRC, "kv_tiles.cu")) as f:
        text = f.read()
    told = "*static_cast<volatile uint32_t*>(&bars.gave_up) = 1;\n        mbar_arrive(smem_u32(&bars.tail_here));"
    assert text.count("bars.gave_up = 0;") == 1 and text.count(told) == 2
    assert text.count("mbar_arrive(smem_u32(&bars.tail_here));") == 4  # two a step, two when given up
    wait = text.index("60000000000ull")
    assert wait < text.index("if (*static_cast<volatile uint32_t*>(&bars.gave_up)) break;") < text.index("- 1) % C::kSlots * C::kSlot;")
