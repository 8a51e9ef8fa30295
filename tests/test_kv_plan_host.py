"""The plan of an attention call (paper_2609_33224_gb300/csrc/kv_plan.h): every (query, head, key) that a span
gives a query is in exactly one piece, no piece reaches past its blocks, every row's result is written once, from
exactly the parts that its pieces leave, and the shares are even."""
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_33224_gb300", "csrc")

HARNESS = r"""
#include <cstdio>
#include <map>
#include <set>
#include "kv_plan.h"
using namespace pskv;
#define CHECK(x) do { if (!(x)) { std::printf("line %d: %s\n", __LINE__, #x); return 1; } } while (0)
int main() {
  unsigned sms, D, fmt, H, g, T, n;
  while (std::scanf("%u %u %u %u %u %u %u", &sms, &D, &fmt, &H, &g, &T, &n) == 7) {
    std::vector<ps_kv_span> sp(n);
    uint64_t blocks = 0;
    for (auto& s : sp) {
      unsigned a, b, c, d;
      if (std::scanf("%u %u %u %u", &a, &b, &c, &d) != 4) return 2;
      s = ps_kv_span{a, b, c, d, blocks};
      blocks += (c + 15) / 16;
    }
    Layout o;
    const PlanShape shape{(int)sms, D, (int)fmt, H, g};
    lay_out(shape, T, sp.data(), n, &o);
    // parts: (part row) -> (row of the batch); keys seen per (query, q head)
    std::map<uint64_t, uint64_t> part_of;                 // part row -> query * H * g + head
    std::vector<std::map<unsigned, std::vector<std::pair<long, long>>>> seen(T * H * g);  // first block of a span -> key ranges
    std::vector<int> written(T * H * g, 0);
    std::vector<std::set<uint64_t>> parts(T * H * g);     // part rows that a row's pieces leave
    std::vector<std::set<uint64_t>> folded(T * H * g);    // part rows that a piece joins in
    for (int kind = 0; kind < 2; ++kind) {
      const auto& pieces = kind ? o.tile_pieces : o.row_pieces;
      const auto& off = kind ? o.tile_off : o.row_off;
      // side by side, the kernels share the SMs
      CHECK(o.row_sms > 0 && o.row_sms <= (int)sms);
      const unsigned tile_sms = o.row_sms < (int)sms ? sms - o.row_sms : sms;
      const unsigned workers = kind ? tile_sms / tile_ctas_of(D) : o.row_sms * kRowWarps;
      if (pieces.empty()) { CHECK(off.size() <= 1); continue; }
      CHECK(off.front() == 0 && off.back() == pieces.size() && off.size() - 1 <= workers);
      uint64_t total = 0, most = 0;
      for (size_t w = 0; w + 1 < off.size(); ++w) {
        CHECK(off[w] < off[w + 1]);
        uint64_t mine = 0;
        for (uint32_t k = off[w]; k < off[w + 1]; ++k) mine += pieces[k].nblocks + (kind ? 4 : 2);
        total += mine;
        most = std::max(most, mine);
      }
      CHECK(most * workers <= total * 5 / 4 + workers * 8);
      for (const Piece& p : pieces) {
        const ps_kv_span* s = nullptr;
        for (const auto& x : sp)
          if (x.length && p.block >= x.first_block && p.block < x.first_block + (x.length + 15) / 16) s = &x;
        CHECK(s && p.query0 == s->first_query && p.head < H && p.nblocks > 0 && p.nrows > 0);
        const unsigned step = kind ? kTileKeys : kBlock;
        CHECK(p.key0 % kBlock == 0 && p.block == s->first_block + p.key0 / kBlock);
        CHECK(p.key0 < p.end && p.end <= s->length && p.key0 + (p.nblocks - 1) * step < p.end);
        const unsigned keys = std::min<unsigned>(p.end - p.key0, p.nblocks * step);
        CHECK(p.row0 % (kind ? shape.tile_rows(s->num_queries * g) : kSmallRows) == 0);
        CHECK(p.nrows <= (kind ? shape.tile_rows(s->num_queries * g) : kSmallRows) && p.row0 + p.nrows <= s->num_queries * g);
        if (p.split) CHECK(kind && D == 128 && p.nrows <= tile_rows_of(128) / 2 && p.nblocks > 1);
        if (kind) CHECK(p.end == p.key0 + keys || keys % kTileKeys == 0);
        for (unsigned i = 0; i < p.nrows; ++i) {
          const unsigned r = p.row0 + i, q = r / g;
          const uint64_t row = ((uint64_t)(s->first_query + q) * H + p.head) * g + r % g;
          long last = (long)std::min<unsigned>(p.key0 + keys, p.end);
          const long lim = s->causal ? (long)s->length - (long)s->num_queries + q + 1 : (long)s->length;
          if (kind) CHECK(last <= lim);  // every row of a tile sees all of its keys
          else CHECK((long)p.climit == (s->causal ? lim - 1 - (long)q : (long)kNoLimit));
          last = std::min(last, lim);
          if (last > (long)p.key0) seen[row][s->first_block].push_back({p.key0, last});
          if (p.part_row == kDirect) {
            ++written[row];
            CHECK(kind == 0 || !p.nfold);
          } else {
            for (unsigned x = 0; x < (p.split ? 2u : 1u); ++x) {
              const uint64_t pr = (uint64_t)p.part_row + x * p.split + i;
              CHECK(pr < o.part_rows && part_of.emplace(pr, row).second);
              parts[row].insert(pr);
            }
          }
        }
        unsigned next = 0;
        for (unsigned x = 0; x < p.nfold; ++x) {
          const Fold& f = o.folds[p.fold0 + x];
          CHECK(f.first == next && f.count > 0);
          next += f.count;
          for (unsigned i = f.first; i < next; ++i) {
            const unsigned r = p.row0 + i;
            const uint64_t row = ((uint64_t)(s->first_query + r / g) * H + p.head) * g + r % g;
            for (unsigned y = 0; y < f.nsegs; ++y) {
              const JoinSeg& sg = o.segs[f.seg0 + y];
              for (unsigned k = 0; k < sg.nparts; ++k) CHECK(folded[row].insert(sg.row + (i - f.first) + (uint64_t)k * sg.stride).second);
            }
          }
        }
        if (p.nfold) CHECK(next == p.nrows);
      }
    }
    std::vector<std::set<uint64_t>> joined(T * H * g);
    for (const JoinEntry& e : o.join)
      for (unsigned i = 0; i < e.count; ++i) {
        const uint64_t row = (uint64_t)e.query * H * g + e.head0 + i;
        ++written[row];
        for (unsigned x = 0; x < e.nsegs; ++x) {
          const JoinSeg& sg = o.segs[e.seg0 + x];
          for (unsigned k = 0; k < sg.nparts; ++k) CHECK(joined[row].insert(sg.row + i + (uint64_t)k * sg.stride).second);
        }
      }
    for (uint64_t row = 0; row < (uint64_t)T * H * g; ++row) {
      CHECK(written[row] == 1);
      std::set<uint64_t> all = joined[row];
      all.insert(folded[row].begin(), folded[row].end());
      CHECK(all.size() == joined[row].size() + folded[row].size() && all == parts[row]);
      const unsigned q = row / (H * g);
      for (const auto& s : sp) {
        auto r = seen[row][s.first_block];
        const long lim = q < s.first_query || q >= s.first_query + s.num_queries ? 0
                         : s.causal ? std::min<long>(s.length, (long)s.length - (long)s.num_queries + (q - s.first_query) + 1) : (long)s.length;
        if (!s.length) continue;
        std::sort(r.begin(), r.end());
        long at = 0;
        for (auto& x : r) {
          CHECK(x.first == at);
          at = x.second;
        }
        CHECK(at == std::max(0l, lim));
      }
    }
    std::printf("ok %zu %zu %zu %zu\n", o.row_pieces.size(), o.tile_pieces.size(), o.join.size(), o.folds.size());
  }
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    src, exe = d / "p.cpp", d / "p"
    src.write_text(HARNESS)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", CSRC, "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)],
                   check=True)

    def run(cases):
        text = ""
        for (sms, D, fmt, H, g, T), spans in cases:
            text += "%d %d %d %d %d %d %d\n" % (sms, D, fmt, H, g, T, len(spans)) + "".join("%d %d %d %d\n" % s for s in spans)
        r = subprocess.run([str(exe)], input=text, capture_output=True, text=True)
        lines = r.stdout.splitlines()
        assert r.returncode == 0 and len(lines) == len(cases), (cases[len(lines) - 1], lines[-1:])
        return [tuple(int(x) for x in ln.split()[1:]) for ln in lines]
    return run


def _random(rng):
    D, fmt = rng.choice([64, 128]), rng.randrange(3)
    H, g = rng.choice([1, 2, 3]), rng.choice([1, 2, 5, 8, 16, 21])
    T = rng.choice([1, 2, 7, 30, 90])
    spans = []
    for _ in range(rng.randrange(0, 7)):
        a = rng.randrange(T)
        n = rng.randrange(0, T - a + 1)
        length = rng.choice([0, 1, 15, 16, 17, 100, rng.randrange(1, 3000)])
        spans.append((a, n, length, rng.randrange(2)))
    return (rng.choice([2, 8, 152]), D, fmt, H, g, T), spans


def test_every_key_once(plan):
    rng = random.Random(3)
    got = plan([_random(rng) for _ in range(400)])
    assert any(x[1] for x in got) and any(x[0] for x in got) and any(x[2] for x in got)


def test_forms(plan):
    """Batches that use each form: tiles with row-kernel ends, split tiles, joins in the row kernel, direct output."""
    got = plan([
        ((152, 128, 0, 8, 8, 400), [(0, 400, 4000, 0)] + [(i * 100, 100, 700, 1) for i in range(4)]),
        ((8, 128, 2, 8, 8, 4), [(0, 4, 30000, 0)]),
        ((4, 128, 0, 2, 8, 300), [(0, 300, 500, 0)] + [(i * 30, 30, 60, 1) for i in range(10)]),
        ((152, 64, 1, 1, 1, 200), [(i, 1, 3000, 0) for i in range(200)]),
    ])
    assert got[0][0] and got[0][1]
    assert got[1][1] or got[1][0]
    assert got[2][3] > 0  # joined in by the row kernel
    assert got[3][1] == 0
