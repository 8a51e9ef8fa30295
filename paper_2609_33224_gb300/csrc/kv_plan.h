// How a batch's spans are laid out for the attention kernels: host code without CUDA, so that it can be tested
// alone.
//
// A span's rows are its queries' heads of a group.  The row kernel takes 16 of them at a time, the tile kernel up
// to 512; which one takes a span (or the front of a causal one) is a matter of the time it adds.  The (rows,
// key/value head, keys) of each kernel are cut into equal shares for its workers.  A piece whose rows have other
// pieces leaves a partial result; the rest of the plan says which partial results make up a query's rows.
#pragma once

#include <stdint.h>

#include <algorithm>
#include <vector>

#include "packserve_kv.h"

namespace pskv {

constexpr int kBlock = PS_BLOCK_TOKENS;
constexpr int kSmallRows = 16;  // rows of a tile of the row kernel (one m16 of mma.sync)

// Rows of a tile of the tile kernel, two accumulators of 128 rows a CTA: with head_dim 128 a pair of CTAs
// shares the keys and values.
constexpr int tile_ctas_of(int D) { return D == 128 ? 2 : 1; }
constexpr int tile_rows_of(int D) { return 256 * tile_ctas_of(D); }
constexpr int kTileKeys = 128;  // keys of one step of the tile kernel

// Workers (warps) of a CTA of the row kernel.  12 hide more of a block's latency than 8 where instructions bind it (131072
// tokens of 5 requests, fp8: 166 us, 183; 256 queries on 32768: 249 and 274; 16-bit ones are bound by bytes: 64 queries
// on 8192 39.2 and 37.9); 16 would leave 128 registers a thread, and spill.
constexpr int kRowWarps = 12;

// A piece of work of either attention kernel: a run of key blocks for the rows of one tile and one
// key/value head.  A span's rows are its queries' heads of the group, row r = (r / g)-th query, head r % g.
struct alignas(16) Piece {
  uint32_t block;     // where the piece's block ids start
  uint32_t nblocks;   // blocks (row kernel) or key tiles of 8 blocks (tile kernel; the last may be partial)
  uint32_t key0;      // index in the span of the first key
  uint32_t end;       // keys end before this index
  int32_t climit;     // the span's i-th query sees keys j <= climit + i
  uint32_t query0;    // the span's first query
  uint32_t row0;      // the tile's first row
  uint32_t part_row;  // first row of the partial result, or kDirect: the output is written
  uint16_t nrows;
  uint16_t head;
  uint32_t fold0, nfold;  // row kernel, kDirect: the tile kernel's parts of these rows, to be joined in
  uint32_t split;  // tile kernel: not 0: its even steps in tile 0, its odd ones in tile 1, so many rows behind
};
static_assert(sizeof(Piece) == 48, "Piece layout");
constexpr uint32_t kDirect = 0xFFFFFFFFu;
constexpr int32_t kNoLimit = 0x3FFFFFFF;

// What is to be joined: the rows head0 .. head0 + count - 1 of a query, whose parts are the segments
// segs[seg0] ..: the i-th row's are the partial rows row + i + k * stride, k < nparts.  The join kernel gives every entry
// as many rows as the largest has (Layout::join_stride).
struct JoinEntry {
  uint32_t query;
  uint16_t head0, count;
  uint32_t seg0, nsegs;
};
struct JoinSeg {
  uint32_t row, stride, nparts;
};
// The same for the rows first .. first + count - 1 of a piece.
struct Fold {
  uint32_t seg0;
  uint16_t nsegs;
  uint8_t first, count;
};

struct PlanShape {
  int sms;
  uint32_t D;
  int fmt;
  uint32_t heads, group;  // key/value heads; query heads of each

  // rows of the tile kernel's tiles for a span of so many rows
  uint32_t tile_rows(uint32_t rows) const {
    const uint32_t full = (uint32_t)tile_rows_of((int)D);
    return rows <= full / 2 ? full / 2 : full;
  }
};

// Which kernel takes the rows of a tile and head over the keys that all of them see: the one that adds less time to
// the batch.  Nanoseconds of the whole GPU, from spans of 24 to 256 rows on 512 to 65536 keys: the row kernel per 16
// rows and 16 keys, the tile kernel per step of 128 keys, a piece of it costing three steps more; the tile kernel
// adds kTileLaunch to a call.  In front of a causal span's end, of which the row kernel has a short piece per 16 rows
// anyway, its blocks cost about four times as much, as its pieces then are of uneven lengths (192 new tokens on 16384:
// 457 us, 500 without this).  By tiles / by rows, us, one span of 8 key/value heads: bf16 with head_dim 128,
// 128 rows on 512 keys 10.9/11.2, on 4096 16.7/19.0, 64 rows on 2048 12.0/10.3, on 16384 22.7/24.7, 32 rows on 16384
// 22.4/18.8; fp8, 64 rows on 4096 15.5/16.3; bf16 with head_dim 64, 64 rows on 4096 9.1/10.3.
constexpr double kTileLaunch = 1000.0;
inline double block_ns(const PlanShape& kv) {
  const bool fp8 = kv.fmt == PS_KV_FP8;
  return kv.D == 128 ? (fp8 ? 0.60 : 0.51) : (fp8 ? 0.50 : 0.40);
}
inline double step_ns(const PlanShape& kv) {
  const bool fp8 = kv.fmt == PS_KV_FP8;
  return kv.D == 128 ? (fp8 ? 20.5 : 17.5) : (fp8 ? 9.0 : 8.0);
}
constexpr int kPieceSteps = 3;
// Bytes that a token has in one head.
inline double token_bytes(const PlanShape& kv) { return kv.fmt == PS_KV_FP8 ? 2 * (kv.D + 1.0) : 4.0 * kv.D; }
inline double tile_saves(const PlanShape& kv, uint32_t rows, int64_t keys, bool causal) {
  const uint32_t row_tiles = (rows + kSmallRows - 1) / kSmallRows;
  const double dear = causal && row_tiles > 1 ? 4 : 1;
  double by_rows = dear * block_ns(kv) * row_tiles * (double)((keys + kBlock - 1) / kBlock);
  // Keys that L2 does not hold come from memory again for every other 16 rows: 64 rows on 65536 tokens (268 MB) 124 us,
  // 65 by tiles; 32 rows 55 and 65.
  if (row_tiles > 2 && (double)keys * token_bytes(kv) * kv.heads > 96e6)
    by_rows = std::max(by_rows, row_tiles / 2.0 * (double)keys * token_bytes(kv) / 5000.0);
  return by_rows - step_ns(kv) * (double)((keys + kTileKeys - 1) / kTileKeys + kPieceSteps);
}

// From so many steps on, a piece of one tile of rows runs as two.  64 rows on 65536 tokens: 65 us, 79 as one; on
// 1024 (2 steps a piece), where the second result costs more than it brings, 11.4 and 11.0.  With head_dim 64,
// whose steps are half as long, it brought nothing (35 and 34 us).
constexpr uint32_t kSplitSteps = 8;

// The row kernel is bound by the cache's bytes, which a part of the SMs can draw, the tile kernel by its SMs: side by
// side they take less time than one after the other.  Returns how many SMs the row kernel gets (all: one after the
// other), by the times above, 3.3 ns of the GPU for a unit's start and end, the bytes at 6.2 TB/s, and what the
// kernels take whatever their SMs: 6 and 4 us.  64 queries on 8192 shared tokens 55.7 -> 41.8 us, 9 groups under one
// prompt with head_dim 64 24.6 -> 20.4, 256 queries on 32768 (fp8) 267 -> 260, with the kernels of then (39.2, 17.8 and
// 248 now).
constexpr double kUnitNs = 3.3, kBytesPerNs = 6200.0, kTileFixed = 6000.0, kRowFixed = 4000.0;
inline int row_sms(const PlanShape& kv, double steps, double blocks, double units) {
  const double tile = step_ns(kv) * steps, work = block_ns(kv) * blocks + kUnitNs * units;
  const double bytes = blocks * kBlock * token_bytes(kv) / kBytesPerNs;
  double best = kTileFixed + tile + kRowFixed + std::max(work, bytes);
  int sms = kv.sms;
  for (int x = 2; x < kv.sms; x += 2) {
    const double f = (double)x / kv.sms;
    const double t = std::max(kTileFixed + tile / (1 - f), kRowFixed + std::max(work / f, bytes));
    if (t < 0.995 * best || (sms < kv.sms && t < best)) {
      best = t;
      sms = x;
    }
  }
  return sms;
}

// A piece of the row kernel joins up to this many tile parts into its rows, where an SM has at least so many units
// of rows that the time this takes evens out.  192 new tokens on 16384 (31 units an SM, 2 to 3 parts): 456 us, 491
// with the join kernel; 256 queries on 32768 (13 units an SM, 3 parts) 288 and 277 us, 64 on 8192 (10 parts) 92
// and 60.
constexpr size_t kFoldMost = 3, kFoldUnits = 24;

// Rows of one tile and one head over a range of key blocks, before it is cut into pieces.
struct Unit {
  Piece p;             // block, key0: of the whole range
  uint32_t group;      // its entry of the groups
  uint32_t tile_rows;  // rows of its partial results
  uint32_t layer;
};

// The rows of a span, tiled one way; tile t and head h have the parts groups[group0 + t * kv_heads + h].
struct Layer {
  uint32_t query0, num_queries, tile_rows, group0;
};
struct Group {
  uint32_t part_row;  // kDirect: written by the attention kernel
  uint32_t nparts;
};

struct Layout {
  std::vector<Layer> layers;
  std::vector<Group> groups;
  std::vector<Unit> row_units, tile_units;
  std::vector<Piece> row_pieces, tile_pieces;
  std::vector<uint32_t> row_off, tile_off, tok_off, tok_layer;
  std::vector<JoinEntry> join;
  std::vector<JoinSeg> segs;
  std::vector<Fold> folds;
  uint64_t part_rows = 0;
  uint32_t max_parts = 1;
  uint32_t join_stride = 0;  // the largest entry's count
  int row_sms = 0;  // SMs of the row kernel; fewer than all: beside the tile kernel
};

// Rows of the join kernel's launch.
inline uint64_t join_rows(const Layout& o) { return (uint64_t)o.join.size() * o.join_stride; }

// A unit of the layer and group that come last.
inline Unit unit(const ps_kv_span& s, uint32_t r0, uint32_t nr, uint32_t h, int64_t from, int64_t end, int step, int32_t climit,
          uint32_t tile_rows, const Layout& o) {
  Unit u{};
  u.p.block = (uint32_t)(s.first_block + (uint64_t)from / kBlock);
  u.p.nblocks = (uint32_t)((end - from + step - 1) / step);
  u.p.key0 = (uint32_t)from;
  u.p.end = (uint32_t)end;
  u.p.climit = climit;
  u.p.query0 = s.first_query;
  u.p.row0 = r0;
  u.p.nrows = (uint16_t)nr;
  u.p.head = (uint16_t)h;
  u.group = (uint32_t)o.groups.size();
  u.tile_rows = tile_rows;
  u.layer = (uint32_t)o.layers.size() - 1;
  return u;
}

// Cuts units into pieces for at most `most` workers with equal shares of the work; a piece costs its steps
// and `extra` (its rows' load and result).  Every worker gets whole steps; a remainder of one step stays
// with its piece.
inline void share_out(const std::vector<Unit>& units, uint32_t most, uint32_t extra, uint32_t least, uint32_t step_blocks,
               std::vector<Piece>* pieces, std::vector<uint32_t>* off, std::vector<uint32_t>* first_piece) {
  uint64_t total = 0;
  for (const Unit& u : units) total += u.p.nblocks + extra;
  uint64_t share = std::max<uint64_t>((total + most - 1) / most, least + extra);
  for (;;) {
    pieces->clear();
    off->assign(1, 0);
    first_piece->clear();
    uint64_t room = share;
    for (const Unit& u : units) {
      first_piece->push_back((uint32_t)pieces->size());
      uint32_t done = 0;
      while (done < u.p.nblocks) {
        const uint32_t left = u.p.nblocks - done;
        if (room < share && room < extra + std::min<uint64_t>(left, least)) {
          off->push_back((uint32_t)pieces->size());
          room = share;
        }
        uint64_t take = std::max<uint64_t>(room > extra ? room - extra : 1, 1);
        if (take + 1 >= left) take = left;
        Piece p = u.p;
        p.block += done * step_blocks;
        p.key0 += done * step_blocks * kBlock;
        p.nblocks = (uint32_t)take;
        pieces->push_back(p);
        done += (uint32_t)take;
        room -= std::min<uint64_t>(room, take + extra);
      }
    }
    off->push_back((uint32_t)pieces->size());
    if (off->size() - 1 <= most) return;
    share += std::max<uint64_t>(1, share / 64);
  }
}

inline void lay_out(const PlanShape& pl, uint32_t T, const ps_kv_span* spans, uint32_t n_spans, Layout* out) {
  Layout& o = *out;
  const uint32_t H = pl.heads, g = pl.group;
  // The keys that all rows of a tile see, where the tile kernel is the one to take them (else 0).
  auto cut_of = [&](const ps_kv_span& s, uint32_t r0, uint32_t nr) -> int64_t {
    int64_t c = (int64_t)s.length;
    if (s.causal) c = std::max<int64_t>(0, c - (int64_t)s.num_queries + r0 / g + 1) / kBlock * kBlock;
    return tile_saves(pl, nr, c, s.causal != 0) > 0 ? c : 0;
  };
  auto tiles_save = [&](const ps_kv_span& s) {
    double sum = 0;
    const uint32_t rows = s.num_queries * g, tr = pl.tile_rows(rows);
    for (uint32_t r0 = 0; r0 < rows; r0 += tr) {
      const uint32_t nr = std::min(rows - r0, tr);
      const int64_t c = cut_of(s, r0, nr);
      if (c > 0) sum += tile_saves(pl, nr, c, s.causal != 0) * H;
    }
    return sum;
  };
  double saved = 0;
  for (uint32_t si = 0; si < n_spans; ++si) saved += tiles_save(spans[si]);
  auto tiles_for = [&](const ps_kv_span& s) { return saved > kTileLaunch && tiles_save(s) > 0; };

  for (uint32_t si = 0; si < n_spans; ++si) {
    const ps_kv_span& s = spans[si];
    if (s.num_queries == 0 || s.length == 0) continue;
    const uint32_t rows = s.num_queries * g;
    const int64_t len = (int64_t)s.length;
    const int32_t climit = s.causal ? (int32_t)(len - (int64_t)s.num_queries) : kNoLimit;

    // Tiles take the keys that all their rows see; cut[t]: how many those are for tile t.
    std::vector<int64_t> cut;
    const uint32_t tile_rows = pl.tile_rows(rows);
    if (tiles_for(s)) {
      o.layers.push_back(Layer{s.first_query, s.num_queries, tile_rows, (uint32_t)o.groups.size()});
      for (uint32_t r0 = 0; r0 < rows; r0 += tile_rows) {
        const uint32_t nr = std::min(rows - r0, tile_rows);
        const int64_t c = cut_of(s, r0, nr);
        cut.push_back(c);
        for (uint32_t h = 0; h < H; ++h) {
          if (c > 0) o.tile_units.push_back(unit(s, r0, nr, h, 0, c, kTileKeys, kNoLimit, tile_rows, o));
          o.groups.push_back(Group{0, 0});
        }
      }
      if (*std::min_element(cut.begin(), cut.end()) == len) continue;  // not causal, and all of it to tiles
    }
    o.layers.push_back(Layer{s.first_query, s.num_queries, (uint32_t)kSmallRows, (uint32_t)o.groups.size()});
    for (uint32_t r0 = 0; r0 < rows; r0 += kSmallRows) {
      const uint32_t nr = std::min<uint32_t>(rows - r0, kSmallRows);
      const int64_t from = cut.empty() ? 0 : cut[r0 / tile_rows];
      const int64_t end = s.causal ? std::min<int64_t>(len, (int64_t)climit + (r0 + nr - 1) / g + 1) : len;
      for (uint32_t h = 0; h < H; ++h) {
        if (end > from) o.row_units.push_back(unit(s, r0, nr, h, from, end, kBlock, climit, kSmallRows, o));
        o.groups.push_back(Group{0, 0});
      }
    }
  }

  // which layers cover a query
  o.tok_off.assign((size_t)T + 1, 0);
  for (size_t l = 0; l < o.layers.size(); ++l)
    for (uint32_t i = 0; i < o.layers[l].num_queries; ++i) ++o.tok_off[o.layers[l].query0 + i + 1];
  std::vector<uint8_t> alone(T, 0);
  for (uint32_t t = 0; t < T; ++t) {
    alone[t] = o.tok_off[t + 1] == 1;
    o.tok_off[t + 1] += o.tok_off[t];
  }
  o.tok_layer.resize(o.tok_off[T]);
  {
    std::vector<uint32_t> at(o.tok_off.begin(), o.tok_off.end() - 1);
    for (size_t l = 0; l < o.layers.size(); ++l)
      for (uint32_t i = 0; i < o.layers[l].num_queries; ++i) o.tok_layer[at[o.layers[l].query0 + i]++] = (uint32_t)l;
  }

  // Pieces, and where their results go.  A group of one piece writes the output where nothing is to be joined,
  // or, in the row kernel, which comes after the tile kernel, where only tiles are to be joined.
  auto layers_of = [&](uint32_t t, uint32_t* n) {
    *n = o.tok_off[t + 1] - o.tok_off[t];
    return o.tok_layer.data() + o.tok_off[t];
  };
  auto fold = [&](const Unit& u, Piece* p) {
    const size_t segs = o.segs.size(), folds = o.folds.size();
    for (uint32_t i = 0, n; i < p->nrows; i += n) {
      const uint32_t r = p->row0 + i, t = p->query0 + r / g;
      uint32_t nl;
      const uint32_t* ls = layers_of(t, &nl);
      n = g - r % g;  // and the queries after it that have the same layers
      for (uint32_t t2 = t + 1; i + n < p->nrows; ++t2, n += g) {
        uint32_t nl2;
        const uint32_t* ls2 = layers_of(t2, &nl2);
        if (nl2 != nl || !std::equal(ls, ls + nl, ls2)) break;
      }
      n = std::min<uint32_t>(n, p->nrows - i);
      const uint32_t seg0 = (uint32_t)o.segs.size();
      for (uint32_t l = 0; l < nl; ++l) {
        const Layer& ly = o.layers[ls[l]];
        if (ls[l] == u.layer) continue;
        if (ly.tile_rows <= (uint32_t)kSmallRows) {
          o.segs.resize(segs);
          o.folds.resize(folds);
          return false;
        }
        n = std::min(n, ly.tile_rows - ((t - ly.query0) * g + r % g) % ly.tile_rows);
      }
      for (uint32_t l = 0; l < nl; ++l) {
        const Layer& ly = o.layers[ls[l]];
        if (ls[l] == u.layer) continue;
        const uint32_t rr = (t - ly.query0) * g + r % g;
        const Group& gr = o.groups[ly.group0 + rr / ly.tile_rows * H + p->head];
        if (gr.nparts) o.segs.push_back(JoinSeg{gr.part_row + rr % ly.tile_rows, ly.tile_rows, gr.nparts});
      }
      o.folds.push_back(Fold{seg0, (uint16_t)(o.segs.size() - seg0), (uint8_t)i, (uint8_t)n});
    }
    uint32_t parts = 0;
    for (size_t x = segs; x < o.segs.size(); ++x) parts += o.segs[x].nparts;
    if (parts > kFoldMost * (o.folds.size() - folds)) {
      o.segs.resize(segs);
      o.folds.resize(folds);
      return false;
    }
    p->fold0 = (uint32_t)folds;
    p->nfold = (uint32_t)(o.folds.size() - folds);
    return true;
  };
  const bool may_fold = o.row_units.size() >= kFoldUnits * (size_t)pl.sms;
  o.row_sms = pl.sms;
  if (!o.tile_units.empty() && !o.row_units.empty() && !may_fold) {
    double steps = 0, blocks = 0;
    for (const Unit& u : o.tile_units) steps += u.p.nblocks + kPieceSteps;
    for (const Unit& u : o.row_units) blocks += u.p.nblocks;
    o.row_sms = row_sms(pl, steps, blocks, (double)o.row_units.size());
  }
  const int tile_sms = o.row_sms < pl.sms ? pl.sms - o.row_sms : pl.sms;
  const uint32_t row_workers = (uint32_t)(o.row_sms * kRowWarps);
  auto finish = [&](std::vector<Unit>& units, std::vector<Piece>& pieces, std::vector<uint32_t>& first, bool rows) {
    for (size_t i = 0; i < units.size(); ++i) {
      const uint32_t a = first[i], b = i + 1 < units.size() ? first[i + 1] : (uint32_t)pieces.size();
      const Piece& p = units[i].p;
      // a tile piece that is split by steps has two parts
      uint32_t nparts = 0;
      for (uint32_t k = a; k < b; ++k) {
        if (!rows && pl.D == 128 && p.nrows <= tile_rows_of(128) / 2 && pieces[k].nblocks >= kSplitSteps)
          pieces[k].split = units[i].tile_rows;
        nparts += pieces[k].split ? 2 : 1;
      }
      bool direct = nparts == 1;
      for (uint32_t q = p.row0 / g; direct && q <= (p.row0 + p.nrows - 1) / g; ++q) direct = alone[p.query0 + q];
      if (!direct && rows && may_fold && nparts == 1) direct = fold(units[i], &pieces[a]);
      Group& gr = o.groups[units[i].group];
      if (direct) {
        gr = Group{kDirect, 1};
        pieces[a].part_row = kDirect;
        continue;
      }
      gr = Group{(uint32_t)o.part_rows, nparts};
      o.max_parts = std::max(o.max_parts, nparts);
      for (uint32_t k = a; k < b; ++k) {
        pieces[k].part_row = (uint32_t)o.part_rows;
        o.part_rows += units[i].tile_rows * (pieces[k].split ? 2 : 1);
      }
    }
  };
  std::vector<uint32_t> first;
  if (!o.tile_units.empty()) {
    const uint32_t workers = (uint32_t)std::max(1, tile_sms / tile_ctas_of((int)pl.D));
    share_out(o.tile_units, workers, 4, 2, kTileKeys / kBlock, &o.tile_pieces, &o.tile_off, &first);
    finish(o.tile_units, o.tile_pieces, first, false);
  }
  if (!o.row_units.empty()) {
    share_out(o.row_units, row_workers, 2, 2, 1, &o.row_pieces, &o.row_off, &first);
    finish(o.row_units, o.row_pieces, first, true);
  }

  // The rows of a query and head that have something to join, or no key at all; cut where one of the query's
  // layers begins a new tile, and at `most` rows.
  const size_t fold_segs = o.segs.size();
  auto join = [&](uint32_t most) {
    o.segs.resize(fold_segs);
    o.join.clear();
    o.join_stride = 0;
    for (uint32_t t = 0; t < T; ++t) {
      const uint32_t* ls = o.tok_layer.data() + o.tok_off[t];
      const uint32_t nl = o.tok_off[t + 1] - o.tok_off[t];
      for (uint32_t i = 0, n; i < g; i += n) {
        n = std::min(g - i, most);
        for (uint32_t l = 0; l < nl; ++l) {
          const Layer& ly = o.layers[ls[l]];
          n = std::min(n, ly.tile_rows - ((t - ly.query0) * g + i) % ly.tile_rows);
        }
        for (uint32_t h = 0; h < H; ++h) {
          const uint32_t seg0 = (uint32_t)o.segs.size();
          bool direct = false;
          for (uint32_t l = 0; l < nl; ++l) {
            const Layer& ly = o.layers[ls[l]];
            const uint32_t r = (t - ly.query0) * g + i;
            const Group& gr = o.groups[ly.group0 + r / ly.tile_rows * H + h];
            direct = direct || gr.part_row == kDirect;
            if (gr.nparts) o.segs.push_back(JoinSeg{gr.part_row + r % ly.tile_rows, ly.tile_rows, gr.nparts});
          }
          if (direct) {
            o.segs.resize(seg0);
            continue;
          }
          o.join.push_back(JoinEntry{t, (uint16_t)(h * g + i), (uint16_t)n, seg0, (uint32_t)o.segs.size() - seg0});
          o.join_stride = std::max(o.join_stride, n);
        }
      }
    }
  };
  join(g);
  // A few entries of many rows among many that the row kernel's tiles cut: rows without work are not worth their place.
  if (o.join_stride > (uint32_t)kSmallRows) {
    uint64_t cut = 0;
    for (const JoinEntry& e : o.join) cut += (e.count + kSmallRows - 1) / kSmallRows;
    if (cut * kSmallRows < join_rows(o)) join(kSmallRows);
  }
}

}  // namespace pskv
