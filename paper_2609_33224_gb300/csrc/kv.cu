// C entry points of the serving operators (packserve_kv.h): the block cache, and the plans that lay a
// batch's spans out for the attention kernels.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>
#include <string>
#include <vector>

#include "kv_internal.cuh"

using pskv::Fold;
using pskv::JoinEntry;
using pskv::JoinSeg;
using pskv::Piece;

struct ps_kv {
  int device = 0;
  int sms = 0;
  uint32_t heads = 0, D = 0;
  int fmt = 0;
  uint64_t blocks = 0;
  uint8_t* pool = nullptr;
  uint32_t* err_host = nullptr;  // mapped: kernels set bits, the next call reads them
  uint32_t* err_dev = nullptr;
  std::string err;
};

struct ps_kv_plan {
  ps_kv* kv = nullptr;
  uint32_t q_heads = 0, group = 0, max_queries = 0, max_spans = 0;
  uint64_t max_blocks = 0;
  // Two buffers take turns, so that a set can prepare the next step while calls still read the last one.
  struct Buffer {
    uint8_t* dev = nullptr;
    uint8_t* host = nullptr;
    size_t cap = 0;
    cudaEvent_t used = nullptr;  // after the last call that read it
    bool in_use = false;
    cudaStream_t last = nullptr;
  } buf[2];
  int cur = 0;
  bool set = false, frozen = false;
  cudaStream_t copy = nullptr;
  pskv::PlanDev dev{};
  uint32_t queries = 0;
  uint64_t part_rows = 0;
  uint32_t top_block = 0;

  // rows of the tile kernel's tiles for a span of so many rows
  uint32_t tile_rows(uint32_t rows) const {
    const uint32_t full = (uint32_t)pskv::tile_rows_of((int)kv->D);
    return rows <= full / 2 ? full / 2 : full;
  }
};

namespace {

ps_status fail(ps_kv* kv, ps_status s, const char* msg) {
  try {
    kv->err = msg;
  } catch (...) {
    kv->err.clear();
  }
  return s;
}
ps_status fail_cuda(ps_kv* kv, const char* what, cudaError_t e) {
  try {
    kv->err = std::string(what) + ": " + cudaGetErrorString(e);
  } catch (...) {
    kv->err.clear();
  }
  return PS_ERR_CUDA;
}
#define KV_CUDA(kv, call)                                       \
  do {                                                          \
    const cudaError_t e_ = (call);                              \
    if (e_ != cudaSuccess) return fail_cuda((kv), #call, e_);   \
  } while (0)

// Makes the cache's device current for a call.
struct OnDevice {
  int was = -1;
  explicit OnDevice(int d) {
    int c = -1;
    if (cudaGetDevice(&c) == cudaSuccess && c != d && cudaSetDevice(d) == cudaSuccess) was = c;
  }
  ~OnDevice() {
    if (was >= 0) cudaSetDevice(was);
  }
};

// What kernels have reported since the last report.
ps_status reported(ps_kv* kv) {
  if (__atomic_load_n(kv->err_host, __ATOMIC_RELAXED) == 0) return PS_OK;
  const uint32_t e = __atomic_exchange_n(kv->err_host, 0u, __ATOMIC_ACQ_REL);
  if (e & pskv::kErrWait)
    return fail(kv, PS_ERR_TIMEOUT, "a bounded device-side wait of an earlier attention call gave up");
  return fail(kv, PS_ERR_INVALID, "an earlier write or read named a slot outside the cache");
}

size_t elem_size(int type) { return type == PS_KV_FP32 ? 4 : 2; }

const char* rows_error(const ps_kv_rows* r, uint32_t heads, uint64_t n) {
  if (!r) return "a tensor is NULL";
  if (r->type != PS_KV_BF16 && r->type != PS_KV_FP16 && r->type != PS_KV_FP32)
    return "element type must be PS_KV_BF16, PS_KV_FP16 or PS_KV_FP32";
  if (n == 0) return nullptr;
  if (!r->data) return "a tensor's data is NULL";
  const size_t sz = elem_size(r->type);
  if (reinterpret_cast<uintptr_t>(r->data) % 16) return "tensors must start on a 16-byte boundary";
  if ((n > 1 && (r->token_stride * (int64_t)sz) % 16) || (heads > 1 && (r->head_stride * (int64_t)sz) % 16))
    return "token and head strides must be multiples of 16 bytes";
  return nullptr;
}

ps_status store_args(ps_kv* kv, const ps_kv_rows* k, const ps_kv_rows* v, const int64_t* slots, uint64_t n,
                     pskv::StoreArgs* a) {
  const char* m = rows_error(k, kv->heads, n);
  if (!m) m = rows_error(v, kv->heads, n);
  if (!m && k->type != v->type) m = "k and v must have one element type";
  if (!m && n > 0 && !slots) m = "slots is NULL";
  if (!m && n > 0 && reinterpret_cast<uintptr_t>(slots) % 8) m = "slots must start on an 8-byte boundary";
  if (!m && n > (1ull << 40)) m = "too many tokens";
  if (m) return fail(kv, PS_ERR_INVALID, m);
  *a = pskv::StoreArgs{kv->pool,         slots,          n,
                       kv->blocks * pskv::kBlock, kv->heads, k->data, v->data, k->token_stride, k->head_stride,
                       v->token_stride,  v->head_stride, kv->err_dev};
  return PS_OK;
}

// ---- planning -----------------------------------------------------------------------------------------

using pskv::kBlock;
using pskv::kSmallRows;
using pskv::kTileKeys;

// Which kernel takes the rows of a tile and head over the keys that all of them see: the one that adds less time to
// the batch.  Nanoseconds of the whole GPU, from spans of 24 to 256 rows on 512 to 65536 keys: the row kernel per 16
// rows and 16 keys, the tile kernel per step of 128 keys, a piece of it costing three steps more; the tile kernel
// adds kTileLaunch to a call.  In front of a causal span's end, of which the row kernel has a short piece per 16 rows
// anyway, its blocks cost about four times as much, as its pieces then are of uneven lengths (192 new tokens on 16384:
// 457 us, 500 without this).  By tiles / by rows, us, one span of 8 key/value heads: bf16 with head_dim 128,
// 128 rows on 512 keys 10.9/11.2, on 4096 16.7/19.0, 64 rows on 2048 12.0/10.3, on 16384 22.7/24.7, 32 rows on 16384
// 22.4/18.8; fp8, 64 rows on 4096 15.5/16.3; bf16 with head_dim 64, 64 rows on 4096 9.1/10.3.
constexpr double kTileLaunch = 1000.0;
double tile_saves(const ps_kv& kv, uint32_t rows, int64_t keys, bool causal) {
  const bool fp8 = kv.fmt == PS_KV_FP8;
  const double block = (kv.D == 128 ? (fp8 ? 0.73 : 0.51) : (fp8 ? 0.50 : 0.40)) * (causal && rows > (uint32_t)kSmallRows ? 4 : 1);
  const double step = kv.D == 128 ? (fp8 ? 18.0 : 16.0) : (fp8 ? 9.0 : 8.0);
  const double by_rows = block * ((rows + kSmallRows - 1) / kSmallRows) * (double)((keys + kBlock - 1) / kBlock);
  return by_rows - step * (double)((keys + kTileKeys - 1) / kTileKeys + 3);
}

// From so many steps on, a piece of one tile of rows runs as two.  64 rows on 65536 tokens: 65 us, 79 as one; on
// 1024 (2 steps a piece), where the second result costs more than it brings, 11.4 and 11.0.  With head_dim 64,
// whose steps are half as long, it brought nothing (35 and 34 us).
constexpr uint32_t kSplitSteps = 8;

// A piece of the row kernel joins up to this many tile parts into its rows, where a worker has at least so many
// units of rows that the time this takes evens out.  192 new tokens on 16384 (4 units a worker, 2 to 3 parts):
// 456 us, 491 with the join kernel; 256 queries on 32768 (1 unit a worker, 3 parts) 288 and 277 us, 64 on 8192
// (10 parts) 92 and 60.
constexpr size_t kFoldMost = 3, kFoldUnits = 3;

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
};

// A unit of the layer and group that come last.
Unit unit(const ps_kv_span& s, uint32_t r0, uint32_t nr, uint32_t h, int64_t from, int64_t end, int step, int32_t climit,
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
void share_out(const std::vector<Unit>& units, uint32_t most, uint32_t extra, uint32_t least, uint32_t step_blocks,
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
        p.key0 += done * step_blocks * pskv::kBlock;
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

void lay_out(const ps_kv_plan& pl, uint32_t T, const ps_kv_span* spans, uint32_t n_spans, Layout* out) {
  Layout& o = *out;
  const uint32_t H = pl.kv->heads, g = pl.group;
  // The keys that all rows of a tile see, where the tile kernel is the one to take them (else 0).
  auto cut_of = [&](const ps_kv_span& s, uint32_t r0, uint32_t nr) -> int64_t {
    int64_t c = (int64_t)s.length;
    if (s.causal) c = std::max<int64_t>(0, c - (int64_t)s.num_queries + r0 / g + 1) / kBlock * kBlock;
    return tile_saves(*pl.kv, nr, c, s.causal != 0) > 0 ? c : 0;
  };
  auto tiles_save = [&](const ps_kv_span& s) {
    double sum = 0;
    const uint32_t rows = s.num_queries * g, tr = pl.tile_rows(rows);
    for (uint32_t r0 = 0; r0 < rows; r0 += tr) {
      const uint32_t nr = std::min(rows - r0, tr);
      const int64_t c = cut_of(s, r0, nr);
      if (c > 0) sum += tile_saves(*pl.kv, nr, c, s.causal != 0) * H;
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
    const int32_t climit = s.causal ? (int32_t)(len - (int64_t)s.num_queries) : pskv::kNoLimit;

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
          if (c > 0) o.tile_units.push_back(unit(s, r0, nr, h, 0, c, kTileKeys, pskv::kNoLimit, tile_rows, o));
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
  const uint32_t row_workers = (uint32_t)(pl.kv->sms * pskv::row_warps_of(pl.kv->fmt));
  const bool may_fold = o.row_units.size() >= kFoldUnits * row_workers;
  auto finish = [&](std::vector<Unit>& units, std::vector<Piece>& pieces, std::vector<uint32_t>& first, bool rows) {
    for (size_t i = 0; i < units.size(); ++i) {
      const uint32_t a = first[i], b = i + 1 < units.size() ? first[i + 1] : (uint32_t)pieces.size();
      const Piece& p = units[i].p;
      // a tile piece that is split by steps has two parts
      uint32_t nparts = 0;
      for (uint32_t k = a; k < b; ++k) {
        if (!rows && pl.kv->D == 128 && p.nrows <= pskv::tile_rows_of(128) / 2 && pieces[k].nblocks >= kSplitSteps)
          pieces[k].split = units[i].tile_rows;
        nparts += pieces[k].split ? 2 : 1;
      }
      bool direct = nparts == 1;
      for (uint32_t q = p.row0 / g; direct && q <= (p.row0 + p.nrows - 1) / g; ++q) direct = alone[p.query0 + q];
      if (!direct && rows && may_fold && nparts == 1) direct = fold(units[i], &pieces[a]);
      Group& gr = o.groups[units[i].group];
      if (direct) {
        gr = Group{pskv::kDirect, 1};
        pieces[a].part_row = pskv::kDirect;
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
    const uint32_t workers = (uint32_t)(pl.kv->sms / pskv::tile_ctas_of((int)pl.kv->D));
    share_out(o.tile_units, workers, 4, 2, kTileKeys / kBlock, &o.tile_pieces, &o.tile_off, &first);
    finish(o.tile_units, o.tile_pieces, first, false);
  }
  if (!o.row_units.empty()) {
    share_out(o.row_units, row_workers, 2, 2, 1, &o.row_pieces, &o.row_off, &first);
    finish(o.row_units, o.row_pieces, first, true);
  }

  // The rows of a query and head that have something to join, or no key at all; cut where one of the query's
  // layers begins a new tile.
  for (uint32_t t = 0; t < T; ++t) {
    const uint32_t* ls = o.tok_layer.data() + o.tok_off[t];
    const uint32_t nl = o.tok_off[t + 1] - o.tok_off[t];
    for (uint32_t i = 0, n; i < g; i += n) {
      n = g - i;
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
          direct = direct || gr.part_row == pskv::kDirect;
          if (gr.nparts) o.segs.push_back(JoinSeg{gr.part_row + r % ly.tile_rows, ly.tile_rows, gr.nparts});
        }
        if (direct) {
          o.segs.resize(seg0);
          continue;
        }
        o.join.push_back(JoinEntry{t, (uint16_t)(h * g + i), (uint16_t)n, seg0, (uint32_t)o.segs.size() - seg0});
      }
    }
  }
}

template <class T>
size_t place(std::vector<std::pair<const void*, size_t>>* parts, size_t* at, const std::vector<T>& v) {
  const size_t here = *at;
  parts->emplace_back(v.data(), v.size() * sizeof(T));
  *at += (v.size() * sizeof(T) + 255) / 256 * 256;
  return here;
}

void release(ps_kv_plan::Buffer& b) {
  if (b.in_use) cudaEventSynchronize(b.used);
  if (b.used) cudaEventDestroy(b.used);
  if (b.dev) cudaFree(b.dev);
  if (b.host) cudaFreeHost(b.host);
  b = ps_kv_plan::Buffer{};
}

ps_status grow(ps_kv* kv, ps_kv_plan::Buffer& b, size_t need) {
  if (need <= b.cap) return PS_OK;
  size_t cap = std::max<size_t>(b.cap * 2, 1 << 16);
  while (cap < need) cap *= 2;
  if (b.dev) cudaFree(b.dev);
  if (b.host) cudaFreeHost(b.host);
  b.dev = b.host = nullptr;
  b.cap = 0;
  cudaError_t e = cudaMalloc(&b.dev, cap);
  if (e == cudaSuccess) e = cudaHostAlloc(&b.host, cap, cudaHostAllocDefault);
  if (e != cudaSuccess) {
    cudaGetLastError();
    if (b.dev) cudaFree(b.dev);
    b.dev = b.host = nullptr;
    return fail(kv, e == cudaErrorMemoryAllocation ? PS_ERR_OOM : PS_ERR_CUDA, "plan buffers could not be allocated");
  }
  b.cap = cap;
  return PS_OK;
}

ps_status plan_set(ps_kv_plan* pl, uint32_t T, const ps_kv_span* spans, uint32_t n_spans, const uint32_t* blocks,
                   uint64_t n_blocks) {
  ps_kv* kv = pl->kv;
  pl->set = false;
  if (T > pl->max_queries) return fail(kv, PS_ERR_INVALID, "more queries than max_queries");
  if (n_spans > pl->max_spans) return fail(kv, PS_ERR_INVALID, "more spans than max_spans");
  if (n_blocks > pl->max_blocks) return fail(kv, PS_ERR_INVALID, "more block ids than max_blocks");
  if ((n_spans && !spans) || (n_blocks && !blocks)) return fail(kv, PS_ERR_INVALID, "spans or blocks is NULL");
  for (uint32_t i = 0; i < n_spans; ++i) {
    const ps_kv_span& s = spans[i];
    if (s.causal > 1) return fail(kv, PS_ERR_INVALID, "a span's causal must be 0 or 1");
    if (s.first_query > T || s.num_queries > T - s.first_query)
      return fail(kv, PS_ERR_INVALID, "a span's queries must lie inside the batch");
    if (s.length >= (1ull << 30)) return fail(kv, PS_ERR_INVALID, "a span's length must be < 2^30");
    const uint64_t nb = (s.length + pskv::kBlock - 1) / pskv::kBlock;
    if (s.first_block > n_blocks || nb > n_blocks - s.first_block)
      return fail(kv, PS_ERR_INVALID, "a span's blocks must lie inside the block array");
  }
  uint32_t top = 0;
  for (uint64_t i = 0; i < n_blocks; ++i) top = std::max(top, blocks[i]);
  if (n_blocks && top >= kv->blocks) return fail(kv, PS_ERR_INVALID, "a block id lies outside the cache");

  Layout o;
  lay_out(*pl, T, spans, n_spans, &o);
  if (o.part_rows >= 0xFFFFFF00ull || o.groups.size() >= 0xFFFFFF00ull)
    return fail(kv, PS_ERR_INVALID, "the batch is too large for one plan");

  std::vector<std::pair<const void*, size_t>> parts;
  size_t at = 0;
  const size_t rp = place(&parts, &at, o.row_pieces), ro = place(&parts, &at, o.row_off);
  const size_t tp = place(&parts, &at, o.tile_pieces), to = place(&parts, &at, o.tile_off);
  const size_t jn = place(&parts, &at, o.join), sg = place(&parts, &at, o.segs), fd = place(&parts, &at, o.folds);
  const size_t bl = at;
  parts.emplace_back(blocks, n_blocks * sizeof(uint32_t));
  at += n_blocks * sizeof(uint32_t);

  ps_kv_plan::Buffer& b = pl->buf[pl->cur ^ 1];
  if (b.in_use) {
    KV_CUDA(kv, cudaEventSynchronize(b.used));
    b.in_use = false;
  }
  const ps_status st = grow(kv, b, at);
  if (st != PS_OK) return st;
  size_t w = 0;
  for (const auto& part : parts) {
    if (part.second) std::memcpy(b.host + w, part.first, part.second);
    w += (part.second + 255) / 256 * 256;
  }
  if (at) KV_CUDA(kv, cudaMemcpyAsync(b.dev, b.host, at, cudaMemcpyHostToDevice, pl->copy));
  KV_CUDA(kv, cudaStreamSynchronize(pl->copy));

  pskv::PlanDev d{};
  d.row_pieces = reinterpret_cast<const Piece*>(b.dev + rp);
  d.row_off = reinterpret_cast<const uint32_t*>(b.dev + ro);
  d.row_workers = o.row_off.empty() ? 0 : (uint32_t)o.row_off.size() - 1;
  d.row_ctas = std::min<uint32_t>(d.row_workers, (uint32_t)kv->sms);
  d.tile_pieces = reinterpret_cast<const Piece*>(b.dev + tp);
  d.tile_off = reinterpret_cast<const uint32_t*>(b.dev + to);
  d.tile_workers = o.tile_off.empty() ? 0 : (uint32_t)o.tile_off.size() - 1;
  d.join = reinterpret_cast<const JoinEntry*>(b.dev + jn);
  d.segs = reinterpret_cast<const JoinSeg*>(b.dev + sg);
  d.folds = reinterpret_cast<const Fold*>(b.dev + fd);
  d.njoin = (uint32_t)o.join.size();
  d.max_parts = o.max_parts;
  d.blocks = reinterpret_cast<const uint32_t*>(b.dev + bl);
  pl->dev = d;
  pl->cur ^= 1;
  pl->queries = T;
  pl->part_rows = o.part_rows;
  pl->top_block = n_blocks ? top : 0;
  pl->set = true;
  return PS_OK;
}

uint64_t workspace_bytes(const ps_kv_plan* pl) {
  const uint64_t ml = (pl->part_rows * sizeof(float2) + 255) / 256 * 256;
  return ml + pl->part_rows * pl->kv->D * sizeof(float);
}

}  // namespace

extern "C" {

ps_status ps_kv_create(const ps_kv_config* cfg, ps_kv** out) {
  if (!cfg || !out) return PS_ERR_INVALID;
  *out = nullptr;
  if (cfg->kv_heads < 1 || cfg->kv_heads > 1024 || cfg->num_blocks < 1 || cfg->num_blocks > 0xFFFFFFFFull ||
      (cfg->head_dim != 64 && cfg->head_dim != 128) || cfg->format < PS_KV_BF16 || cfg->format > PS_KV_FP8)
    return PS_ERR_INVALID;
  int count = 0;
  if (cudaGetDeviceCount(&count) != cudaSuccess || count < 1) {
    cudaGetLastError();
    return PS_ERR_CUDA;
  }
  if (cfg->device < 0 || cfg->device >= count) return PS_ERR_INVALID;
  ps_kv* kv = new (std::nothrow) ps_kv;
  if (!kv) return PS_ERR_OOM;
  kv->device = cfg->device;
  kv->heads = cfg->kv_heads;
  kv->D = cfg->head_dim;
  kv->fmt = cfg->format;
  kv->blocks = cfg->num_blocks;
  OnDevice on(kv->device);
  const uint64_t bytes = kv->blocks * kv->heads * (uint64_t)pskv::record_bytes((int)kv->D, kv->fmt);
  void* dev = nullptr;
  cudaError_t e = cudaDeviceGetAttribute(&kv->sms, cudaDevAttrMultiProcessorCount, kv->device);
  if (e == cudaSuccess) e = cudaMalloc(&kv->pool, bytes);
  if (e == cudaSuccess) e = cudaMemset(kv->pool, 0, bytes);
  if (e == cudaSuccess) e = cudaHostAlloc(&kv->err_host, 64, cudaHostAllocMapped);
  if (e == cudaSuccess) {
    std::memset(kv->err_host, 0, 64);
    e = cudaHostGetDevicePointer(&dev, kv->err_host, 0);
  }
  if (e == cudaSuccess) e = pskv::prepare_rows((int)kv->D, kv->fmt);
  if (e == cudaSuccess) e = pskv::prepare_tiles((int)kv->D, kv->fmt);
  if (e == cudaSuccess) e = cudaDeviceSynchronize();
  kv->err_dev = static_cast<uint32_t*>(dev);
  if (e != cudaSuccess) {
    cudaGetLastError();
    ps_kv_destroy(kv);
    return e == cudaErrorMemoryAllocation ? PS_ERR_OOM : PS_ERR_CUDA;
  }
  *out = kv;
  return PS_OK;
}

ps_status ps_kv_write(ps_kv* kv, const ps_kv_rows* k, const ps_kv_rows* v, const int64_t* slots, uint64_t n, void* stream) {
  if (!kv) return PS_ERR_INVALID;
  ps_status st = reported(kv);
  if (st != PS_OK) return st;
  pskv::StoreArgs a;
  st = store_args(kv, k, v, slots, n, &a);
  if (st != PS_OK || n == 0) return st;
  OnDevice on(kv->device);
  KV_CUDA(kv, pskv::launch_write((int)kv->D, kv->fmt, k->type, a, kv->sms, static_cast<cudaStream_t>(stream)));
  return PS_OK;
}

ps_status ps_kv_read(ps_kv* kv, const int64_t* slots, uint64_t n, const ps_kv_rows* k, const ps_kv_rows* v, void* stream) {
  if (!kv) return PS_ERR_INVALID;
  ps_status st = reported(kv);
  if (st != PS_OK) return st;
  pskv::StoreArgs a;
  st = store_args(kv, k, v, slots, n, &a);
  if (st != PS_OK || n == 0) return st;
  OnDevice on(kv->device);
  KV_CUDA(kv, pskv::launch_read((int)kv->D, kv->fmt, k->type, a, kv->sms, static_cast<cudaStream_t>(stream)));
  return PS_OK;
}

ps_status ps_kv_check(ps_kv* kv, void* stream) {
  if (!kv) return PS_ERR_INVALID;
  OnDevice on(kv->device);
  KV_CUDA(kv, cudaStreamSynchronize(static_cast<cudaStream_t>(stream)));
  return reported(kv);
}

ps_status ps_kv_plan_create(ps_kv* kv, uint32_t q_heads, uint32_t max_queries, uint32_t max_spans, uint64_t max_blocks,
                            ps_kv_plan** out) {
  if (!kv) return PS_ERR_INVALID;
  if (!out) return fail(kv, PS_ERR_INVALID, "out is NULL");
  *out = nullptr;
  if (q_heads < 1 || q_heads > 65535 || q_heads % kv->heads)
    return fail(kv, PS_ERR_INVALID, "q_heads must be a multiple of kv_heads, at most 65535");
  if (max_queries < 1 || (uint64_t)max_queries * q_heads >= (1ull << 30))
    return fail(kv, PS_ERR_INVALID, "max_queries must be at least 1 and max_queries * q_heads < 2^30");
  if (max_blocks >= (1ull << 32)) return fail(kv, PS_ERR_INVALID, "max_blocks must be < 2^32");
  ps_kv_plan* pl = new (std::nothrow) ps_kv_plan;
  if (!pl) return fail(kv, PS_ERR_OOM, "no host memory for a plan");
  pl->kv = kv;
  pl->q_heads = q_heads;
  pl->group = q_heads / kv->heads;
  pl->max_queries = max_queries;
  pl->max_spans = max_spans;
  pl->max_blocks = max_blocks;
  OnDevice on(kv->device);
  cudaError_t e = cudaStreamCreateWithFlags(&pl->copy, cudaStreamNonBlocking);
  for (int i = 0; i < 2 && e == cudaSuccess; ++i) e = cudaEventCreateWithFlags(&pl->buf[i].used, cudaEventDisableTiming);
  ps_status st = PS_OK;
  for (int i = 0; i < 2 && e == cudaSuccess && st == PS_OK; ++i) st = grow(kv, pl->buf[i], max_blocks * 4 + max_spans * 256);
  if (e != cudaSuccess || st != PS_OK) {
    ps_kv_plan_destroy(pl);
    return e != cudaSuccess ? fail_cuda(kv, "ps_kv_plan_create", e) : st;
  }
  *out = pl;
  return PS_OK;
}

ps_status ps_kv_plan_set(ps_kv_plan* pl, uint32_t num_queries, const ps_kv_span* spans, uint32_t num_spans,
                         const uint32_t* blocks, uint64_t num_blocks) {
  if (!pl) return PS_ERR_INVALID;
  if (pl->frozen) return fail(pl->kv, PS_ERR_STATE, "a CUDA graph holds this plan's arrays: make another plan");
  OnDevice on(pl->kv->device);
  try {
    return plan_set(pl, num_queries, spans, num_spans, blocks, num_blocks);
  } catch (...) {
    pl->set = false;
    return fail(pl->kv, PS_ERR_OOM, "no host memory for the plan");
  }
}

ps_status ps_kv_plan_workspace(ps_kv_plan* pl, uint64_t* bytes) {
  if (!pl) return PS_ERR_INVALID;
  if (!bytes) return fail(pl->kv, PS_ERR_INVALID, "bytes is NULL");
  if (!pl->set) return fail(pl->kv, PS_ERR_STATE, "no batch is set");
  *bytes = workspace_bytes(pl);
  return PS_OK;
}

ps_status ps_kv_attend(ps_kv* kv, ps_kv_plan* pl, const ps_kv_rows* q, const ps_kv_rows* out, float* lse, float scale,
                       void* workspace, uint64_t bytes, void* stream) {
  if (!kv) return PS_ERR_INVALID;
  ps_status st = reported(kv);
  if (st != PS_OK) return st;
  if (!pl) return fail(kv, PS_ERR_INVALID, "plan is NULL");
  if (!pl->set) return fail(kv, PS_ERR_STATE, "no batch is set");
  if (kv != pl->kv && (kv->device != pl->kv->device || kv->heads != pl->kv->heads || kv->D != pl->kv->D ||
                       kv->fmt != pl->kv->fmt || kv->blocks <= pl->top_block))
    return fail(kv, PS_ERR_INVALID, "the plan was made for a cache of another shape");
  const uint32_t T = pl->queries;
  const char* m = rows_error(q, pl->q_heads, T);
  if (!m) m = rows_error(out, pl->q_heads, T);
  const int want = kv->fmt == PS_KV_FP16 ? PS_KV_FP16 : PS_KV_BF16;
  if (!m && (q->type != want || out->type != want)) m = "q and out must have the cache's 16-bit type (bf16 with fp8)";
  if (!m && lse && reinterpret_cast<uintptr_t>(lse) % 4) m = "lse must start on a 4-byte boundary";
  if (!m && !std::isfinite(scale)) m = "scale must be finite";
  const uint64_t need = workspace_bytes(pl);
  if (!m && need && (!workspace || bytes < need)) m = "the workspace is smaller than ps_kv_plan_workspace says";
  if (!m && need && reinterpret_cast<uintptr_t>(workspace) % 256) m = "the workspace must start on a 256-byte boundary";
  if (m) return fail(kv, PS_ERR_INVALID, m);
  if (T == 0) return PS_OK;
  OnDevice on(kv->device);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaStreamCaptureStatus cap = cudaStreamCaptureStatusNone;
  KV_CUDA(kv, cudaStreamIsCapturing(s, &cap));
  ps_kv_plan::Buffer& b = pl->buf[pl->cur];
  const bool capturing = cap != cudaStreamCaptureStatusNone;
  if (capturing)
    pl->frozen = true;
  else if (b.in_use && b.last != s)  // so that the last call's event stands for all calls before it
    KV_CUDA(kv, cudaStreamWaitEvent(s, b.used, 0));

  pskv::AttnArgs a{};
  a.pool = kv->pool;
  a.q = static_cast<const uint16_t*>(q->data);
  a.q_tok = q->token_stride;
  a.q_head = q->head_stride;
  a.out = static_cast<uint16_t*>(out->data);
  a.o_tok = out->token_stride;
  a.o_head = out->head_stride;
  a.lse = lse;
  a.part_ml = static_cast<float2*>(workspace);
  a.part = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + (need - pl->part_rows * kv->D * sizeof(float)));
  a.kv_heads = kv->heads;
  a.group = pl->group;
  a.scale_log2 = scale * 1.4426950408889634f;
  a.err = kv->err_dev;
  const int D = (int)kv->D;
  cudaError_t e = cudaSuccess;
  if (pl->dev.tile_workers) e = pskv::launch_tiles(D, kv->fmt, a, pl->dev, s);
  if (e == cudaSuccess && pl->dev.row_workers) e = pskv::launch_rows(D, kv->fmt, a, pl->dev, pl->dev.tile_workers != 0, s);
  if (e == cudaSuccess && pl->dev.njoin) e = pskv::launch_join(D, kv->fmt == PS_KV_FP16, a, pl->dev, s);
  if (!capturing) {  // also after a failed launch: the ones before it read the buffer
    const cudaError_t r = cudaEventRecord(b.used, s);
    if (r == cudaSuccess) {
      b.in_use = true;
      b.last = s;
    } else if (e == cudaSuccess) {
      e = r;
    }
  }
  if (e != cudaSuccess) return fail_cuda(kv, "ps_kv_attend", e);
  return PS_OK;
}

const char* ps_kv_last_error(const ps_kv* kv) { return kv ? kv->err.c_str() : ""; }

void ps_kv_plan_destroy(ps_kv_plan* pl) {
  if (!pl) return;
  OnDevice on(pl->kv->device);
  release(pl->buf[0]);
  release(pl->buf[1]);
  if (pl->copy) cudaStreamDestroy(pl->copy);
  delete pl;
}

void ps_kv_destroy(ps_kv* kv) {
  if (!kv) return;
  OnDevice on(kv->device);
  cudaDeviceSynchronize();
  if (kv->pool) cudaFree(kv->pool);
  if (kv->err_host) cudaFreeHost(kv->err_host);
  delete kv;
}

}  // extern "C"
