// C entry points of the serving operators (packserve_kv.h): the block cache, and the plans that lay a
// batch's spans out for the attention kernels.
#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstring>
#include <new>
#include <string>
#include <vector>

#include "kv_internal.cuh"

namespace {

// Memory of a cache or a plan.  A CUDA graph that has captured a call on it keeps it after its owner is gone: each such
// graph holds a reference.
struct Memory {
  std::atomic<uint32_t> refs{1};
  int device = 0;
  uint8_t* dev = nullptr;
  void* host = nullptr;             // pinned
  unsigned long long capture = 0;   // the last one whose graph has a reference
  Memory* next = nullptr;
};

}  // namespace

struct ps_kv {
  int device = 0;
  int sms = 0;
  uint32_t heads = 0, D = 0;
  int fmt = 0;
  uint64_t blocks = 0;
  Memory* mem = nullptr;  // the blocks, and the error word
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
    Memory* mem = nullptr;
    uint8_t* dev = nullptr;
    uint8_t* host = nullptr;
    size_t cap = 0;
    cudaEvent_t used = nullptr;  // after the calls that read it, once recorded
    bool in_use = false, recorded = false;
    cudaStream_t last = nullptr;  // of the last such call, which comes after all others
  } buf[2];
  int cur = 0;
  bool set = false;
  cudaStream_t copy = nullptr;
  pskv::PlanDev dev{};
  uint32_t queries = 0;
  uint64_t part_rows = 0;
  uint32_t top_block = 0;
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

// Memory that nothing refers to any more.  It is freed by a later call: the one that gives up a graph's reference
// may not call CUDA.
std::atomic<Memory*> unused{nullptr};

void drop(void* p) {
  Memory* m = static_cast<Memory*>(p);
  if (m->refs.fetch_sub(1, std::memory_order_acq_rel) != 1) return;
  m->next = unused.load(std::memory_order_relaxed);
  while (!unused.compare_exchange_weak(m->next, m, std::memory_order_release, std::memory_order_relaxed)) {
  }
}

void free_unused() {
  Memory* m = unused.exchange(nullptr, std::memory_order_acquire);
  while (m) {
    Memory* next = m->next;
    OnDevice on(m->device);
    if (m->dev) cudaFree(m->dev);
    if (m->host) cudaFreeHost(m->host);
    delete m;
    m = next;
  }
}

// The graph that a call on the stream is captured into (0: none), and a reference to memory from it.
struct Capture {
  cudaStreamCaptureStatus status = cudaStreamCaptureStatusNone;
  unsigned long long id = 0;
  cudaGraph_t graph = nullptr;
  cudaError_t look(cudaStream_t s) { return cudaStreamGetCaptureInfo(s, &status, &id, &graph, nullptr, nullptr, nullptr); }
  bool on() const { return status != cudaStreamCaptureStatusNone; }
  cudaError_t keep(Memory* m) const {
    if (status != cudaStreamCaptureStatusActive || m->capture == id) return cudaSuccess;
    cudaUserObject_t o;
    m->refs.fetch_add(1, std::memory_order_relaxed);
    cudaError_t e = cudaUserObjectCreate(&o, m, drop, 1, cudaUserObjectNoDestructorSync);
    if (e != cudaSuccess) {
      drop(m);
      return e;
    }
    e = cudaGraphRetainUserObject(graph, o, 1, cudaGraphUserObjectMove);
    if (e != cudaSuccess)
      cudaUserObjectRelease(o, 1);  // drops the reference
    else
      m->capture = id;
    return e;
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

// Whether some two of n x heads rows of D elements overlap, which a result's must not.
bool rows_overlap(const ps_kv_rows* r, uint64_t n, uint32_t heads, uint32_t D) {
  using Wide = unsigned __int128;
  const auto size = [](int64_t x) { return x < 0 ? 0 - (uint64_t)x : (uint64_t)x; };
  if (n == 0) return false;
  uint64_t s0 = n > 1 ? size(r->token_stride) : 0, s1 = heads > 1 ? size(r->head_stride) : 0, c0 = n, c1 = heads;
  if (n > 1 && s0 < D) return true;
  if (heads > 1 && s1 < D) return true;
  if (n == 1 || heads == 1) return false;
  if (s0 > s1) {
    std::swap(s0, s1);
    std::swap(c0, c1);
  }
  // i rows of the wider stride on, the nearest of the narrower: none where all of those lie before the first of them
  const Wide extent = (Wide)(c0 - 1) * s0 + D;
  for (uint64_t i = 1; i < c1 && (Wide)i * s1 < extent; ++i) {
    const Wide j = (Wide)i * s1 / s0, rest = (Wide)i * s1 % s0;
    if ((j < c0 && rest < D) || (j + 1 < c0 && s0 - rest < D)) return true;
  }
  return false;
}

ps_status store_args(ps_kv* kv, const ps_kv_rows* k, const ps_kv_rows* v, const int64_t* slots, uint64_t n,
                     bool results, pskv::StoreArgs* a) {
  const char* m = rows_error(k, kv->heads, n);
  if (!m) m = rows_error(v, kv->heads, n);
  if (!m && k->type != v->type) m = "k and v must have one element type";
  if (!m && n > 0 && !slots) m = "slots is NULL";
  if (!m && n > 0 && reinterpret_cast<uintptr_t>(slots) % 8) m = "slots must start on an 8-byte boundary";
  if (!m && n > (1ull << 40)) m = "too many tokens";
  if (!m && results && (rows_overlap(k, n, kv->heads, kv->D) || rows_overlap(v, n, kv->heads, kv->D)))
    m = "rows of a result overlap";
  if (m) return fail(kv, PS_ERR_INVALID, m);
  *a = pskv::StoreArgs{kv->pool,         slots,          n,
                       kv->blocks * pskv::kBlock, kv->heads, k->data, v->data, k->token_stride, k->head_stride,
                       v->token_stride,  v->head_stride, kv->err_dev};
  return PS_OK;
}

template <class T>
size_t place(std::vector<std::pair<const void*, size_t>>* parts, size_t* at, const std::vector<T>& v) {
  const size_t here = *at;
  parts->emplace_back(v.data(), v.size() * sizeof(T));
  *at += (v.size() * sizeof(T) + 255) / 256 * 256;
  return here;
}

// Marks the end of the calls that have read a buffer so far.
cudaError_t mark_used(ps_kv_plan::Buffer& b) {
  if (!b.in_use || b.recorded) return cudaSuccess;
  const cudaError_t e = cudaEventRecord(b.used, b.last);
  b.recorded = e == cudaSuccess;
  return e;
}

void release(ps_kv_plan::Buffer& b) {
  if (mark_used(b) != cudaSuccess)
    cudaDeviceSynchronize();
  else if (b.in_use)
    cudaEventSynchronize(b.used);
  if (b.used) cudaEventDestroy(b.used);
  if (b.mem) drop(b.mem);
  b = ps_kv_plan::Buffer{};
}

ps_status grow(ps_kv* kv, ps_kv_plan::Buffer& b, size_t need) {
  if (b.mem && need <= b.cap) return PS_OK;
  size_t cap = std::max<size_t>(b.cap * 2, 1 << 16);
  while (cap < need) cap *= 2;
  if (b.mem) drop(b.mem);
  b.mem = nullptr;
  b.dev = b.host = nullptr;
  b.cap = 0;
  free_unused();
  Memory* m = new (std::nothrow) Memory;
  if (!m) return fail(kv, PS_ERR_OOM, "no host memory for a plan");
  m->device = kv->device;
  cudaError_t e = cudaMalloc(&m->dev, cap);
  if (e == cudaSuccess) e = cudaHostAlloc(&m->host, cap, cudaHostAllocDefault);
  if (e != cudaSuccess) {
    cudaGetLastError();
    drop(m);
    free_unused();
    return fail(kv, e == cudaErrorMemoryAllocation ? PS_ERR_OOM : PS_ERR_CUDA, "plan buffers could not be allocated");
  }
  b.mem = m;
  b.dev = m->dev;
  b.host = static_cast<uint8_t*>(m->host);
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
  uint64_t seen = 0;  // (query, layer) pairs of the layout: a span may become two layers
  for (uint32_t i = 0; i < n_spans; ++i) {
    const ps_kv_span& s = spans[i];
    if (s.causal > 1) return fail(kv, PS_ERR_INVALID, "a span's causal must be 0 or 1");
    if (s.first_query > T || s.num_queries > T - s.first_query)
      return fail(kv, PS_ERR_INVALID, "a span's queries must lie inside the batch");
    if (s.length >= (1ull << 30)) return fail(kv, PS_ERR_INVALID, "a span's length must be < 2^30");
    const uint64_t nb = (s.length + pskv::kBlock - 1) / pskv::kBlock;
    if (s.first_block > n_blocks || nb > n_blocks - s.first_block)
      return fail(kv, PS_ERR_INVALID, "a span's blocks must lie inside the block array");
    if (s.length) seen += 2ull * s.num_queries;
  }
  if (seen >= 0xFFFFFF00ull) return fail(kv, PS_ERR_INVALID, "the batch is too large for one plan");
  uint32_t top = 0;
  for (uint64_t i = 0; i < n_blocks; ++i) top = std::max(top, blocks[i]);
  if (n_blocks && top >= kv->blocks) return fail(kv, PS_ERR_INVALID, "a block id lies outside the cache");

  pskv::Layout o;
  pskv::lay_out(pskv::PlanShape{kv->sms, kv->D, kv->fmt, kv->heads, pl->group}, T, spans, n_spans, &o);
  if (o.part_rows >= 0xFFFFFF00ull || o.groups.size() >= 0xFFFFFF00ull || o.segs.size() >= 0xFFFFFF00ull ||
      pskv::join_rows(o) >= 0xFFFFFF00ull)
    return fail(kv, PS_ERR_INVALID, "the batch is too large for one plan");

  std::vector<std::pair<const void*, size_t>> parts;
  size_t at = 0;
  const size_t rp = place(&parts, &at, o.row_pieces), ro = place(&parts, &at, o.row_off);
  const size_t tp = place(&parts, &at, o.tile_pieces), to = place(&parts, &at, o.tile_off);
  const size_t jn = place(&parts, &at, o.join), sg = place(&parts, &at, o.segs), fd = place(&parts, &at, o.folds);
  const size_t bl = at;
  parts.emplace_back(blocks, n_blocks * sizeof(uint32_t));
  at += n_blocks * sizeof(uint32_t);

  // The calls of the set before keep reading their buffer: their end is marked now, while nothing else has been
  // queued behind them, and waited for when that buffer's turn comes.
  KV_CUDA(kv, mark_used(pl->buf[pl->cur]));
  ps_kv_plan::Buffer& b = pl->buf[pl->cur ^ 1];
  if (b.in_use) {
    KV_CUDA(kv, mark_used(b));
    KV_CUDA(kv, cudaEventSynchronize(b.used));
    b.in_use = b.recorded = false;
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
  d.row_pieces = reinterpret_cast<const pskv::Piece*>(b.dev + rp);
  d.row_off = reinterpret_cast<const uint32_t*>(b.dev + ro);
  d.row_workers = o.row_off.empty() ? 0 : (uint32_t)o.row_off.size() - 1;
  d.row_ctas = std::min<uint32_t>(d.row_workers, (uint32_t)o.row_sms);
  d.tile_pieces = reinterpret_cast<const pskv::Piece*>(b.dev + tp);
  d.tile_off = reinterpret_cast<const uint32_t*>(b.dev + to);
  d.tile_workers = o.tile_off.empty() ? 0 : (uint32_t)o.tile_off.size() - 1;
  d.join = reinterpret_cast<const pskv::JoinEntry*>(b.dev + jn);
  d.segs = reinterpret_cast<const pskv::JoinSeg*>(b.dev + sg);
  d.folds = reinterpret_cast<const pskv::Fold*>(b.dev + fd);
  d.njoin = (uint32_t)o.join.size();
  d.join_stride = o.join_stride;
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
  if (kv) kv->mem = new (std::nothrow) Memory;
  if (!kv || !kv->mem) {
    delete kv;
    return PS_ERR_OOM;
  }
  kv->device = kv->mem->device = cfg->device;
  kv->heads = cfg->kv_heads;
  kv->D = cfg->head_dim;
  kv->fmt = cfg->format;
  kv->blocks = cfg->num_blocks;
  OnDevice on(kv->device);
  const uint64_t bytes = kv->blocks * kv->heads * (uint64_t)pskv::record_bytes((int)kv->D, kv->fmt);
  void* dev = nullptr;
  free_unused();
  cudaError_t e = cudaDeviceGetAttribute(&kv->sms, cudaDevAttrMultiProcessorCount, kv->device);
  if (e == cudaSuccess) e = cudaMalloc(&kv->mem->dev, bytes);
  if (e == cudaSuccess) e = cudaMemset(kv->mem->dev, 0, bytes);
  if (e == cudaSuccess) e = cudaHostAlloc(&kv->mem->host, 64, cudaHostAllocMapped);
  kv->pool = kv->mem->dev;
  if (e == cudaSuccess) {
    kv->err_host = static_cast<uint32_t*>(kv->mem->host);
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

ps_status ps_kv_write(ps_kv* kv, const ps_kv_rows* k, const ps_kv_rows* v, const int64_t* slots, uint64_t n,
                      void* stream) {
  if (!kv) return PS_ERR_INVALID;
  ps_status st = reported(kv);
  if (st != PS_OK) return st;
  pskv::StoreArgs a;
  st = store_args(kv, k, v, slots, n, false, &a);
  if (st != PS_OK || n == 0) return st;
  OnDevice on(kv->device);
  Capture cap;
  KV_CUDA(kv, cap.look(static_cast<cudaStream_t>(stream)));
  KV_CUDA(kv, cap.keep(kv->mem));
  KV_CUDA(kv, pskv::launch_write((int)kv->D, kv->fmt, k->type, a, kv->sms, static_cast<cudaStream_t>(stream)));
  return PS_OK;
}

ps_status ps_kv_read(ps_kv* kv, const int64_t* slots, uint64_t n, const ps_kv_rows* k, const ps_kv_rows* v,
                     void* stream) {
  if (!kv) return PS_ERR_INVALID;
  ps_status st = reported(kv);
  if (st != PS_OK) return st;
  pskv::StoreArgs a;
  st = store_args(kv, k, v, slots, n, true, &a);
  if (st != PS_OK || n == 0) return st;
  OnDevice on(kv->device);
  Capture cap;
  KV_CUDA(kv, cap.look(static_cast<cudaStream_t>(stream)));
  KV_CUDA(kv, cap.keep(kv->mem));
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
  for (int i = 0; i < 2 && e == cudaSuccess && st == PS_OK; ++i)
    st = grow(kv, pl->buf[i], max_blocks * 4 + max_spans * 256);
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
  if (pl->buf[pl->cur].mem->refs.load(std::memory_order_acquire) > 1)  // the other buffer was last set before this one
    return fail(pl->kv, PS_ERR_STATE, "a CUDA graph holds this plan's arrays: make another plan");
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
  if (!m && rows_overlap(out, T, pl->q_heads, kv->D)) m = "rows of a result overlap";
  if (!m && lse && reinterpret_cast<uintptr_t>(lse) % 4) m = "lse must start on a 4-byte boundary";
  if (!m && !std::isfinite(scale)) m = "scale must be finite";
  const uint64_t need = workspace_bytes(pl);
  if (!m && need && (!workspace || bytes < need)) m = "the workspace is smaller than ps_kv_plan_workspace says";
  if (!m && need && reinterpret_cast<uintptr_t>(workspace) % 256) m = "the workspace must start on a 256-byte boundary";
  if (m) return fail(kv, PS_ERR_INVALID, m);
  if (T == 0) return PS_OK;
  OnDevice on(kv->device);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  Capture cap;
  KV_CUDA(kv, cap.look(s));
  ps_kv_plan::Buffer& b = pl->buf[pl->cur];
  const bool capturing = cap.on();
  if (capturing) {
    KV_CUDA(kv, cap.keep(kv->mem));
    KV_CUDA(kv, cap.keep(b.mem));
  } else if (b.in_use && b.last != s) {  // so that the last call's stream stands for all calls before it
    KV_CUDA(kv, mark_used(b));
    KV_CUDA(kv, cudaStreamWaitEvent(s, b.used, 0));
  }

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
  // In a graph the first kernel, the join of a batch without a key too, follows whatever node it has to: it takes the
  // plain dependency.
  a.rows_first = pl->dev.tile_workers == 0;
  if (pl->dev.tile_workers) e = pskv::launch_tiles(D, kv->fmt, a, pl->dev, !capturing, s);
  if (e == cudaSuccess && pl->dev.row_workers)
    e = pskv::launch_rows(D, kv->fmt, a, pl->dev, pl->dev.tile_workers != 0 || !capturing, s);
  if (e == cudaSuccess && pl->dev.njoin)
    e = pskv::launch_join(D, kv->fmt == PS_KV_FP16, a, pl->dev,
                          pl->dev.tile_workers || pl->dev.row_workers || !capturing, s);
  if (!capturing) {  // also after a failed launch: the ones before it read the buffer
    b.in_use = true;
    b.recorded = false;
    b.last = s;
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
  free_unused();
  delete pl;
}

void ps_kv_destroy(ps_kv* kv) {
  if (!kv) return;
  OnDevice on(kv->device);
  cudaDeviceSynchronize();
  drop(kv->mem);
  free_unused();
  delete kv;
}

}  // extern "C"
