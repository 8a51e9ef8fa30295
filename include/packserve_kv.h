/*
 * packserve_kv.h -- C ABI of the serving operators: the paged key/value cache whose 16-token blocks the
 * scheduler of packserve.h counts hits in, and attention of a batch over it.
 *
 * A request is sent to the instance that caches most of its prompt (Algorithm 1's KVC-first filter); the
 * instance then writes the request's new keys and values into blocks of its cache and attends to the
 * cached prefix and to them.  Requests of a batch mostly share their prefixes (the system prompt, a
 * session's history), so the attention takes the batch as spans: a span is a run of cached tokens and the
 * range of the batch's queries that see it.  A prefix that a range of requests shares is one span, read
 * and multiplied once for all of them; what a request has alone is a span of its own; nested prefixes are
 * nested spans.
 *
 * Conventions:
 *   - Every call returns a ps_status; on failure ps_kv_last_error() describes it.
 *   - ps_kv_write, ps_kv_write_rotated, ps_kv_read, ps_kv_move, ps_kv_copy_blocks, ps_kv_tree_mask, ps_kv_attend and
 *     ps_kv_attend_masked only enqueue work on the given stream (a cudaStream_t, NULL
 *     for the default stream) and return.  Their tensors are device memory of the cache's device, which
 *     must stay valid until that work is done; ordering between streams is the caller's.  What a kernel
 *     finds wrong (a slot outside the cache, a wait that gave up) is reported by the next call on the
 *     cache, or by ps_kv_check.
 *   - Tensors have their head_dim elements next to each other; token and head strides are free, in
 *     elements.  Base addresses are 16-byte aligned and strides multiples of 16 bytes.  Rows of a result do not
 *     overlap (rows that are read may: a stride of 0 repeats one).
 *   - Calls may be captured into a CUDA graph.  The graph keeps the cache's blocks and the plan's arrays that its calls
 *     read, also after ps_kv_destroy and ps_kv_plan_destroy; they are freed by the first ps_kv_create,
 *     ps_kv_plan_create, ps_kv_plan_destroy or ps_kv_destroy after the graph and its executable graphs are gone.  The
 *     caller's tensors and the workspace are the caller's to keep.
 *   - One cache or plan must not be used from two threads at once.
 */
#ifndef PACKSERVE_KV_H
#define PACKSERVE_KV_H

#include "packserve.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct ps_kv ps_kv;           /* opaque, owned by the library */
typedef struct ps_kv_plan ps_kv_plan; /* opaque, owned by the library */

/* Formats of the cached keys and values, and element types of the caller's tensors.
 * PS_KV_FP8: e4m3 codes with one power-of-two scale per (token, head) row, keys and values apart.  The
 * scale's exponent is the smallest e in [-110, 119] with max|x| <= 448 * 2^e (an infinity counts as the
 * largest finite float); a row is stored as the e4m3 numbers nearest to x * 2^-e (ties to even, magnitudes
 * above 448 as 448).  A row that holds a NaN reads back as NaN in every element.  Scales being powers of
 * two, every value of the cache is exact in bf16, and there is one rounding between x and the cache. */
enum { PS_KV_BF16 = 0, PS_KV_FP16 = 1, PS_KV_FP8 = 2, PS_KV_FP32 = 3 };

typedef struct {
  int32_t device;
  uint32_t kv_heads;   /* 1..1024 */
  uint64_t num_blocks; /* blocks of PS_BLOCK_TOKENS tokens, 1..2^32-1 */
  uint32_t head_dim;   /* 64 or 128 */
  int32_t format;      /* PS_KV_BF16, PS_KV_FP16 or PS_KV_FP8 */
} ps_kv_config;

/* rows x heads x head_dim elements */
typedef struct {
  void* data;
  int64_t token_stride; /* in elements */
  int64_t head_stride;
  int32_t type; /* PS_KV_BF16, PS_KV_FP16 or PS_KV_FP32 */
} ps_kv_rows;

/* One run of cached tokens and the queries that see it. */
typedef struct {
  uint32_t first_query; /* the queries first_query .. first_query + num_queries - 1 of the batch */
  uint32_t num_queries;
  uint64_t length; /* tokens, < 2^30; 0: the span has no key */
  /* 1: the span's last num_queries tokens are the queries' own: query first_query + i sees the tokens
   * j <= length - num_queries + i (none where that is negative).  0: every query sees every token. */
  uint32_t causal;
  uint64_t first_block; /* where the span's ceil(length / 16) block ids start in the plan's block array */
} ps_kv_span;

/* A cache of num_blocks blocks; its memory is allocated here and zeroed.  The paper's instances keep such
 * a cache (Section 7.1, the served engine's KV cache); the call itself has no counterpart.
 * Errors: PS_ERR_INVALID, PS_ERR_OOM, PS_ERR_CUDA (no object, so no message). */
PS_API ps_status ps_kv_create(const ps_kv_config* cfg, ps_kv** out);

/* Store n tokens' keys and values: row t of k and v goes to slot slots[t] (block slots[t] / 16, token
 * slots[t] % 16 in it) for every head.  slots: device array of n int64; a negative slot skips its token; a
 * slot past the cache is skipped and reported.  Slots of one call must be different (else it is undefined
 * which token a slot ends up with).  k and v have the same type.  The paper has no counterpart.
 * Errors: PS_ERR_INVALID (a NULL or misaligned array, a type or stride), PS_ERR_CUDA. */
PS_API ps_status ps_kv_write(ps_kv* kv, const ps_kv_rows* k, const ps_kv_rows* v, const int64_t* slots, uint64_t n,
                             void* stream);

/* Rotary positions.  Of a head's elements the first dims (a multiple of 16, at most head_dim) are taken in dims / 2
 * pairs (a, b): elements i and i + dims / 2, or with `interleaved` 2 i and 2 i + 1.  At position p pair i turns by
 * p * frequency[i] radians: (a, b) becomes magnitude * (a cos - b sin, b cos + a sin); the other elements stay.  A
 * frequency, of either sign, is held as a 64-bit fraction of a turn, and its product with the position wraps at a whole
 * turn, so that nothing but the frequency's own rounding grows with the position: an angle is off by no more than
 * |p| * (|frequency[i]| * 2^-52 + 2^-62). */
typedef struct {
  uint32_t dims;
  uint32_t interleaved; /* 0 or 1 */
  float magnitude;
  double frequency[64];
} ps_kv_rotary;

/* ps_kv_write of keys that are first rotated by positions[t] (device array of n int64, negative ones too), and the same
 * rotation of queries: row t of q (q_heads heads) goes to row t of q_out.  Rotation is in 32 bits, and what is stored is
 * rounded once; an fp8 row's scale is that of the row turned exactly by the angles as they are held, but where its maximum
 * is within 2^-26 of a border.  q, k and v have one element type; q_out the type that ps_kv_attend takes.  q and q_out:
 * both NULL (and q_heads 0) for keys alone; q_out may be q itself, and must not overlap it or k or v otherwise.  Queries
 * of tokens whose slot is negative or outside the cache are rotated all the same.  The paper has no counterpart.
 * Errors: as ps_kv_write. */
PS_API ps_status ps_kv_write_rotated(ps_kv* kv, const ps_kv_rotary* rotary, const int64_t* positions, const ps_kv_rows* q,
                                     const ps_kv_rows* q_out, uint32_t q_heads, const ps_kv_rows* k, const ps_kv_rows* v,
                                     const int64_t* slots, uint64_t n, void* stream);

/* Read n tokens back: k and v (of one type, rounded to it) receive the values that the cache holds at
 * slots[t]; a negative slot gives zeros, a slot past the cache zeros and a report.
 * The paper has no counterpart.  Errors: as ps_kv_write. */
PS_API ps_status ps_kv_read(ps_kv* kv, const int64_t* slots, uint64_t n, const ps_kv_rows* k, const ps_kv_rows* v,
                            void* stream);

/* Move n tokens inside the cache: the keys and values at slot src[i] go to slot dst[i], as they are held, all heads.  It is
 * as if every source were read before any slot is written: an accepted path of drafted tokens moves to the front of its
 * blocks, and slots may change places.  src, dst: device arrays of n int64.  A negative dst[i] skips the move, a
 * negative src[i] clears dst[i] to zeros; where either lies past the cache, the move is skipped and reported.  Slots of
 * dst must be different.  workspace: as ps_kv_attend's, of the bytes that ps_kv_move_workspace gives (0 possible).
 * The paper has no counterpart.  Errors: PS_ERR_INVALID, PS_ERR_CUDA. */
PS_API ps_status ps_kv_move(ps_kv* kv, const int64_t* src, const int64_t* dst, uint64_t n, void* workspace,
                            uint64_t workspace_bytes, void* stream);

/* Bytes of workspace that ps_kv_move needs for n tokens.  The paper has no counterpart. */
PS_API ps_status ps_kv_move_workspace(ps_kv* kv, uint64_t n, uint64_t* bytes);

/* Copy n whole blocks of `from` (which may be kv, or another cache of the same device, heads, head_dim and format) to
 * blocks of kv: src[i] to dst[i] (device arrays of n int64).  A request is forked so at its open block, or a chain is
 * handed to another cache.  A negative src[i] clears dst[i] to zeros, a negative dst[i] skips the copy; a block past its
 * cache skips it and is reported by kv.  A block may be copied to many places.  Blocks of dst must be different, and where
 * from is kv, none of them may be another copy's source.  The paper has no counterpart.
 * Errors: PS_ERR_INVALID, PS_ERR_CUDA. */
PS_API ps_status ps_kv_copy_blocks(ps_kv* kv, ps_kv* from, const int64_t* src, const int64_t* dst, uint64_t n,
                                   void* stream);

/* Masks and positions of trees of drafted tokens, for ps_kv_attend_masked and ps_kv_write_rotated.  Tree b's nodes are
 * rows offsets[b] .. offsets[b + 1] - 1 of num_nodes (device array of num_trees + 1 int64, rising), or with offsets NULL
 * each tree has num_nodes / num_trees of them.  parents[t] (int32): the number in its tree, below t's own, of node t's
 * parent; -1: t is a root, a child of the request's context; less: t is no node.  mask row t (`words` 32-bit words,
 * mask_stride words apart): bit j is set where node j of the tree is t itself or an ancestor of it; none for no node.
 * positions (NULL, or num_nodes int64): the node's depth, 0 for a root, plus start[b] (device array of num_trees int64,
 * or NULL for 0).  A tree has at most 32 * words nodes, words at most 256.  Rows of no tree stay as they are.  A parent
 * that is not below its node, or offsets that do not rise within num_nodes or give a tree too many nodes, are reported
 * (such a node counts as a root, such a tree is skipped).  The paper has no counterpart.
 * Errors: PS_ERR_INVALID, PS_ERR_CUDA. */
PS_API ps_status ps_kv_tree_mask(ps_kv* kv, const int32_t* parents, uint64_t num_nodes, const int64_t* offsets,
                                 uint32_t num_trees, const int64_t* start, uint32_t* mask, int64_t mask_stride,
                                 uint32_t words, int64_t* positions, void* stream);

/* Waits for the stream and returns what the kernels reported since the last report: PS_OK,
 * PS_ERR_INVALID (a slot or block outside the cache, a wrong tree) or PS_ERR_TIMEOUT (a bounded wait of the attention
 * gave up; that call's outputs are not valid).  Error reporting only: no counterpart in the paper. */
PS_API ps_status ps_kv_check(ps_kv* kv, void* stream);

/* A plan: the spans of a batch, laid out for the device.  It is made once and set again for every step
 * whose spans or lengths change; one plan serves every layer's call of a step (and every cache of the same
 * shape).  q_heads is a multiple of kv_heads.  The cache must outlive the plan.  The paper has no counterpart.
 * Errors: PS_ERR_INVALID, PS_ERR_OOM, PS_ERR_CUDA. */
PS_API ps_status ps_kv_plan_create(ps_kv* kv, uint32_t q_heads, uint32_t max_queries, uint32_t max_spans,
                                   uint64_t max_blocks, ps_kv_plan** out);

/* Set the batch: num_queries queries, the spans over them and their blocks (host arrays, copied before the
 * call returns).  A query that no span covers, or none with a key, gets zeros.  Spans may share blocks and
 * overlap; a query's softmax runs over the tokens of all its spans (a token listed twice counts twice).
 * The call may follow calls that still run: the arrays of the last set but one are overwritten, after
 * waiting for the calls that read them.  PS_ERR_STATE while there is a CUDA graph that has captured a call on this
 * plan: the graph reads the plan's arrays, so such a plan stays as it is.  The paper has no counterpart.
 * Errors: PS_ERR_INVALID (the plan is left without a batch), PS_ERR_STATE, PS_ERR_OOM, PS_ERR_CUDA. */
PS_API ps_status ps_kv_plan_set(ps_kv_plan* plan, uint32_t num_queries, const ps_kv_span* spans, uint32_t num_spans,
                                const uint32_t* blocks, uint64_t num_blocks);

/* ps_kv_plan_set for a batch in which spans may also have causal = 2: masked.  Such a span's last num_queries tokens
 * (it has at least so many) are its queries' own, as a causal one's; the tokens before them are seen by all its queries,
 * and which of its own a query sees is a row of the mask that ps_kv_attend_masked takes: a tree of drafted tokens.
 * The paper has no counterpart.  Errors: as ps_kv_plan_set. */
PS_API ps_status ps_kv_plan_set_masked(ps_kv_plan* plan, uint32_t num_queries, const ps_kv_span* spans, uint32_t num_spans,
                                       const uint32_t* blocks, uint64_t num_blocks);

/* Bytes of workspace that ps_kv_attend needs for the batch that is set (0 possible).
 * The paper has no counterpart. */
PS_API ps_status ps_kv_plan_workspace(ps_kv_plan* plan, uint64_t* bytes);

/* Attention of the plan's batch over the cache.  With z_ij = scale * q_i . k_j over the keys j of all spans
 * that query i sees (query heads share the key/value head of their group: head h reads h / (q_heads /
 * kv_heads)), out_i = sum_j e^z_ij v_j / sum_j e^z_ij and lse_i = log sum_j e^z_ij; without a key, zeros
 * and -infinity.  q and out have one 16-bit type: the cache's, or PS_KV_BF16 with PS_KV_FP8.  lse: NULL, or
 * num_queries x q_heads floats.  workspace: device memory, 256-byte aligned, used by this call alone while
 * it runs.  The stream has to exist until the plan is set again, used on another stream or destroyed.  kv may
 * be another cache than the plan's, of the same shape.  Scores, sums and partial results are held in 32 bits,
 * probabilities are rounded to 16 bits for their product with the values: bf16 ones to 8 bits whatever their size; fp16
 * ones (PS_KV_FP16, and PS_KV_FP8 where few rows see the keys) to 11 bits, but where the largest of a row counts 1,
 * those below 2^-14 (PS_KV_FP8: 2^-9) are off by up to 2^-25 (2^-20).
 * The decode and prefill steps of Eq. 6 and Eq. 7 consist of it; the paper has no counterpart.
 * Errors: PS_ERR_INVALID, PS_ERR_STATE (no batch is set), PS_ERR_CUDA. */
PS_API ps_status ps_kv_attend(ps_kv* kv, ps_kv_plan* plan, const ps_kv_rows* q, const ps_kv_rows* out, float* lse,
                              float scale, void* workspace, uint64_t workspace_bytes, void* stream);

/* ps_kv_attend of a batch with masked spans.  mask: device memory, a row of mask_words 32-bit words per query of the batch,
 * rows mask_stride words apart (4-byte aligned): bit j of query i's row (bit j % 32 of word j / 32) is set where i sees
 * token j of its masked span's own ones, the span's length - num_queries + j-th.  Bits past the span's queries and rows of
 * queries without a masked span are not looked at; 32 * mask_words is at least the queries of the longest masked span.
 * Any mask will do: a query need not see itself, nor anything.  A batch without masked spans takes no mask (NULL): one that
 * is given would not be looked at, and is refused.  The paper has no counterpart.
 * Errors: as ps_kv_attend, which refuses a batch with masked spans. */
PS_API ps_status ps_kv_attend_masked(ps_kv* kv, ps_kv_plan* plan, const ps_kv_rows* q, const ps_kv_rows* out, float* lse,
                                     float scale, const uint32_t* mask, int64_t mask_stride, uint32_t mask_words,
                                     void* workspace, uint64_t workspace_bytes, void* stream);

/* Text of the last error of this cache's calls, its plans' among them ("" if none).
 * The paper has no counterpart. */
PS_API const char* ps_kv_last_error(const ps_kv* kv);

/* Release a plan: waits for the calls that read it, and leaves its arrays to the graphs that captured one.  NULL is
 * accepted.  The paper has no counterpart. */
PS_API void ps_kv_plan_destroy(ps_kv_plan* plan);

/* Release a cache and its memory (to the graphs that captured a call on it, where there are any): waits for the
 * device.  NULL is accepted.  The paper has no counterpart. */
PS_API void ps_kv_destroy(ps_kv* kv);

#ifdef __cplusplus
}
#endif

#endif /* PACKSERVE_KV_H */
