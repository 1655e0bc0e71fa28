/*
 * grand.h -- C ABI of the B200 (sm_100a) library for batched dynamic maintenance and search of a
 * Vamana-style proximity graph (GrAND).
 *
 * One handle = one index on one GPU = one mutator at a time.  The library owns the device-resident
 * vector store (row stride padded to 16 B), the fixed-stride adjacency array uint32[capacity x R]
 * with a degree counter per node, the live bitmap and a workspace pool that is allocated when the
 * index is created (the pre-allocated resource pool of Sec. 3.1): grand_insert_batch, grand_delete_batch,
 * grand_search and the host variants of the two update calls allocate nothing.  (grand_reverse_graph and
 * grand_search_host keep buffers of their own that grow with the largest request.)  The caller owns
 * every buffer it passes in, and the library keeps no caller pointer past a call.  Unless a
 * function says "host", pointer arguments are DEVICE pointers, row-major and densely packed.
 *
 * Batch semantics are deterministic (one legal outcome of the lock-free scheme of Sec. 4): every
 * search of a batch runs on the batch-start snapshot, reverse-edge candidates of one target merge
 * in (distance, id) order, ties break by id.  Distances: L2 = squared Euclidean, IP = negated dot
 * product; uint8/int8 vectors use exact int32 arithmetic, fp32 vectors accumulate in fp32.
 *
 * Errors: every function returns 0 (GRAND_OK) or a negative grand_status.  Update calls validate the
 * whole batch on the device before mutating anything, so a failing call leaves the index unchanged.
 * No exception crosses this boundary and there is no CPU fallback.
 */
#ifndef GRAND_H_
#define GRAND_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct grand_index grand_index; /* opaque */
typedef void* grand_stream;             /* a cudaStream_t; NULL = the default stream */

typedef enum {
  GRAND_U8 = 0, GRAND_I8 = 1, GRAND_F32 = 2, /* vectors of an index */
  GRAND_F16 = 3, GRAND_BF16 = 4              /* token cache only (grand_rope takes GRAND_F32 as well) */
} grand_dtype;
typedef enum { GRAND_L2 = 0, GRAND_IP = 1 } grand_metric;
typedef enum { GRAND_MODE_VAMANA = 0, GRAND_MODE_FIXED_DEGREE = 1 } grand_mode;

typedef enum {
  GRAND_OK = 0,
  GRAND_ERR_INVALID_ARG = -1,  /* null pointer, k > L, parameter beyond a compile-time bound */
  GRAND_ERR_CAPACITY = -2,     /* id >= capacity, batch larger than max_batch, or a delete batch that touches more
                                  in-neighbour entries than max_delete_edges */
  GRAND_ERR_DUPLICATE_ID = -3, /* the same id twice in one batch */
  GRAND_ERR_ALREADY_LIVE = -4, /* insert of a live id */
  GRAND_ERR_NOT_LIVE = -5,     /* delete of an id that is not live */
  GRAND_ERR_UNSUPPORTED = -6,  /* Vamana mode with the IP metric and no mips_max_norm (alpha-pruning needs a metric) */
  GRAND_ERR_CUDA = -7,         /* a CUDA call failed; text in grand_last_error */
  GRAND_ERR_NOMEM = -9         /* device allocation failed (index creation, or growth of an introspection buffer) */
} grand_status;

#define GRAND_INVALID_ID 0xFFFFFFFFu
#define GRAND_MAX_R 128u      /* degree bound limit */
#define GRAND_MAX_L 512u      /* worklist size limit */
#define GRAND_MAX_ROW_BYTES 4096u /* dim * sizeof(element), after padding to 16 B */

/* Optional parameters; a zero field selects the default.  P, c and k follow the parameter list of
 * Alg. 5 / Alg. 6 (scratch capacity, replacement edges per repair, repair candidates). */
typedef struct {
  uint64_t capacity;  /* peak number of ids N; ids live in [0, N-1]; default 1<<20; < 2^31 */
  uint64_t max_batch; /* largest update batch; default 1<<17 */
  uint32_t P;         /* reverse-edge candidates kept per target and batch; default 64; <= 256 */
  uint32_t c;         /* replacement edges per repaired neighbour; default 2; <= 8 */
  uint32_t k_repair;  /* repair candidates per deleted node; default min(50, L); <= 128 */
  uint32_t vmax;      /* expansion cap of update searches; default 2*L; <= 1024 */
  uint32_t mode;      /* grand_mode; default GRAND_MODE_VAMANA.  GRAND_MODE_FIXED_DEGREE needs R <= L (Alg. 7 keeps
                         the R closest entries of a search result of L entries); else GRAND_ERR_INVALID_ARG */
  uint32_t hash_bits; /* log2 of the per-query visited cache in 4-byte words; 8..13, and 4 << hash_bits >= padded row bytes;
                         0 = default: 10, and on rows above 512 bytes up to three times that where shared memory is left over */
  uint32_t full_transpose; /* 1: every delete batch builds the whole reverse graph; default 0: only the rows of the
                              batch's nodes (the only rows the repair reads; identical result) */
  float mips_max_norm;     /* > 0: Vamana mode accepts the IP metric on fp32 vectors through the MIPS -> L2
                              reduction of Sec. 5.3, x -> [x, sqrt(M^2 - |x|^2)] with M = this bound on every base
                              vector's norm (an insert with a larger norm fails with GRAND_ERR_INVALID_ARG);
                              searches still return negated inner products */
  uint32_t visited_set_delete; /* 1: Alg. 6 exactly as printed - the in-neighbours of a deleted node are looked for
                              only in the visited set of its search (no reverse graph).  Edges from nodes that
                              the search did not visit stay behind; searches and rebuilds skip neighbours that
                              are not live.  Default 0: exact in-neighbours, no edge to a deleted node survives.
                              Vamana mode only. */
  uint64_t max_delete_edges;   /* most in-neighbour entries (sum of the in-degrees of its nodes) one delete batch may
                              touch; default min(3 * max_batch * R, capacity * R).  The workspace of the update
                              calls is sized from max_batch and this bound when the index is created; a delete
                              batch beyond it fails with GRAND_ERR_CAPACITY and leaves the index unchanged. */
  uint32_t snapshot_search;    /* 1: searches may run on other streams (and from other host threads) WHILE an update
                              batch runs.  The adjacency is kept twice; a batch works on the unpublished copy and
                              publishes it when it returns, so a search sees exactly the graph of the last batch
                              that had returned when the search was issued.  Costs capacity*R*4 bytes and one
                              copy of the changed rows per batch.  Default 0: one copy, and a search must not
                              overlap an update.  Only grand_search (device pointers) may overlap; the *_host
                              variants share one staging area with the update calls, and profiling
                              (grand_set_profiling) assumes one caller.  Not combinable with visited_set_delete. */
  /* device allocator hooks (default cudaMalloc / cudaFree); lets a host runtime pool the memory */
  void* (*dev_alloc)(size_t bytes, void* user);
  void (*dev_free)(void* ptr, void* user);
  void* user;
} grand_options;

/* Counters since creation (or the last grand_reset_stats).  Times are accumulated only while
 * profiling is on (grand_set_profiling), from CUDA events recorded on the caller's stream. */
typedef struct {
  uint64_t expansions;     /* worklist entries expanded by all beam searches */
  uint64_t dist_evals;     /* query-to-node distances evaluated by beam searches */
  uint64_t pair_dists;     /* node-to-node distances (prune, repair picks, rebuild) */
  uint64_t dirty_nodes;    /* adjacency rows rebuilt */
  uint64_t prunes;         /* RobustPrune invocations (forward + rebuild) */
  uint64_t requests;       /* reverse-edge / repair requests grouped */
  uint64_t kernel_launches; /* kernels launched through this handle */
  uint64_t rebuild_bytes;  /* bytes the dirty-node rebuild has to move: per rebuilt row its read and write (2 * R * 4),
                              its request tuples (12 each) and, when a prune runs, one vector per candidate */
  uint64_t picks_bytes;    /* bytes the delete repair has to move: one vector per (deleted node, surviving in- or
                              out-neighbour) pair plus the repair candidates' vectors once per deleted node */
  uint64_t prune_bytes;    /* forward RobustPrune: one vector per candidate looked at */
  uint64_t rebuild_prunes; /* rebuilt rows that went through a prune (the rest were appends / compactions) */
  double ms_search;        /* beam-search kernels (search, insert and delete searches) */
  double ms_prune;         /* forward RobustPrune */
  double ms_group;         /* request grouping, and the set-up kernels of the repair picks */
  double ms_rebuild;       /* dirty-node rebuild */
  double ms_transpose;     /* reverse-graph construction */
  double ms_picks;         /* delete repair picks (the pick kernel alone) */
  double ms_other;         /* validation, store write, publish / retire */
  uint64_t n_search_launches;  /* launches behind ms_search, ms_prune, ms_rebuild, ms_picks, ms_transpose: */
  uint64_t n_prune_launches;
  uint64_t n_rebuild_launches;
  uint64_t n_picks_launches;
  uint64_t n_transpose_launches;
  uint64_t picks_pair_dists; /* node-to-node distances evaluated by the repair picks alone ... */
  uint64_t prune_pair_dists; /* ... and by the forward RobustPrune alone (both are part of pair_dists) */
} grand_stats;

/* Index life cycle (problem statement of Sec. 3-4: capacity fixed at initialisation, ids in
 * [0, N-1], deleted ids reusable).  dim * sizeof(element) <= GRAND_MAX_ROW_BYTES, R <= GRAND_MAX_R,
 * L <= GRAND_MAX_L.  The device current at creation owns the index. */
int grand_create(uint32_t dim, uint32_t dtype, uint32_t metric, uint32_t R, uint32_t L, float alpha,
                 grand_index** out);
int grand_create_ex(uint32_t dim, uint32_t dtype, uint32_t metric, uint32_t R, uint32_t L, float alpha,
                    const grand_options* opts, grand_index** out);
int grand_destroy(grand_index* idx);

/* BatchInsert (Alg. 5 in Vamana mode, Alg. 7 in fixed-degree mode).  ids_dev: n distinct non-live ids;
 * vecs_dev: n x dim elements.  Work is enqueued on `stream`; the call returns after the batch is
 * applied (it reads back one status block). */
int grand_insert_batch(grand_index* idx, const uint32_t* ids_dev, const void* vecs_dev, uint64_t n,
                       grand_stream stream);

/* BatchDelete (Alg. 6 with in-neighbours from the on-demand CSR reverse graph of Alg. 8; Alg. 8 itself
 * in fixed-degree mode).  ids_dev: n distinct live ids.  After the call no row holds a deleted id. */
int grand_delete_batch(grand_index* idx, const uint32_t* ids_dev, uint64_t n, grand_stream stream);

/* BeamSearch (Alg. 1) from the medoid with worklist size L (k <= L <= GRAND_MAX_L; expansion cap 2L).
 * out_ids_dev: nq x k ids sorted by (distance, id), padded with GRAND_INVALID_ID; out_dists_dev: nq x k
 * int32 (uint8/int8 vectors; padding INT32_MAX) or float (fp32 vectors; padding +inf).  Asynchronous
 * on `stream`; concurrent searches on a quiescent index are allowed. */
int grand_search(const grand_index* idx, const void* queries_dev, uint64_t nq, uint32_t k, uint32_t L,
                 uint32_t* out_ids_dev, void* out_dists_dev, grand_stream stream);

/* The same three calls with HOST buffers (pinned memory gives asynchronous copies): the host-to-device
 * copy of the inputs and the device-to-host copy of the results happen inside the call, which returns
 * after they complete. */
int grand_insert_batch_host(grand_index* idx, const uint32_t* ids_host, const void* vecs_host, uint64_t n,
                            grand_stream stream);
int grand_delete_batch_host(grand_index* idx, const uint32_t* ids_host, uint64_t n, grand_stream stream);
int grand_search_host(grand_index* idx, const void* queries_host, uint64_t nq, uint32_t k, uint32_t L,
                      uint32_t* out_ids_host, void* out_dists_host, grand_stream stream);

/* Introspection for parity checks and measurement.  Any output pointer may be NULL.
 * adj_dev: capacity x R (unused slots hold GRAND_INVALID_ID); deg_dev: capacity; live_bitmap_dev:
 * ceil(capacity/32) words, bit v%32 of word v/32; entry_out_host: HOST pointer to the medoid id. */
int grand_export_graph(const grand_index* idx, uint32_t* adj_dev, uint32_t* deg_dev, uint32_t* live_bitmap_dev,
                       uint32_t* entry_out_host, grand_stream stream);
/* Replaces the whole state (tests, and loading a saved index).  vecs_dev: capacity x dim packed elements.  Every
 * degree must be <= R and every listed neighbour id < capacity, else GRAND_ERR_INVALID_ARG and nothing is replaced. */
int grand_import_graph(grand_index* idx, const uint32_t* adj_dev, const uint32_t* deg_dev,
                       const uint32_t* live_bitmap_dev, uint32_t entry, const void* vecs_dev, grand_stream stream);
/* Exact reverse graph in CSR (Alg. 8): off_dev has capacity+1 entries, row z of src_dev lists every live
 * v with z in N_out(v), ascending.  src_dev needs room for capacity*R entries in the worst case;
 * pass src_dev = NULL to obtain only offsets and *E_out_host (HOST pointer, total edges). */
int grand_reverse_graph(grand_index* idx, uint32_t* off_dev, uint32_t* src_dev, uint64_t* E_out_host,
                        grand_stream stream);

/* The same CSR reverse graph for callers that cannot allocate device memory: hosts whose memory plan is
 * frozen at start-up (a serving process that has handed all of HBM to its own pool, a sandboxed plug-in
 * barred from the driver's allocator, a real-time loop that cannot take cudaMalloc's implicit
 * synchronisation or its failure mid-request).  The paper has no counterpart for this call.  It needs no
 * index handle: adj_dev (n_nodes x R, unused slots ignored through deg_dev; every listed neighbour id must be
 * < n_nodes, otherwise the call returns GRAND_ERR_INVALID_ARG - such an edge is never followed, so nothing is
 * written outside the caller's buffers) and deg_dev (n_nodes) are the caller's inputs, off_dev (n_nodes + 1) and src_dev (src_capacity entries; NULL = offsets only) the caller's
 * outputs, E_out_host a HOST pointer to the edge count.  The result equals grand_reverse_graph on the same
 * graph.  Its working memory is one fixed device array inside the library, GRAND_NOALLOC_SCRATCH_BYTES per GPU
 * for the life of the process: n_nodes > GRAND_NOALLOC_MAX_NODES returns GRAND_ERR_CAPACITY, and so does a
 * src_dev too small for the edges found.  All calls on a device share that array (everything that must be
 * zero is cleared per call), so calls that overlap on the GPU race: serialise them.  The first call on each
 * device resolves the array's address and should be made during set-up, before any stream capture.  No
 * cudaMalloc, cudaFree or allocating library routine is called. */
#define GRAND_NOALLOC_MAX_NODES (1u << 20)
#define GRAND_NOALLOC_SCRATCH_BYTES ((GRAND_NOALLOC_MAX_NODES + GRAND_NOALLOC_MAX_NODES / 2048u + 64u) * 4u)
int grand_reverse_graph_noalloc(const uint32_t* adj_dev, const uint32_t* deg_dev, uint64_t n_nodes, uint32_t R,
                                uint32_t* off_dev, uint32_t* src_dev, uint64_t src_capacity, uint64_t* E_out_host,
                                grand_stream stream);

int grand_get_entry(const grand_index* idx, uint32_t* entry_out_host);
int grand_set_entry(grand_index* idx, uint32_t entry);
int grand_live_count(const grand_index* idx, uint64_t* n_out_host);
int grand_row_bytes(const grand_index* idx, uint32_t* row_bytes_out_host);

int grand_get_stats(const grand_index* idx, grand_stats* out_host);
int grand_reset_stats(grand_index* idx);
int grand_set_profiling(grand_index* idx, int on);

const char* grand_strerror(int status);
const char* grand_last_error(const grand_index* idx);

/* ------------------------------------------------------------------------------------------------------------
 * Token cache: the keys and values of a transformer's past tokens, kept like the vectors of an index in a pool of
 * slots that tokens enter and leave in batches, and read by inner products - here exactly, as softmax attention.
 * The pool is made of pages of page_size slots; a table names the pages of every sequence in order, so token j of
 * a sequence sits in page table[j / page_size], slot j % page_size.  A page of one slot makes the table a list of
 * rows: ids that grand_search returned can be attended directly.  The paper has no counterpart for these calls.
 *
 * The caller owns the pool, the tables and every other buffer; the handle owns a workspace that is allocated at
 * creation, and the calls allocate nothing.  All calls are asynchronous on `stream`, read lengths and tables on
 * the device, and can be captured in a CUDA graph.  One handle serves one stream at a time (its workspace is
 * shared by its calls); make one handle per stream.
 *
 * What a call finds wrong in device data - a page id outside the pool, a position outside the rotary table, a
 * length beyond the table - it skips or clips, never following it, and records in a status word that
 * grand_cache_status reads back.  A token whose page is outside the pool takes no part: a search that pads
 * its answer with GRAND_INVALID_ID may be attended at its full length. */
typedef struct grand_cache grand_cache; /* opaque */

typedef struct {
  uint32_t q_heads;       /* query heads; a multiple of kv_heads */
  uint32_t kv_heads;      /* key / value heads */
  uint32_t head_dim;      /* a multiple of 8, at most 128 */
  uint32_t dtype;         /* GRAND_F16 or GRAND_BF16 */
  uint32_t page_size;     /* tokens per page, any number from 1; at most 2^20 */
  uint32_t weight_groups; /* 0: no weights; 1: one weight per token; kv_heads: one per token and kv head */
  uint32_t max_batch;     /* sequences per call; default 256; at most 4096 */
  uint32_t max_tokens;    /* new tokens per call; default 8192 */
  uint64_t num_pages;     /* pages in the pool; < 2^31 */
  void* (*dev_alloc)(size_t bytes, void* user); /* as in grand_options */
  void (*dev_free)(void* ptr, void* user);
  void* user;
} grand_cache_options;

/* The pool.  Element [page, slot, head, i] of k and of v is at page * page_stride + slot * slot_stride +
 * head * head_stride + i (strides in elements, multiples of 8; both arrays 16-byte aligned).  weights:
 * num_pages x weight_groups x page_size floats, NULL when weight_groups is 0. */
typedef struct {
  void* k;
  void* v;
  float* weights;
  int64_t page_stride, slot_stride, head_stride;
} grand_pool;

/* The sequences of one call.  kv_lens[b] tokens are cached for sequence b, its new ones (if any) last among them;
 * the new tokens of all sequences are packed, those of sequence b being rows cu_new[b] .. cu_new[b + 1] - 1
 * (cu_new: batch + 1 entries; NULL: one new token per sequence).  Only the entries of the table that a length
 * reaches are read. */
typedef struct {
  const int32_t* page_table; /* batch x pages_per_seq, rows table_stride entries apart */
  const int32_t* kv_lens;    /* batch */
  const int32_t* cu_new;
  int64_t table_stride;
  uint32_t pages_per_seq;
  uint32_t batch;
  uint32_t tokens;           /* rows of the packed arrays */
} grand_seqs;

int grand_cache_create(const grand_cache_options* opts, grand_cache** out);
int grand_cache_destroy(grand_cache* cache);
const char* grand_cache_last_error(const grand_cache* cache);

/* Bits set since the last call: 1 page id outside the pool, 2 position outside the rotary table, 4 length
 * negative or beyond the table, or cu_new not ascending, 8 a kernel gave up a wait (its results are void).
 * Waits for `stream`. */
int grand_cache_status(grand_cache* cache, uint32_t* bits_out_host, grand_stream stream);
/* Kernels launched through this handle since its creation. */
int grand_cache_launches(const grand_cache* cache, uint64_t* n_out_host);

/* Rotary positions.  x and out: tokens x heads x dim of `dtype` (GRAND_F16, GRAND_BF16, GRAND_F32), strides in
 * elements, dense along dim; out may be x.  table: table_rows x rot floats, the cosines of the rot / 2 angles of
 * position p in the first half of row p and the sines in the second (any scaling for long contexts is in it).
 * The first rot (even) entries of a head are turned pair by pair, y_a = a c - b s, y_b = b c + a s, with pairs
 * (i, i + rot / 2), or (2i, 2i + 1) if interleaved; the rest is copied.  inverse turns back: the gradient.
 * A position outside the table takes the nearest row of it.  There is no handle to record that: grand_rope_checked
 * sets bit 2 of a status word of the caller's (device memory; NULL: no record) where it finds one. */
int grand_rope(const void* x, void* out, uint32_t dtype, uint64_t tokens, uint32_t heads, uint32_t dim,
               int64_t x_token_stride, int64_t x_head_stride, int64_t out_token_stride, int64_t out_head_stride,
               const float* table, uint64_t table_rows, uint32_t rot, const int32_t* positions,
               uint32_t interleaved, uint32_t inverse, grand_stream stream);
int grand_rope_checked(const void* x, void* out, uint32_t dtype, uint64_t tokens, uint32_t heads, uint32_t dim,
                       int64_t x_token_stride, int64_t x_head_stride, int64_t out_token_stride, int64_t out_head_stride,
                       const float* table, uint64_t table_rows, uint32_t rot, const int32_t* positions,
                       uint32_t interleaved, uint32_t inverse, uint32_t* status_dev, grand_stream stream);

/* New tokens enter the cache: q (may be NULL) is turned into q_out, k is turned and written with v into the slots
 * of the new tokens, kv_lens[b] - new .. kv_lens[b] - 1, whose weights become 0.  A token whose slot is not in the
 * table, or whose sequence's bounds in cu_new are not rows of the call, is dropped.  k, v: tokens x kv_heads x
 * head_dim; q, q_out: tokens x q_heads x head_dim.  strides: six numbers, the token and head strides of q, k, v
 * (q_out is dense).  rot 0: no rotation (table and positions unused). */
int grand_cache_append(grand_cache* cache, const grand_pool* pool, const grand_seqs* seqs, const void* q, void* q_out,
                       const void* k, const void* v, const int64_t* strides_host, const float* table,
                       uint64_t table_rows, uint32_t rot, const int32_t* positions, uint32_t interleaved,
                       grand_stream stream);

/* Attention of the new tokens over the cache: new token i of a sequence with n cached and m new tokens attends
 * the tokens j < n with j <= n - m + i if causal, and j > n - m + i - window if window > 0 (causal only).
 * out = softmax(scale q.k) v, lse = log(sum(exp(scale q.k))) (natural); a row that attends nothing has out 0 and
 * lse -inf, and a row that belongs to no sequence is left as it is.  q: tokens x q_heads x head_dim (token and head stride), out and lse dense, lse may be NULL.
 * Scores, the softmax's maximum and sum, and the output's sum are fp32.  The unnormalised probabilities meet the
 * values in the cache's type: as the sum of two numbers of it with up to 32 rows (query heads of a kv head x new
 * tokens) per sequence on average, rounded to one beyond that.  A key that a row does not see may hold anything; the
 * values of all tokens below kv_lens must be finite, as a masked token takes part in the product with an exact zero. */
int grand_cache_attend(grand_cache* cache, const grand_pool* pool, const grand_seqs* seqs, const void* q,
                       int64_t q_token_stride, int64_t q_head_stride, float scale, uint32_t causal, uint32_t window,
                       void* out, float* lse, grand_stream stream);

/* The attention weight that every cached token collects from the new tokens' queries: for each token j < kv_lens[b],
 * weights = decay * weights + sum over the queries that attend j of exp(scale q.k_j - lse), over the query heads of
 * one kv head, or over all of them (weight_groups 1).  lse is that of grand_cache_attend; a row whose lse is -inf
 * takes no part.  Sums are in a fixed order: equal calls give equal bits.  Sequences may share pages for
 * grand_cache_attend, but not here: a page named twice in one call would have two sums written to it at once (the
 * same holds for grand_cache_append's slots, and for pages that grand_cache_evict moves tokens into). */
int grand_cache_weigh(grand_cache* cache, const grand_pool* pool, const grand_seqs* seqs, const void* q,
                      int64_t q_token_stride, int64_t q_head_stride, const float* lse, float scale, uint32_t causal,
                      uint32_t window, float decay, grand_stream stream);

/* Eviction: sequences of more than `keep` tokens keep the first `sinks`, the last `recent`, and of the others those
 * with the largest weights (ties: the lowest index; a NaN counts as the smallest), `keep` in all; the kept tokens'
 * keys, values and weights move together in their order.  With weight_groups > 1 every kv head chooses for itself.
 * A token whose page is outside the pool is never kept; if it is a sink or among the last, another takes its place.  A kept
 * token whose new slot is outside the pool is lost.
 * into: a table (batch x into_pages_per_seq, rows into_stride entries apart) of the pages that receive them, all
 * other than the source pages; NULL: in place.  kept_out: batch x weight_groups x keep, ascending, -1 behind the
 * last; lens_out: batch, the number of tokens kept; not kv_lens itself.  seqs->cu_new is not read.  keep >= sinks + recent, keep >= 1. */
int grand_cache_evict(grand_cache* cache, const grand_pool* pool, const grand_seqs* seqs, uint32_t keep, uint32_t sinks,
                      uint32_t recent, const int32_t* into, int64_t into_stride, uint32_t into_pages_per_seq,
                      int32_t* kept_out, int32_t* lens_out, grand_stream stream);

#ifdef __cplusplus
}
#endif
#endif /* GRAND_H_ */
