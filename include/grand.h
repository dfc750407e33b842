/*
 * grand.h -- C ABI of the MI355X (gfx950) library for batched dynamic
 * updates of fixed-degree proximity-graph ANN indexes, following
 * "GrAND: GPU-based Dynamic Graph Indexes for Approximate Nearest Neighbour
 * Search": Vamana with GrANDRobustPrune (Alg. 4-6) and a CAGRA-style fixed
 * out-degree variant with lock-free find-and-replace (Alg. 7-8), both
 * searched by BeamSearch (Alg. 1).
 *
 * Conventions for every entry point
 *  - Status codes are returned; nothing is thrown across the ABI.
 *  - Pointer arguments may point to host memory or to device memory of the
 *    index's GPU; the library detects which.  The caller owns every buffer
 *    it passes; the library copies what it needs and keeps no pointer after
 *    the call returns.
 *  - All work is ordered on the index's HIP stream and every call returns
 *    after its work has completed (one host synchronisation per call).
 *  - Arguments are validated before any state changes: a call that fails
 *    validation leaves the index exactly as it was, and grand_last_error()
 *    describes the problem.  A HIP failure during a call returns
 *    GRAND_E_DEVICE and poisons the handle; every later call on it returns
 *    GRAND_E_STATE.
 *  - One index must not be used by two host threads at the same time.
 *  - Ids are the slots of the resource pool (Section 4: a pool of a fixed
 *    peak size N, ids in [0, N-1], deleted ids reusable).
 */
#ifndef GRAND_H
#define GRAND_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define GRAND_INVALID 0xFFFFFFFFu

typedef struct grand_index grand_index;

typedef enum {
  GRAND_OK = 0,
  GRAND_E_ARG = -1,       /* malformed argument (sizes, k > beam, NaN/inf vector element, ...) */
  GRAND_E_ID = -2,        /* id out of range, repeated in a batch, or in the wrong active state */
  GRAND_E_CAPACITY = -3,  /* a size limit of the library would be exceeded */
  GRAND_E_DEVICE = -4,    /* a HIP call failed; the handle is poisoned */
  GRAND_E_OOM = -5,       /* device allocation failed (state unchanged) */
  GRAND_E_STATE = -6      /* the handle was poisoned by an earlier device failure */
} grand_status;

enum { GRAND_VAMANA = 0, GRAND_CAGRA = 1 };
enum { GRAND_F32 = 0, GRAND_U8 = 1 };
/* GRAND_MIPS: inner-product (maximum inner product) search through the L2
 * augmentation of Section 5.4: a stored vector is [x, sqrt(M^2 - |x|^2)]
 * and a query [q, 0], where M (grand_params.mips_norm) bounds every stored
 * norm, so that |x' - q'|^2 = M^2 + |q|^2 - 2 <x, q> orders points like
 * -<x, q>.  Callers pass vectors of `dim` elements; the extra coordinate is
 * computed as the fp32 rounding of the fp64 square root of M^2 - sum x_j^2
 * (the sum in dimension order).  Search distances are the squared L2
 * distances in the augmented space.  fp32 only, Vamana or CAGRA. */
enum { GRAND_L2 = 0, GRAND_IP = 1, GRAND_MIPS = 2 };
/* alpha test of GrANDRobustPrune (Alg. 4): alpha * Dist(p*, p') <= D_p[p']
 * on the squared distance (default), or on the Euclidean distance. */
enum { GRAND_ALPHA_ON_DIST = 0, GRAND_ALPHA_ON_L2 = 1 };
/* CAGRA reverse edges (Alg. 7): grouped per target and applied in
 * (distance, id) order by one owner (deterministic, default), or applied by
 * independent racing compare-and-swap updates as in the paper's lock-free
 * last-writer-wins form. */
enum { GRAND_CAS_GROUPED = 0, GRAND_CAS_RACING = 1 };
/* In-neighbour discovery for deletes (Alg. 8): the reverse lists of the
 * deleted nodes only (default): one pass over every list that keeps the
 * edges into the batch, then a histogram, prefix scan and scatter into CSR
 * rows indexed by batch position; or the full reverse graph of every node in
 * CSR form (the transpose that grand_export_graph also returns). */
enum { GRAND_REV_FULL = 0, GRAND_REV_BATCH = 1 };

typedef struct {
  uint32_t struct_size;  /* sizeof(grand_params) */
  int32_t algo;          /* GRAND_VAMANA | GRAND_CAGRA */
  int32_t dtype;         /* GRAND_F32 | GRAND_U8 (U8 requires L2) */
  int32_t metric;        /* GRAND_L2 | GRAND_IP (IP requires CAGRA and F32) | GRAND_MIPS (F32) */
  uint32_t dim;          /* vector length; f32 <= 1024, u8 <= 4096 */
  uint32_t capacity;     /* pool size N (ids in [0, N)), < 2^31 */
  uint32_t R;            /* degree bound (Vamana) / fixed degree (CAGRA), 1..64 */
  uint32_t L_build;      /* beam width of insert/delete searches (CAGRA: internal top-k), <= 256 */
  uint32_t P;            /* scratch capacity per node (Alg. 5 and 6), 1..128 */
  uint32_t c;            /* replacement edges per repaired neighbour (Alg. 6), <= 64 */
  uint32_t k_repair;     /* top-k of the delete search used for repair (Alg. 6), <= 64 */
  uint32_t max_iters;    /* expansion cap of insert/delete searches; 0 = 2 * L_build; <= 256 */
  float alpha;           /* pruning factor of GrANDRobustPrune */
  int32_t prune_rule;    /* GRAND_ALPHA_ON_DIST | GRAND_ALPHA_ON_L2 */
  int32_t cas_mode;      /* GRAND_CAS_GROUPED | GRAND_CAS_RACING */
  int32_t rev_mode;      /* GRAND_REV_FULL | GRAND_REV_BATCH */
  uint32_t max_batch;    /* batch size the per-batch buffers are first sized for (grown on demand) */
  float mips_norm;       /* GRAND_MIPS: M, at least the norm of every vector inserted or imported */
  int32_t device;        /* HIP device ordinal */
  void *stream;          /* hipStream_t for all work; NULL = the null stream */
} grand_params;

/* Fills p with the defaults (Vamana, f32, L2, R 64, L_build 128, P 64,
 * c 2, k_repair 50, alpha 1.2 -- the parameters of Section 5.4; reverse
 * lists of the delete batch only). */
void grand_default_params(grand_params *p);

/* Creates an index and allocates its whole resource pool on the device
 * (Section 3.1, resource-pool reuse; Section 4, peak size N).  *out
 * receives the handle.  Errors: GRAND_E_ARG for unsupported parameters,
 * GRAND_E_OOM, GRAND_E_DEVICE. */
grand_status grand_create(const grand_params *p, grand_index **out);

/* Frees the index and all its device memory.  NULL is accepted. */
grand_status grand_destroy(grand_index *h);

/* Sets the HIP stream used by later calls (e.g. torch's current stream). */
grand_status grand_set_stream(grand_index *h, void *stream);

/* BatchInsert (Alg. 3; Vamana Alg. 5; CAGRA Alg. 7).
 * vecs: n rows of dim elements of the index dtype, row-major, packed.
 * ids:  n distinct ids in [0, capacity) that are not active.
 * Every point is searched for on the graph as it was at the start of the
 * batch; forward lists are pruned per point; reverse edges are grouped per
 * target and applied once per target.  An index empty at the start of the
 * batch is bootstrapped from the batch itself (each point's candidates are
 * its nearest other batch points) and its medoid computed.
 * n == 0 is a no-op.  Errors: GRAND_E_ID, GRAND_E_ARG (non-finite element;
 * with GRAND_MIPS a vector whose norm exceeds mips_norm). */
grand_status grand_insert_batch(grand_index *h, const void *vecs, const uint32_t *ids, uint32_t n);

/* CAGRA graph construction (Section 2.2 on CAGRA; Section 4.2, CAGRA graph
 * construction): builds the fixed-degree graph of an empty GRAND_CAGRA
 * index over n points in one call, instead of growing it by batches.
 *   1. an approximate k-NN graph of degree knn by NN-Descent, `iters` rounds
 *      with `sample` new and `sample` old entries sampled per list per round
 *      (local joins between the sampled neighbours and reverse neighbours;
 *      every round reads the lists of the round's start);
 *   2. rank-based pruning: per node, the R neighbours with the fewest
 *      detourable routes (a route u -> z -> y with both ranks below the rank
 *      of y in u's list), by (routes, rank);
 *   3. reverse edges: the output list of y is the first R/2 of its pruned
 *      list, then the nodes whose pruned list holds y (ascending by that
 *      position, then id), then the rest of its pruned list, up to R.
 * vecs, ids: as for grand_insert_batch (n distinct inactive ids).
 * init: n x knn row-major batch positions (host or device): row p holds knn
 *   distinct positions in [0, n) other than p, the random initial neighbours
 *   (drawn by the caller, so that a run can be reproduced).
 * Requires R <= knn <= 128, knn < n, 1 <= sample <= 32, and
 * n * (12 sample^2 - 2 sample) < 2^32 (proposals of one round).  The call
 * works in up to 640 MB of record buffers (and a few arrays of n lists), which
 * it gives back when it ends.  The medoid is computed at the end.  Argument and validation errors change nothing.
 * Errors: GRAND_E_ARG
 * (wrong variant, index not empty, bad sizes or initial lists, non-finite
 * element), GRAND_E_ID, GRAND_E_CAPACITY, GRAND_E_OOM. */
grand_status grand_build_cagra(grand_index *h, const void *vecs, const uint32_t *ids, uint32_t n,
                               const uint32_t *init, uint32_t knn, uint32_t iters, uint32_t sample);

/* BatchDelete (Alg. 3; Vamana Alg. 6; CAGRA Alg. 8), in place.
 * ids: n distinct active ids.  In-neighbours of the deleted nodes are found
 * exactly from a reverse graph built on the GPU for this batch; their lists
 * and those of the repair targets are rebuilt so that no edge points to a
 * deleted id; the deleted rows are cleared and their ids become free.  If
 * the medoid is deleted a new one is installed.
 * n == 0 is a no-op.  Errors: GRAND_E_ID. */
grand_status grand_delete_batch(grand_index *h, const uint32_t *ids, uint32_t n);

/* BeamSearch (Alg. 1) from the medoid with l = beam and at most 2*beam
 * expansions, for nq queries (nq rows of dim elements, packed).
 * out_ids / out_dists: nq x k, the k closest (distance, id) found, padded
 * with GRAND_INVALID / +inf (an empty index returns only padding).
 * Requires 1 <= k <= beam <= 256.  Errors: GRAND_E_ARG. */
grand_status grand_search(grand_index *h, const void *queries, uint32_t nq, uint32_t k, uint32_t beam,
                          uint32_t *out_ids, float *out_dists);

/* Bytes of the fixed device array that grand_search_static works in. */
#define GRAND_STATIC_SCRATCH_BYTES (8u << 20)

/* grand_search for callers that cannot allocate device memory: code under
 * HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.
 * Same arguments, semantics and errors as grand_search, and the same
 * kernels; the staged query rows and the result lists live in a fixed
 * device array of GRAND_STATIC_SCRATCH_BYTES that the library holds on
 * every GPU it runs on until the process ends, so the call allocates
 * nothing (no phase timing and no counting run apply to it).
 * Limit: align256(nq * row) + 2 * align256(nq * k * 4) <= that size, where
 * row is the vector length in bytes rounded up to 16 (for 128-byte rows
 * and k = 10 about 40,000 queries); larger calls return GRAND_E_CAPACITY
 * with nothing done.  Every call on one GPU shares that GPU's array: calls
 * that overlap in time on one GPU (from several threads, or several indexes
 * on different streams) race on it and must be serialised by the caller. */
grand_status grand_search_static(grand_index *h, const void *queries, uint32_t nq, uint32_t k, uint32_t beam,
                                 uint32_t *out_ids, float *out_dists);

/* In-neighbour detection, the step a delete batch needs before it can
 * repair (Alg. 8 builds a reverse graph for it; Section 4.2 reports that
 * building it is an order of magnitude faster than a linear scan of the
 * graph for each deleted point).  Counts, for each of n distinct active ids,
 * the lists of active nodes that hold it, by one of three methods so that
 * their costs can be compared:
 *   GRAND_INDEG_SCAN      a scan of every list for each id (n passes over
 *                         the adjacency; n <= 65535);
 *   GRAND_INDEG_REV_BATCH the reverse lists of the ids only, as a delete
 *                         batch builds them (one pass);
 *   GRAND_INDEG_REV_FULL  the full reverse graph of every node.
 * out_counts: n counts (host or device).  ms (may be NULL): GPU time of the
 * method, from events on the index's stream.  The index is not changed.
 * Errors: GRAND_E_ID (ids out of range, repeated or inactive), GRAND_E_ARG. */
enum { GRAND_INDEG_SCAN = 0, GRAND_INDEG_REV_BATCH = 1, GRAND_INDEG_REV_FULL = 2 };
grand_status grand_count_in_edges(grand_index *h, const uint32_t *ids, uint32_t n, int method, uint32_t *out_counts,
                                  float *ms);

/* Readers: searches that may run while the index's own host thread
 * inserts or deletes (Section 2.3 overlaps kernels on several streams;
 * Section 3.1 names the read-write race of a search reading a list that a
 * delete repairs).  A reader has its own HIP stream (`stream`, or a new
 * non-blocking stream of default priority when NULL), its own staging
 * buffers and counters; grand_reader_search may be called from one other
 * host thread at a time per reader, concurrently with any insert, delete or
 * search call on the index.  Readers must be destroyed before the index;
 * grand_import_graph must not overlap a reader's search.
 * Consistency model of a search that overlaps an update batch: every list
 * entry it reads is a pool id below the capacity or INVALID (lists are
 * rewritten one 32-bit entry at a time); a list that the batch rewrites is
 * read before, after, or part-way through its rewrite, so it may mix old
 * and new entries; a node deleted by the batch may still be reached and
 * returned, and an id that the batch re-inserts may be read with its old
 * or new vector (or, while its row is being copied, a mix of the two).  The
 * start node is the index's medoid as each search begins.  A search that
 * overlaps no update sees the state after the last completed call and
 * returns exactly what grand_search returns.
 * grand_reader_search has the arguments, results and errors of
 * grand_search, and returns after its work on the reader's stream has
 * completed. */
typedef struct grand_reader grand_reader;
grand_status grand_reader_create(grand_index *h, void *stream, grand_reader **out);
grand_status grand_reader_search(grand_reader *r, const void *queries, uint32_t nq, uint32_t k, uint32_t beam,
                                 uint32_t *out_ids, float *out_dists);
grand_status grand_reader_destroy(grand_reader *r);
const char *grand_reader_last_error(const grand_reader *r);

/* Copies the index state out.  Any output pointer may be NULL.
 *   adj: capacity x R lists, GRAND_INVALID padding.  Vamana lists are sets
 *        (their order carries no meaning) and are returned canonically:
 *        each row's ids ascending, padding last.  CAGRA lists are returned
 *        in slot order, which the find-and-replace rules depend on;
 *   deg: capacity;
 *   active: capacity bytes (0/1);  medoid: 1 id (GRAND_INVALID if empty).
 *   rev_offsets (capacity + 1) / rev_srcs: the reverse graph of the current
 *        graph in CSR form, rows ascending by source id (Alg. 8).  With
 *        rev_srcs NULL only the offsets and *nnz are produced, so the caller
 *        can size rev_srcs and call again.  nnz: number of edges. */
grand_status grand_export_graph(grand_index *h, uint32_t *adj, uint32_t *deg, uint8_t *active, uint32_t *medoid,
                                uint32_t *rev_offsets, uint32_t *rev_srcs, uint64_t *nnz);

/* Replaces the whole state: vecs (capacity rows, packed), adj (capacity x
 * R), deg, active (capacity bytes), medoid.  Lists must hold only active ids
 * without repeats.  Used to resume from an exported state and by tests.
 * Errors: GRAND_E_ARG (malformed lists). */
grand_status grand_import_graph(grand_index *h, const void *vecs, const uint32_t *adj, const uint32_t *deg,
                                const uint8_t *active, uint32_t medoid);

/* Per-phase timing and work counters. */
enum {
  GRAND_PH_VALIDATE = 0, GRAND_PH_STAGE, GRAND_PH_SEARCH_INSERT, GRAND_PH_BOOTSTRAP, GRAND_PH_PRUNE_FWD,
  GRAND_PH_GROUP, GRAND_PH_REBUILD, GRAND_PH_SEARCH_DELETE, GRAND_PH_REVERSE, GRAND_PH_REPAIR,
  GRAND_PH_CLEAR, GRAND_PH_MEDOID, GRAND_PH_SEARCH_QUERY, GRAND_PH_CAGRA_DETOUR, GRAND_PH_CAGRA_PICKONE,
  GRAND_NPHASE
};

typedef struct {
  uint32_t struct_size;            /* sizeof(grand_stats_t) */
  uint32_t timing_enabled;
  uint64_t inserted, deleted, queried;
  uint64_t search_hops[3];         /* [insert, delete, query] searches: nodes expanded */
  uint64_t search_evals[3];        /* distance evaluations (row gathers) of those searches */
  uint64_t fwd_evals;              /* pairwise distance evaluations in forward prunes (a matrix-core
                                      tile counts its 16 x 16) */
  uint64_t fwd_prunes;             /* forward GrANDRobustPrune invocations */
  uint64_t rebuild_evals;          /* pairwise distance evaluations in dirty rebuilds, likewise */
  uint64_t rebuild_prunes;         /* dirty rebuilds that ran GrANDRobustPrune */
  uint64_t dirty;                  /* dirty nodes rebuilt (or CAGRA targets / affected nodes) */
  uint64_t rebuild_records;        /* scratch records read by dirty rebuilds */
  uint64_t records;                /* reverse-edge / repair records emitted */
  uint64_t rev_edges;              /* edges found by reverse-graph builds */
  uint64_t repair_evals;           /* distance evaluations in delete repair */
  uint64_t rebuild_rows;           /* vector rows pruning rebuilds need (|C| + 1 each) */
  uint64_t repair_rows;            /* vector rows repairs need (neighbours + |C_i|) */
  uint64_t repair_records;         /* records written by repairs */
  uint64_t search_distinct[3];     /* distinct ids whose distance a search needs: {start} and every
                                      neighbour of an expanded node (counting runs only) */
  uint64_t search_capped[3];       /* searches stopped by max_iters with unexpanded candidates left */
  double phase_ms[GRAND_NPHASE];   /* summed kernel time per phase (timing enabled) */
  uint64_t phase_calls[GRAND_NPHASE];
} grand_stats_t;

/* Enables (1) or disables (0) per-phase HIP event timing on the stream.
 * Phases of a few microseconds (validate, stage, clear, medoid) are not
 * timed, since each recorded event adds a short gap on the stream; their
 * phase_ms stay 0. */
grand_status grand_set_timing(grand_index *h, int enable);

/* Enables (1) or disables (0) counting runs, a measurement mode: every
 * search then uses an exact visited bitmap of one bit per pool id in device
 * memory (capacity/8 bytes per search of a launch, allocated on demand)
 * instead of its lossy visited hash, so that each needed distance is
 * evaluated once and search_distinct counts the method's own distance
 * evaluations (Alg. 1 needs Dist for the start and for every neighbour of
 * an expanded node).  Results are the same as without counting; searches
 * are slower.  Errors: GRAND_E_OOM when the bitmap cannot be allocated. */
grand_status grand_set_counting(grand_index *h, int enable);

/* Copies the counters into out, which must point to at least `size` >=
 * sizeof(grand_stats_t) bytes laid out as grand_stats_t (its struct_size
 * is set).  Errors: GRAND_E_ARG for a null or smaller buffer. */
grand_status grand_stats(grand_index *h, void *out, size_t size);
grand_status grand_reset_stats(grand_index *h);

/* Text of the last error on this handle ("" if none). */
const char *grand_last_error(const grand_index *h);

/* ------------------------------------------------------------------------
 * Key/value caches: the operators with which a language model's attention
 * uses pools of slots beside an index of its keys.  A query's search in a
 * GRAND_MIPS index returns the slots to attend to (grand_cache_attend_ids),
 * the newest tokens are attended to where they lie (grand_cache_attend),
 * and the slots that draw the least attention leave (grand_cache_evict); the
 * freed ids are what grand_delete_batch takes.
 *
 * A pool holds n_pages pages of page_size slots; a slot holds one token's
 * key and value rows of every key/value head.  A sequence's tokens lie in
 * the pages that its row of the page table names, in order.  With
 * page_size 1 a page is a slot and page ids are slot ids.
 *
 * Conventions of grand_cache_* beside those at the top of this file
 *  - Every pointer to data is device memory of the cache's GPU, and the
 *    calls only enqueue work on the cache's stream: they return before it
 *    is done, and the memory must live until then.  A handle keeps
 *    workspaces, no results; calls on one handle are ordered by its stream,
 *    and one host thread at a time makes them.
 *  - A workspace grows when a call needs more than any call before it (the
 *    growth waits for the device).  A stream capture does not allow that:
 *    run the call once before the capture, else it fails with
 *    GRAND_E_CAPACITY and nothing is done.  A workspace that a captured call
 *    uses is kept until the handle is destroyed, so its graph may be replayed
 *    after larger calls, ordered among the handle's calls as they are.
 *    grand_cache_check and grand_cache_set_stream wait for the stream and
 *    fail with GRAND_E_STATE while it is captured, as does a call that HIP
 *    refuses because of a capture of another stream: the handle is as it was
 *    (only GRAND_E_DEVICE poisons it).  Handles are created and destroyed
 *    outside captures.
 *  - Sizes, strides, alignment and the extent of device buffers are checked
 *    before anything is enqueued.  What lies in device memory (page ids,
 *    lengths, chunk starts, slot ids) is checked by the kernels: nothing is
 *    read or written outside the buffers, the results of the sequence
 *    concerned are unspecified, and grand_cache_check reports it.
 *  - Strides are in elements; that of an axis of one element is not looked at.
 *    The elements of one head's row are contiguous; rows start at multiples
 *    of 16 bytes (8 elements).
 */
typedef struct grand_cache grand_cache;
enum { GRAND_BF16 = 2, GRAND_F16 = 3 };

typedef struct {
  uint32_t struct_size;  /* sizeof(grand_cache_params) */
  int32_t dtype;         /* of queries, keys, values and results: GRAND_BF16 | GRAND_F16 */
  uint32_t q_heads;      /* a multiple of kv_heads */
  uint32_t kv_heads;
  uint32_t head_dim;     /* a multiple of 8, 8..256 */
  uint32_t page_size;    /* slots of a page, a power of two, 1..1024 */
  int32_t device;
  void *stream;
} grand_cache_params;

/* A pool.  keys and values have the same strides. */
typedef struct {
  void *k, *v;
  uint32_t n_pages;
  int64_t page_stride, slot_stride, head_stride;
} grand_pages;

/* A pool held in 4 bits.  A row's blocks of 32 elements (the last may be
 * shorter) are 16 bytes of codes each, rows side by side in `k` and `v`, and a
 * scale byte s each in `k_scales` and `v_scales`.  A code is a sign (bit 3) and a
 * magnitude of 0, 0.5, 1, 1.5, 2, 3, 4 or 6 (bits 0 to 2), elements of even index in a
 * byte's low half; an element is its code times 2^(s - 127).  Blocks with s
 * above 252 (bf16) or 140 (fp16) count as NaN.  Elements below the type's
 * normal range that it holds in part only (no append writes their scales) are
 * rounded to it, but for the values that grand_cache_attend_ids_packed sums
 * up, which keep 32 bits.  Strides are in bytes: of codes multiples of 16 and
 * rows aligned to 16, of scales any.  The four arrays may be one buffer's
 * parts (rows whose scales follow their codes, pages that hold both). */
typedef struct {
  uint8_t *k, *v, *k_scales, *v_scales;
  uint32_t n_pages;
  int64_t page_stride, slot_stride, head_stride;
  int64_t scale_page_stride, scale_slot_stride, scale_head_stride;
} grand_packed;

/* Rows by (token, head). */
typedef struct {
  void *p;
  int64_t token_stride, head_stride;
} grand_rows;

/* Sums of attention weight by (sequence, key/value head, token), fp32. */
typedef struct {
  float *p;
  int64_t seq_stride, head_stride;
} grand_weights;

/* The sequences of a call.  The new tokens of sequence b are rows
 * q_start[b] .. q_start[b + 1] - 1 of the call's n_tokens rows (q_start
 * null: row b only, n_tokens = n_seq); lens[b] tokens are cached, the new ones
 * included (they are the last).  max_q and max_k bound the new and the
 * cached tokens of a sequence: work is laid out by them (attention and appends:
 * max_k and min(max_q, n_tokens) together at most 2^31 - 64). */
typedef struct {
  uint32_t n_seq, n_tokens, max_q, max_k;
  const uint32_t *table;   /* n_seq rows of max_pages page ids, table_stride apart */
  int64_t table_stride;
  uint32_t max_pages;
  const uint32_t *q_start; /* n_seq + 1, or null */
  const uint32_t *lens;    /* n_seq */
} grand_seqs;

/* bf16, 32 query heads, 8 key/value heads of 128 elements, pages of 16. */
void grand_default_cache_params(grand_cache_params *p);
grand_status grand_cache_create(const grand_cache_params *p, grand_cache **out);
grand_status grand_cache_destroy(grand_cache *h);
/* Waits for the old stream's work, as the workspaces are shared. */
grand_status grand_cache_set_stream(grand_cache *h, void *stream);
/* Waits for the stream and reports what kernels found wrong in device memory
 * since the last check: GRAND_E_ID (a page or slot id, or an entry of a list of
 * pages, outside the pool), GRAND_E_ARG (lengths, chunk starts or parents out of range, a page
 * with more names than its count says) or GRAND_E_CAPACITY (a pool without
 * enough free pages for grand_pages_grow), else GRAND_OK. */
grand_status grand_cache_check(grand_cache *h);
const char *grand_cache_last_error(const grand_cache *h);

/* Writes the new tokens' keys and values (n_tokens rows by kv_heads) to their
 * places in the pages: new token i of sequence b is cached token
 * lens[b] - chunk length + i.  No other slot is touched.  No two slots of
 * the pages may share memory; keys and values may be one pool (and then the same rows). */
grand_status grand_cache_append(grand_cache *h, const grand_seqs *s, const grand_rows *k, const grand_rows *v,
                                const grand_pages *pages);

/* Attention of the new tokens over the cached ones, which hold the new ones
 * already (grand_cache_append).  Row i of sequence b has position
 * p = lens[b] - chunk length + i and sees the cached tokens j < lens[b] with
 * j <= p if causal, and j > p - window if window > 0.  With
 * s_j = scale <q, k_j>, out = sum_j exp(s_j) v_j / sum_j exp(s_j) and
 * lse = ln sum_j exp(s_j), by (token, q_head); a row that sees nothing has
 * out = 0 and lse = -inf.  Hidden tokens have no influence, whatever their
 * keys and values hold, and pages that no row sees may have any id.  Query
 * head h uses key/value head h / (q_heads / kv_heads).  scale > 0.
 * Scores, sums, lse and weights are computed in 32 bits; the probabilities are
 * rounded to the type of the values for their product, and out at the end.
 * lse: n_tokens x q_heads, or null.  Rows of no sequence are not written.
 * weights_in, weights_out: null, or rows of at least max_k entries: entry j
 * of weights_out becomes entry j of weights_in plus the softmax weight that
 * the new tokens give to cached token j, summed over them and the query
 * heads of the key/value head; entries from lens[b] on are not written.
 * The two may be one buffer, but not overlap otherwise.  Without weights out
 * may be q itself, with its strides; out shares no memory with q otherwise,
 * nor with the pages (GRAND_E_ARG; rows of equal strides may lie between
 * each other's, rows of different strides may not lie inside each other's
 * extent), nor with any other buffer. */
grand_status grand_cache_attend(grand_cache *h, const grand_seqs *s, const grand_rows *q, const grand_pages *pages,
                                float scale, int causal, uint32_t window, const grand_rows *out, float *lse,
                                const grand_weights *weights_in, const grand_weights *weights_out);

/* grand_cache_attend with first tokens that stay visible: beside its window
 * (window > 0) a row sees the tokens j < sinks, as far as it would without a window. */
grand_status grand_cache_attend_sinks(grand_cache *h, const grand_seqs *s, const grand_rows *q, const grand_pages *pages,
                                      float scale, int causal, uint32_t window, uint32_t sinks, const grand_rows *out, float *lse,
                                      const grand_weights *weights_in, const grand_weights *weights_out);

/* The same over packed pages (sinks may be 0): the attention over the values
 * that the codes stand for.  A hidden token has no influence whatever its
 * codes and scales are. */
grand_status grand_cache_attend_packed(grand_cache *h, const grand_seqs *s, const grand_rows *q, const grand_packed *pages,
                                       float scale, int causal, uint32_t window, uint32_t sinks, const grand_rows *out, float *lse,
                                       const grand_weights *weights_in, const grand_weights *weights_out);

/* grand_cache_append into packed pages.  A block's scale is the smallest power of
 * two at which no element is 7 times it or more, from 2^-125 to 2^125 (bf16) or
 * 2^-23 to 2^13 (fp16); its codes are the nearest to the elements, the even code on a
 * tie, 6 at most.  A block that holds an infinity or NaN has scale 255 and codes of 0.
 * Codes past head_dim are 0.  No two rows of codes or scales may share memory. */
grand_status grand_cache_append_packed(grand_cache *h, const grand_seqs *s, const grand_rows *k, const grand_rows *v,
                                       const grand_packed *pages);

/* Attention of one token per sequence (n_seq rows) over listed slots: row
 * (b, query head h) over the k ids at ids + b * ids_seq_stride +
 * h * ids_head_stride, in any order; GRAND_INVALID entries are passed over,
 * so the lists may be a search's results (a stride of 0 shares a list).
 * Slot id i is slot i % page_size of page i / page_size.  A repeated id
 * counts each time.
 * prior, prior_lse: null, or another attention's result of the same rows
 * over other tokens (out and lse of grand_cache_attend): the call returns
 * what attention over both would.  lse: n_seq x q_heads, or null.
 * out and lse may be prior (with its strides) and prior_lse themselves, out
 * may be q; they overlap them in no other way, nor the pages. */
grand_status grand_cache_attend_ids(grand_cache *h, uint32_t n_seq, const grand_rows *q, const grand_pages *pages,
                                    const uint32_t *ids, uint32_t k, int64_t ids_seq_stride, int64_t ids_head_stride,
                                    float scale, const grand_rows *prior, const float *prior_lse,
                                    const grand_rows *out, float *lse);

/* The same over packed pages. */
grand_status grand_cache_attend_ids_packed(grand_cache *h, uint32_t n_seq, const grand_rows *q, const grand_packed *pages,
                                           const uint32_t *ids, uint32_t k, int64_t ids_seq_stride, int64_t ids_head_stride,
                                           float scale, const grand_rows *prior, const float *prior_lse, const grand_rows *out,
                                           float *lse);

/* The keys and values of listed slots of packed pages, as the cache holds them
 * (an index of the keys takes them from here): rows n x kv_heads of the cache's
 * type.  GRAND_INVALID entries give rows of zeros.  k or v may be null. */
grand_status grand_packed_read(grand_cache *h, uint32_t n, const uint32_t *slots, const grand_packed *pages,
                               const grand_rows *k, const grand_rows *v);

/* Eviction by accumulated weight, in pages.  Of the n = ceil(lens[b] /
 * page_size) pages of sequence b stay: the first `sinks`, the last
 * max(recent, 1 if the last page is not full), and of the others those with
 * the largest score, up to budget[b] pages in all (more only if the fixed
 * ones are more).  A page's score is the fp32 sum, head by head and in a
 * head token by token, of its entries of `weights` (`heads` heads, rows of
 * `cap` entries); equal scores stay lowest index first, NaN counts as
 * -inf.  The order of the pages is kept.
 * Outputs, which overlap no input and not each other: out_table (n_seq x max_pages, packed; the
 * kept pages, then GRAND_INVALID), out_weights (`cap` entries a row: the
 * kept tokens' weights, then zeros), out_lens, freed (n_seq x max_pages: the
 * freed page ids in table order, then GRAND_INVALID), n_freed.  The pages'
 * keys and values stay where they are.  q_start, max_q and n_tokens of s are
 * not used. */
grand_status grand_cache_evict(grand_cache *h, const grand_seqs *s, uint32_t heads, uint32_t cap,
                               const grand_weights *weights, const uint32_t *budget, uint32_t sinks, uint32_t recent,
                               uint32_t *out_table, const grand_weights *out_weights, uint32_t *out_lens,
                               uint32_t *freed, uint32_t *n_freed);

/* Pages that sequences share.  refs: for every page of the pool the number of
 * entries of page tables that name it (rows' first ceil(lens[b] / page_size)
 * entries); a page with refs 0 is free.  The calls keep that so, on the GPU: a
 * program forks, grows and drops sequences without waiting for it.  refs_out may
 * be refs_in, and shares no memory with it otherwise.  Tables, lengths, counts and lists share no
 * memory with each other.  Keys and values stay where they are, except where
 * grand_pages_copy and grand_packed_copy move them, which is for each layer's pool.
 * Of s only the table, lens, max_k, max_pages and n_seq are used. */

/* New sequences that go on from others: row i of out_table (n_out x max_pages,
 * packed) names the pages of row parents[i] and then GRAND_INVALID, out_lens[i] is its
 * length, and their refs are counted.  A parent may be named often or never; GRAND_INVALID
 * gives an empty sequence.  drop: the names in s's table are given up in the
 * same call (a step of a beam), before the new ones are counted.  out_table shares no memory with s's table. */
grand_status grand_pages_fork(grand_cache *h, const grand_seqs *s, uint32_t n_out, const uint32_t *parents, int drop,
                              uint32_t n_pages, const uint32_t *refs_in, uint32_t *refs_out, uint32_t *out_table,
                              uint32_t *out_lens);

/* Room for n_new[b] more tokens a sequence: s's table and lens are brought up to
 * date in place (table and lens: the same memory as in s).  A sequence whose
 * last page is partly filled and named elsewhere too gets a page of its
 * own in its place, src[b] and dst[b] being the old page and the new one, else
 * GRAND_INVALID: grand_pages_copy(n_seq, src, dst) then copies them.  Free
 * pages are given out in ascending order, to the sequences in order and in a sequence to
 * its tokens in order.  A sequence that needs more pages than are left stays as it was, and so does
 * every later one that needs any (reported by grand_cache_check, and
 * to be seen from lens); so does one whose tokens would not fit max_pages, or
 * whose length is above max_k before the call (after it, it may be). */
grand_status grand_pages_grow(grand_cache *h, const grand_seqs *s, const uint32_t *n_new, uint32_t n_pages, const uint32_t *refs_in,
                              uint32_t *refs_out, uint32_t *table, uint32_t *lens, uint32_t *src, uint32_t *dst);

/* Names given up: the entries of n_rows rows of ids (row_stride apart), the
 * first counts[i] of each (counts null: `width`; tokens != 0: counts are
 * tokens, and pages of page_size are meant), GRAND_INVALID entries passed over.  Rows are tables
 * of sequences that have ended, or the freed pages of grand_cache_evict.  freed (min(n_pages,
 * n_rows * width) entries): the pages that nothing names any more, ascending,
 * then GRAND_INVALID; n_freed their number. */
grand_status grand_pages_release(grand_cache *h, uint32_t n_rows, uint32_t width, const uint32_t *ids, int64_t row_stride,
                                 const uint32_t *counts, int tokens, uint32_t n_pages, const uint32_t *refs_in, uint32_t *refs_out,
                                 uint32_t *freed, uint32_t *n_freed);

/* The pages in use become the pool's first: of n pages in use those with ids from n on
 * move, in ascending order, to the free ids below n, in ascending order.  src and dst (n_pages entries):
 * from where to where, then GRAND_INVALID (grand_pages_copy moves the data); n_moves their
 * number.  out_table (n_seq x max_pages, packed; or s's table itself, with its stride): the
 * table with the new ids, and where it is not s's own GRAND_INVALID after each row's pages.
 * s names every sequence that has pages. */
grand_status grand_pages_compact(grand_cache *h, const grand_seqs *s, uint32_t n_pages, const uint32_t *refs_in, uint32_t *refs_out,
                                 uint32_t *out_table, uint32_t *src, uint32_t *dst, uint32_t *n_moves);

/* Copies keys and values of page src[i] to page dst[i], all slots, i < n; entries with
 * GRAND_INVALID in either are passed over.  A page that is named in dst is named there
 * once, and not in src.  No two slots of the pages may share memory; keys and values may be one pool. */
grand_status grand_pages_copy(grand_cache *h, uint32_t n, const uint32_t *src, const uint32_t *dst, const grand_pages *pages);
grand_status grand_packed_copy(grand_cache *h, uint32_t n, const uint32_t *src, const uint32_t *dst, const grand_packed *pages);

#ifdef __cplusplus
}
#endif
#endif /* GRAND_H */
