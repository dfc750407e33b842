// cache.h -- definitions shared by the host side and the kernels of the
// key/value-cache operators (grand_cache_*).
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace gr {

// What a kernel found wrong in device-resident arguments; grand_cache_check
// reports it.  Nothing is read or written out of bounds because of it.
enum { kCacheOk = 0, kCachePage = 1, kCacheLen = 2, kCacheStart = 3, kCacheId = 4, kCacheParent = 5, kCacheFull = 6, kCacheRefs = 7, kCacheList = 8 };
struct CacheErr {
  uint32_t code;
  uint32_t where;  // the sequence (list, page) it was found in
};
__device__ __forceinline__ void cache_err(CacheErr *e, uint32_t code, uint32_t where) {
  if (atomicCAS(&e->code, (uint32_t)kCacheOk, code) == kCacheOk) e->where = where;
}

struct PagesView {
  const uint8_t *k, *v;
  uint32_t page, slot, head; // strides in bytes; a page's rows lie within 2^32 bytes of its start
  uint32_t n_pages;
  uint32_t shift;            // log2 of the page size
  uint64_t bytes;            // up to the last page's last row
};

// Scales of packed pages: bytes, strides in bytes; k null: the pages are not packed.
struct ScalesView {
  const uint8_t *k, *v;
  uint32_t page, slot, head;
};

struct SeqsView {
  const uint32_t *table;
  int64_t table_stride;
  const uint32_t *q_start;   // null: one token a sequence
  const uint32_t *lens;
  uint32_t n_seq, n_tokens, max_pages, max_q, max_k;
};

struct RowsView {
  uint8_t *p;
  int64_t token, head;       // strides in bytes
};

struct WeightsView {
  float *p;
  int64_t seq, head;         // strides in elements
};

struct AttendArgs {
  SeqsView s;
  PagesView pg;
  ScalesView sc;
  RowsView q, out;
  float *lse;                // n_tokens x q_heads, may be null
  WeightsView win, wout;     // wout.p null: no weights
  uint32_t q_heads, kv_heads, group, dim;
  float c;                   // scale * log2(e)
  uint32_t window;           // keys a row sees, its own included; 0: all; below 2^31
  int causal;
  uint32_t sinks;            // first tokens that rows see beside their window (0 without one)
  uint32_t sink_keys;        // that rounded up to whole tiles
  // plan
  uint32_t row_tiles;        // row tiles of the longest chunk
  uint32_t split;            // keys of one split (a multiple of the keys a workgroup takes at once)
  uint32_t n_splits;         // most splits a row tile has; 1: results are written directly
  uint32_t units;            // packed pages, few rows: shares of all sequences' keys; 0: splits of each
  float *part;               // partial sums: (token x q_heads x n_splits) x dim
  float2 *part_ml;           // their running maxima (log2 units) and sums
  float *lse2;               // log2-unit lse of every row, for the weights
  float *scores;             // log2-unit scores by (sequence, key/value head, row, key); null: recomputed
  uint32_t score_rows, score_keys;
  uint32_t row_splits;       // where they are recomputed: splits of the rows, whose sums are
  float *row_sums;           // by (split, sequence, key/value head, tile of again_tiles, key) if there is more than one, or a window
  uint32_t sum_keys;         // keys of those tiles
  CacheErr *err;
};

struct IdsArgs {
  PagesView pg;
  ScalesView sc;
  RowsView q, out, prior;    // prior.p null: none
  const float *prior_lse;
  float *lse;
  const uint32_t *ids;
  int64_t ids_seq, ids_head; // strides in elements
  uint32_t n_seq, k, q_heads, group, dim;
  float c;
  CacheErr *err;
};

struct AppendArgs {
  SeqsView s;
  PagesView pg;
  ScalesView sc;
  RowsView k, v;
  uint32_t kv_heads, dim;
  bool f16;                  // packed pages: what the rows hold
  CacheErr *err;
};

struct EvictArgs {
  SeqsView s;
  WeightsView win, wout;
  uint32_t heads, page, shift;
  uint32_t sinks, recent;
  const uint32_t *budget;
  uint32_t *out_table;
  int64_t out_table_stride;
  uint32_t *out_lens, *freed, *n_freed;
  int64_t freed_stride;
  uint32_t cap;              // tokens of a weights row
  int quads;                 // pages of weights are whole, aligned groups of four floats
  // workspace
  uint32_t *keys;            // n_seq x max_pages order keys (larger: kept first)
  // tables above kEvictSmall pages only
  uint32_t *hist;            // n_seq x 3 x 2048 digit counts
  uint32_t *blk;             // n_seq x tiles x 2: keys above and at the threshold
  uint32_t *state;           // n_seq x 2: the threshold, how many equal to it stay
  CacheErr *err;
};

struct ReadArgs {
  PagesView pg;
  ScalesView sc;
  RowsView k, v;             // p null: not wanted
  const uint32_t *slots;
  uint32_t n, kv_heads, dim;
  bool f16;
  CacheErr *err;
};

// Page handling.  refs_in and refs_out may be the same memory.
struct RefArgs {
  SeqsView s;                // the old sequences
  uint32_t shift, n_pages;
  const uint32_t *refs_in;
  uint32_t *refs_out;
  // fork
  const uint32_t *parents;
  uint32_t n_out;
  int drop;
  uint32_t *out_table, *out_lens;
  int64_t out_stride;        // of out_table's rows
  // grow
  const uint32_t *n_new;
  uint32_t *lens;
  // grow: by sequence; compact: lists of n_pages
  uint32_t *src, *dst;
  // release
  const uint32_t *ids, *counts;
  int64_t row_stride;
  uint32_t n_rows, width, cap;
  int tokens;
  uint32_t *freed, *n_freed; // compact: n_freed counts its moves
  // workspace
  uint64_t *below;           // release: pages with more names than counted
  uint64_t *bits;            // a bit a page: free (grow), in use (compact), freed (release)
  uint32_t *blk;             // set bits by block of kRefPages pages
  uint32_t *rank, *total;    // compact: a moving page's place in the lists; pages in use
  uint32_t *need;            // grow: pages a sequence needs, bit 31: one of them for a copy
  uint32_t *at;              // grow: the place in its row of the first page that a sequence gets
  uint32_t *start;           // grow: pages that the sequences before it need (more than kFewSeqs)
  CacheErr *err;
};
constexpr uint32_t kRefPages = 2048;  // pages of a workgroup
constexpr uint32_t kFewBlocks = 256; // workgroups that count the set bits of all themselves
constexpr uint32_t kFewSeqs = 2048;   // sequences whose needs every workgroup adds up

struct CopyArgs {
  PagesView pg;
  ScalesView sc;
  const uint32_t *src, *dst;
  uint32_t n;
  uint32_t row, slots, heads;      // bytes of a head's row, slots of a page
  bool flat;                       // a page's rows lie side by side
  uint32_t scale_row;
  uint32_t pieces;                 // of 16 bytes, of a page's keys
  CacheErr *err;
};

// Pages: tables up to kEvictSmall are handled by one launch whose workgroups
// all find the threshold (8 x 8,000 pages of 16: 36 us, by tiles 44; 8 x 16,000:
// 62 and 51).
constexpr uint32_t kEvictSmall = 8192, kEvictTile = 2048;

// Rows of a workgroup's tile: 16 or 32, its waves taking different keys, or
// 128, its waves taking different rows.
constexpr uint32_t kFewRows = 32, kManyRows = 128;
// Packed pages, few rows: workgroups that a CU's registers hold (a fourth of 128 elements
// spills: 64 single tokens over up to 8,192 86 us instead of 70; tiles of 64 keys a wave 74).
constexpr int packed_groups(int dp, int nb) { return dp > 128 ? (nb > 1 ? 1 : 2) : nb == 1 ? 3 : 2; }
// the row length that their kernel is built for, and whether it takes runs of 16 keys that lie
// in one page, whole rows of scales at once
constexpr uint32_t packed_row(uint32_t dim) { return dim <= 64 ? 64 : dim <= 128 ? 128 : 256; }
inline bool packed_wide(const AttendArgs &a) {
  const uint32_t row = packed_row(a.dim) / 32;  // a row's scales
  return a.pg.shift >= 4 && (a.dim + 31) / 32 == row && ((uintptr_t)a.sc.k | (uintptr_t)a.sc.v | a.sc.page | a.sc.slot | a.sc.head) % row == 0;
}
// keys of a tile of many rows
constexpr uint32_t rows_tile(uint32_t dim) { return dim > 128 ? 32 : 64; }
constexpr uint32_t kAgainKeys = 256;  // keys of a workgroup that computes scores again
// Tiles of keys that some row of a sequence may see.
inline uint32_t again_tiles(const AttendArgs &a) {
  const uint64_t all = ((uint64_t)a.s.max_k + kAgainKeys - 1) / kAgainKeys;
  const uint64_t seen = ((uint64_t)a.sinks + kAgainKeys - 1) / kAgainKeys + ((uint64_t)a.window + a.s.max_q) / kAgainKeys + 2;
  return (uint32_t)(a.window && seen < all ? seen : all);
}
constexpr uint32_t kKeysStep = 128;  // keys that a workgroup of few rows takes at once (four waves of 32)

// (16-bit pages without first tokens; the others are called from there)
hipError_t launch_attend_sinks(uint32_t tile_rows, bool f16, const AttendArgs &a, hipStream_t st);
hipError_t launch_attend_packed(uint32_t tile_rows, bool f16, const AttendArgs &a, hipStream_t st);
hipError_t launch_weights_sinks(bool f16, const AttendArgs &a, hipStream_t st);
hipError_t launch_weights_packed(bool f16, const AttendArgs &a, hipStream_t st);
hipError_t launch_ids_packed(bool f16, const IdsArgs &a, hipStream_t st);
hipError_t launch_append_packed(const AppendArgs &a, hipStream_t st);
hipError_t launch_read(const ReadArgs &a, hipStream_t st);
hipError_t launch_fork(const RefArgs &a, hipStream_t st);
hipError_t launch_grow(const RefArgs &a, hipStream_t st);
hipError_t launch_release(const RefArgs &a, hipStream_t st);
hipError_t launch_compact(const RefArgs &a, hipStream_t st);
hipError_t launch_copy(const CopyArgs &a, hipStream_t st);
hipError_t launch_attend(uint32_t tile_rows, bool f16, const AttendArgs &a, hipStream_t st);
hipError_t launch_attend_join(bool f16, const AttendArgs &a, uint32_t tile_rows, hipStream_t st);
hipError_t launch_attend_weights(bool f16, const AttendArgs &a, hipStream_t st);
hipError_t launch_attend_ids(bool f16, const IdsArgs &a, hipStream_t st);
hipError_t launch_append(const AppendArgs &a, hipStream_t st);
hipError_t launch_evict(const EvictArgs &a, hipStream_t st);

// The rows and keys of sequence b, with every value from device memory
// brought into range.
struct Chunk {
  uint32_t r0, ql, kl;  // first token, chunk length, cached length
  int p0;               // position of the first new token (kl - ql; negative if the chunk is longer than the cache)
};
__device__ __forceinline__ Chunk chunk_of(const SeqsView &s, uint32_t b, CacheErr *err) {
  Chunk c;
  uint32_t r0 = s.q_start ? s.q_start[b] : b, r1 = s.q_start ? s.q_start[b + 1] : b + 1;
  if (r0 > s.n_tokens || r1 > s.n_tokens || r1 < r0 || r1 - r0 > s.max_q) {
    cache_err(err, kCacheStart, b);
    r0 = min(r0, s.n_tokens);
    r1 = min(max(r1, r0), min(s.n_tokens, r0 + s.max_q));
  }
  uint32_t kl = s.lens[b];
  if (kl > s.max_k) {
    cache_err(err, kCacheLen, b);
    kl = s.max_k;
  }
  c.r0 = r0;
  c.ql = r1 - r0;
  c.kl = kl;
  c.p0 = (int)kl - (int)c.ql;
  return c;
}

}  // namespace gr
