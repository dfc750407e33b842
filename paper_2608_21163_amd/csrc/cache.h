// cache.h -- definitions shared by the host side and the kernels of the
// key/value-cache operators (grand_cache_*).
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace gr {

// What a kernel found wrong in device-resident arguments; grand_cache_check
// reports it.  Nothing is read or written out of bounds because of it.
enum { kCacheOk = 0, kCachePage = 1, kCacheLen = 2, kCacheStart = 3, kCacheId = 4 };
struct CacheErr {
  uint32_t code;
  uint32_t where;  // the sequence (or list) it was found in
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
  RowsView q, out;
  float *lse;                // n_tokens x q_heads, may be null
  WeightsView win, wout;     // wout.p null: no weights
  uint32_t q_heads, kv_heads, group, dim;
  float c;                   // scale * log2(e)
  uint32_t window;           // keys a row sees, its own included; 0: all; below 2^31
  int causal;
  // plan
  uint32_t row_tiles;        // row tiles of the longest chunk
  uint32_t split;            // keys of one split (a multiple of the keys a workgroup takes at once)
  uint32_t n_splits;         // most splits a row tile has; 1: results are written directly
  float *part;               // partial sums: (token x q_heads x n_splits) x dim
  float2 *part_ml;           // their running maxima (log2 units) and sums
  float *lse2;               // log2-unit lse of every row, for the weights
  float *scores;             // log2-unit scores by (sequence, key/value head, row, key); null: recomputed
  uint32_t score_rows, score_keys;
  uint32_t row_splits;       // where they are recomputed: splits of the rows, whose sums are
  float *row_sums;           // by (split, sequence, key/value head, key) if there is more than one
  CacheErr *err;
};

struct IdsArgs {
  PagesView pg;
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
  RowsView k, v;
  uint32_t kv_heads, dim;
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

// Pages: tables up to kEvictSmall are handled by one launch whose workgroups
// all find the threshold (8 x 8,000 pages of 16: 36 us, by tiles 44; 8 x 16,000:
// 62 and 51).
constexpr uint32_t kEvictSmall = 8192, kEvictTile = 2048;

// Rows of a workgroup's tile: 16 or 32, its waves taking different keys, or
// 128, its waves taking different rows.
constexpr uint32_t kFewRows = 32, kManyRows = 128;
constexpr uint32_t kAgainKeys = 256;  // keys of a workgroup that computes scores again
constexpr uint32_t kKeysStep = 128;  // keys that a workgroup of few rows takes at once (four waves of 32)

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
