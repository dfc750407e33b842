// k_pages.hip -- pages that sequences share: counts of the table entries that
// name a page (0: free), kept on the GPU.  Which free page goes where, and
// the order of lists, follow from ranks among the pages' bits in ascending order,
// never from the order in which workgroups run.  Integer atomics count
// names; their order does not show.  Pools of 10,000s of pages and tables of 100s of rows are
// a few hundred KB: what counts is the number of launches that depend on one
// another.
#include "cache.h"
#include "wave.h"

namespace gr {
namespace {

typedef uint32_t v4u __attribute__((ext_vector_type(4)));
constexpr uint32_t kOneCopy = 0x80000000u;

// Entries of a sequence's row.
__device__ __forceinline__ uint32_t row_pages(const RefArgs &a, uint32_t b, uint32_t &len) {
  len = a.s.lens[b];
  if (len > a.s.max_k) {
    cache_err(a.err, kCacheLen, b);
    len = a.s.max_k;
  }
  return (uint32_t)(((uint64_t)len + (1u << a.shift) - 1) >> a.shift);
}

__global__ __launch_bounds__(256) void k_copy_refs(RefArgs a) {
  const uint64_t p = (uint64_t)blockIdx.x * 256 + threadIdx.x;
  if (p < a.n_pages) a.refs_out[p] = a.refs_in[p];
}

// Takes a name off a page's count.  One that finds nothing left is put back and reported:
// what is taken off in all is what was there, and the count ends at 0, whoever comes first.
__device__ __forceinline__ void drop_name(const RefArgs &a, uint32_t id) {
  if ((int)atomicSub(&a.refs_out[id], 1u) > 0) return;
  atomicAdd(&a.refs_out[id], 1u);
  cache_err(a.err, kCacheRefs, id);
}

// A workgroup per 256 entries of an old row whose names are dropped.  Before the
// new names are counted, so that whether more are dropped than were counted
// does not depend on who comes first.  (Its own launch is 2.9 us; 64
// beams' fork, growth and copies 37.4 us, with names dropped and counted in one launch 34.5.)
__global__ __launch_bounds__(256) void k_fork_drop(RefArgs a) {
  const uint32_t chunks = max((a.s.max_pages + 255) / 256, 1u), b = blockIdx.x / chunks, i = blockIdx.x % chunks * 256 + threadIdx.x;
  uint32_t len;
  if (i >= row_pages(a, b, len)) return;
  const uint32_t id = a.s.table[(int64_t)b * a.s.table_stride + i];
  if (id >= a.n_pages) cache_err(a.err, kCachePage, b);
  else drop_name(a, id);
}

// A workgroup per 256 entries of a new row.
__global__ __launch_bounds__(256) void k_fork(RefArgs a) {
  const uint32_t chunks = max((a.s.max_pages + 255) / 256, 1u), row = blockIdx.x / chunks, i = blockIdx.x % chunks * 256 + threadIdx.x;
  uint32_t len = 0, n = 0;
  const uint32_t b = a.parents[row];
  if (b != kInvalid && b >= a.s.n_seq) cache_err(a.err, kCacheParent, row);
  if (b < a.s.n_seq) n = row_pages(a, b, len);
  if (i == 0) a.out_lens[row] = len;
  const uint32_t id = i < n ? a.s.table[(int64_t)b * a.s.table_stride + i] : kInvalid;
  if (i < a.s.max_pages) a.out_table[(int64_t)row * a.out_stride + i] = id;
  if (i >= n) return;
  if (id >= a.n_pages) cache_err(a.err, kCachePage, b);
  else atomicAdd(&a.refs_out[id], 1u);
}

// A thread's eight pages of a workgroup's 2,048 are 256 apart, so that a wave's
// ballot is a word of the bits.  The workgroup's number of set bits goes to blk.
template <class F>
__device__ __forceinline__ void block_bits(const RefArgs &a, uint32_t blk, F set) {
  __shared__ uint32_t sum[4];
  const uint32_t t = threadIdx.x;
  uint32_t n = 0;
#pragma unroll
  for (uint32_t i = 0; i < kRefPages / 256; i++) {
    const uint64_t p = (uint64_t)blk * kRefPages + i * 256 + t;
    const uint64_t m = ballot(p < a.n_pages && set((uint32_t)p));
    if (t % 64 == 0 && p < a.n_pages) a.bits[p / 64] = m;
    n += popc(m);
  }
  if (t % 64 == 0) sum[t / 64] = n;
  __syncthreads();
  if (t == 0) a.blk[blk] = sum[0] + sum[1] + sum[2] + sum[3];
}

// The sums of x and y over a workgroup of 256.
__device__ __forceinline__ void sum_pair(uint32_t &x, uint32_t &y) {
  __shared__ uint32_t tmp[4][2];
  const uint32_t t = threadIdx.x;
#pragma unroll
  for (int j = 32; j; j >>= 1) {
    x += (uint32_t)__shfl_xor((int)x, j, 64);
    y += (uint32_t)__shfl_xor((int)y, j, 64);
  }
  if (t % 64 == 0) tmp[t / 64][0] = x, tmp[t / 64][1] = y;
  __syncthreads();
  x = tmp[0][0] + tmp[1][0] + tmp[2][0] + tmp[3][0];
  y = tmp[0][1] + tmp[1][1] + tmp[2][1] + tmp[3][1];
  __syncthreads();
}

// Sums of blk[0 .. n) before and in all, by a workgroup of 256.
__device__ __forceinline__ void blk_sums(const RefArgs &a, uint32_t n, uint32_t before, uint32_t &sum_before, uint32_t &sum_all) {
  const uint32_t t = threadIdx.x;
  uint32_t x = 0, y = 0;
  for (uint32_t i = t; i < n; i += 256) {
    const uint32_t c = a.blk[i];
    y += c;
    if (i < before) x += c;
  }
  sum_pair(x, y);
  sum_before = x, sum_all = y;
}

// The same from the bits themselves, for the set bits of the words before `before`:
// one launch less (pages given back in a pool of 165,000: 17.4 us, 21.5 with it).
__device__ __forceinline__ void word_sums(const RefArgs &a, uint32_t before, uint32_t &sum_before, uint32_t &sum_all) {
  const uint32_t words = (a.n_pages + 63) / 64;
  uint32_t x = 0, y = 0;
  for (uint32_t i = threadIdx.x; i < words; i += 256) {
    const uint32_t c = popc(a.bits[i]);
    y += c;
    if (i < before) x += c;
  }
  sum_pair(x, y);
  sum_before = x, sum_all = y;
}
__global__ __launch_bounds__(256) void k_count_bits(RefArgs a) {
  const uint32_t words = kRefPages / 64, t = threadIdx.x;
  const uint64_t w = (uint64_t)blockIdx.x * words + t;
  uint32_t n = t < words && w * 64 < a.n_pages ? popc(a.bits[w]) : 0, all = n;
  sum_pair(n, all);
  if (t == 0) a.blk[blockIdx.x] = all;
}

// Calls f(page, is its bit set, set bits of the workgroup before it) for every page
// of a workgroup.  The 32 words' counts are summed up by one wave.
template <class F>
__device__ __forceinline__ void each_bit(const RefArgs &a, uint32_t blk, F f) {
  __shared__ uint32_t before[kRefPages / 64];
  const uint32_t t = threadIdx.x, words = kRefPages / 64;
  if (t < 64) {
    const uint64_t w = (uint64_t)blk * words + t;
    uint32_t n = t < words && w * 64 < a.n_pages ? popc(a.bits[w]) : 0, s = n;
#pragma unroll
    for (int j = 1; j < 64; j <<= 1) {
      const uint32_t x = (uint32_t)__shfl_up((int)s, j, 64);
      if ((int)t >= j) s += x;
    }
    if (t < words) before[t] = s - n;
  }
  __syncthreads();
#pragma unroll
  for (uint32_t i = 0; i < kRefPages / 256; i++) {
    const uint64_t p = (uint64_t)blk * kRefPages + i * 256 + t;
    if (p < a.n_pages) {
      const uint64_t m = a.bits[p / 64];
      f((uint32_t)p, (bool)(m >> (p % 64) & 1), before[(i * 256 + t) / 64] + popc(m & ((1ull << (p % 64)) - 1)));
    }
  }
}

// ---------------------------------------------------------------- grow
struct GrowSeq {
  uint32_t len, n0, n1;  // tokens, pages before and after
  bool fits;             // its length is within max_k, and the new one within max_pages
};
__device__ __forceinline__ GrowSeq grow_seq(const RefArgs &a, uint32_t b) {
  GrowSeq g;
  g.n0 = row_pages(a, b, g.len);
  const uint64_t after = (uint64_t)g.len + a.n_new[b];
  g.fits = a.s.lens[b] <= a.s.max_k && (after + (1u << a.shift) - 1) >> a.shift <= a.s.max_pages && after <= 0xFFFFFFFFull;
  g.n1 = g.fits ? (uint32_t)((after + (1u << a.shift) - 1) >> a.shift) : g.n0;
  return g;
}

// Free pages, and the pages that sequences need.
__global__ __launch_bounds__(256) void k_grow_need(RefArgs a) {
  const uint32_t blocks = (uint32_t)(((uint64_t)a.n_pages + kRefPages - 1) / kRefPages);
  if (blockIdx.x < blocks) {
    block_bits(a, blockIdx.x, [&](uint32_t p) {
      const uint32_t r = a.refs_in[p];
      if (a.refs_out != a.refs_in) a.refs_out[p] = r;
      return r == 0;
    });
    return;
  }
  const uint32_t b = (blockIdx.x - blocks) * 256 + threadIdx.x;
  if (b >= a.s.n_seq) return;
  const GrowSeq g = grow_seq(a, b);
  if (!g.fits) cache_err(a.err, kCacheLen, b);
  uint32_t need = g.n1 - g.n0, from = kInvalid;
  if (g.fits && a.n_new[b] && (g.len & ((1u << a.shift) - 1))) {
    const uint32_t id = a.s.table[(int64_t)b * a.s.table_stride + g.n0 - 1];
    if (id >= a.n_pages) cache_err(a.err, kCachePage, b);
    else if (a.refs_in[id] > 1) need = (need + 1) | kOneCopy, from = id;
  }
  a.need[b] = need;
  a.at[b] = g.n0 - (need & kOneCopy ? 1 : 0);
  a.src[b] = from;
}

// Sums that stay at 2^32 - 1.
__device__ __forceinline__ uint32_t add_sat(uint32_t x, uint32_t y) { return x + y < x ? ~0u : x + y; }
__device__ __forceinline__ uint32_t wave_scan_sat(uint32_t x, int lane) {
#pragma unroll
  for (int j = 1; j < 64; j <<= 1) {
    const uint32_t y = (uint32_t)__shfl_up((int)x, j, 64);
    if (lane >= j) x = add_sat(x, y);
  }
  return x;
}

// Where each sequence's pages begin among the free ones: start[b], and their
// number at start[n_seq].  A workgroup of NT threads.
template <int NT>
__device__ __forceinline__ void grow_starts(const RefArgs &a, uint32_t *start) {
  __shared__ uint32_t sum[NT / 64];
  const uint32_t t = threadIdx.x, lane = t & 63, wave = t >> 6;
  uint32_t base = 0;
  for (uint32_t b0 = 0; b0 < a.s.n_seq; b0 += NT) {
    const uint32_t b = b0 + t, n = b < a.s.n_seq ? a.need[b] & ~kOneCopy : 0, s = wave_scan_sat(n, lane);
    if (lane == 63) sum[wave] = s;
    __syncthreads();
    uint32_t before = base;
    for (uint32_t w = 0; w < NT / 64; w++) {
      if (w < wave) before = add_sat(before, sum[w]);
      base = add_sat(base, sum[w]);
    }
    const uint32_t up = (uint32_t)__shfl_up((int)s, 1, 64);
    if (b < a.s.n_seq) start[b] = add_sat(before, lane ? up : 0);
    __syncthreads();
  }
  if (t == 0) start[a.s.n_seq] = base;
  __syncthreads();
}
__global__ __launch_bounds__(1024) void k_grow_start(RefArgs a) { grow_starts<1024>(a, a.start); }

// Up to kFewSeqs sequences every workgroup adds up the needs itself: a launch less.
template <bool FEW>
__global__ __launch_bounds__(256) void k_grow_give(RefArgs a) {
  __shared__ uint32_t own[FEW ? kFewSeqs + 1 : 1];
  const uint32_t blocks = (uint32_t)(((uint64_t)a.n_pages + kRefPages - 1) / kRefPages);
  uint32_t before, all;
  blk_sums(a, blocks, min(blockIdx.x, blocks), before, all);
  if constexpr (FEW) grow_starts<256>(a, own);
  const uint32_t *start = FEW ? own : a.start;
  if (blockIdx.x < blocks) {
    const uint32_t wanted = start[a.s.n_seq];
    if (before >= wanted) return;
    each_bit(a, blockIdx.x, [&](uint32_t p, bool free, uint32_t rank) {
      const uint32_t r = before + rank;
      if (!free || r >= wanted) return;
      // the last sequence that starts at r or before it
      uint32_t lo = 0, hi = a.s.n_seq;
      while (hi - lo > 1) {
        const uint32_t mid = lo + (hi - lo) / 2;
        if (start[mid] <= r) lo = mid;
        else hi = mid;
      }
      const uint32_t need = a.need[lo], j = r - start[lo];
      if (add_sat(start[lo], need & ~kOneCopy) > all) return;
      if ((need & kOneCopy) && j == 0) a.dst[lo] = p;
      a.refs_out[p] = 1;
      a.out_table[(int64_t)lo * a.s.table_stride + a.at[lo] + j] = p;
    });
    return;
  }
  const uint32_t b = (blockIdx.x - blocks) * 256 + threadIdx.x;
  if (b >= a.s.n_seq) return;
  const uint32_t need = a.need[b];
  if ((need & ~kOneCopy) && add_sat(start[b], need & ~kOneCopy) > all) {
    cache_err(a.err, kCacheFull, b);
    a.src[b] = a.dst[b] = kInvalid;
    return;
  }
  if (need & kOneCopy) drop_name(a, a.src[b]);
  else a.dst[b] = kInvalid;
  const GrowSeq g = grow_seq(a, b);
  if (g.fits) a.lens[b] = g.len + a.n_new[b];
}

// ---------------------------------------------------------------- release
// A name takes one off its page's count in refs_out.  The one that finds 1 sets the
// page's bit of those that are freed; one that finds 0 (more names than counted)
// sets its bit of those below 0.  A page of either kind ends at 0.
__global__ __launch_bounds__(256) void k_release_start(RefArgs a) {
  const uint64_t p = (uint64_t)blockIdx.x * 256 + threadIdx.x;
  if (p >= a.n_pages) return;
  if (a.refs_out != a.refs_in) a.refs_out[p] = a.refs_in[p];
  if (p % 64 == 0) a.bits[p / 64] = a.below[p / 64] = 0;
}

__global__ __launch_bounds__(256) void k_release_names(RefArgs a) {
  const uint32_t chunks = (a.width + 255) / 256, row = blockIdx.x / chunks, i = blockIdx.x % chunks * 256 + threadIdx.x;
  uint32_t n = a.width;
  if (a.counts) {
    uint64_t c = a.counts[row];
    if (a.tokens) c = (c + (1u << a.shift) - 1) >> a.shift;
    if (c > a.width) {
      cache_err(a.err, kCacheLen, row);
      c = a.width;
    }
    n = (uint32_t)c;
  }
  if (i >= n) return;
  const uint32_t id = a.ids[(int64_t)row * a.row_stride + i];
  if (id == kInvalid) return;
  if (id >= a.n_pages) {
    cache_err(a.err, kCachePage, row);
    return;
  }
  const uint32_t old = atomicSub(&a.refs_out[id], 1u);
  if (old > 1) return;
  atomicOr((unsigned long long *)(old ? a.bits : a.below) + id / 64, 1ull << (id % 64));
  if (!old) cache_err(a.err, kCacheRefs, id);
}

__global__ __launch_bounds__(256) void k_release_list(RefArgs a) {
  uint32_t before, all;
  if (gridDim.x > kFewBlocks) blk_sums(a, gridDim.x, blockIdx.x, before, all);
  else word_sums(a, blockIdx.x * (kRefPages / 64), before, all);
  each_bit(a, blockIdx.x, [&](uint32_t p, bool freed, uint32_t rank) {
    if (freed || a.below[p / 64] >> (p % 64) & 1) a.refs_out[p] = 0;
    if (freed) a.freed[before + rank] = p;
    if (p >= all && p < a.cap) a.freed[p] = kInvalid;
  });
  if (blockIdx.x == 0 && threadIdx.x == 0) *a.n_freed = all;
}

// ---------------------------------------------------------------- compact
__global__ __launch_bounds__(256) void k_compact_bits(RefArgs a) {
  block_bits(a, blockIdx.x, [&](uint32_t p) { return a.refs_in[p] != 0; });
}

// Set bits before page n.
__device__ __forceinline__ uint32_t bits_before(const RefArgs &a, uint32_t blocks, uint32_t n) {
  __shared__ uint32_t tmp[4];
  uint32_t before, all;
  blk_sums(a, blocks, n / kRefPages, before, all);
  uint32_t x = 0;
  const uint32_t t = threadIdx.x, from = n / kRefPages * kRefPages;
  if (from + t * 64 < n) {
    const uint64_t m = a.bits[(from + t * 64) / 64];
    const uint32_t left = n - (from + t * 64);
    x = popc(left >= 64 ? m : m & ((1ull << left) - 1));
  }
#pragma unroll
  for (int j = 32; j; j >>= 1) x += (uint32_t)__shfl_xor((int)x, j, 64);
  if (t % 64 == 0) tmp[t / 64] = x;
  __syncthreads();
  return before + tmp[0] + tmp[1] + tmp[2] + tmp[3];
}

__global__ __launch_bounds__(256) void k_compact_lists(RefArgs a) {
  uint32_t before, live;
  blk_sums(a, gridDim.x, blockIdx.x, before, live);
  const uint32_t front = bits_before(a, gridDim.x, live), moves = live - front;
  each_bit(a, blockIdx.x, [&](uint32_t p, bool used, uint32_t rank) {
    rank += before;
    if (used && p >= live) {
      a.src[rank - front] = p;
      a.rank[p] = rank - front;
    }
    if (!used && p < live) a.dst[p - rank] = p;
    if (p >= moves) a.src[p] = a.dst[p] = kInvalid;
    if (a.refs_out != a.refs_in) a.refs_out[p] = a.refs_in[p];
  });
  if (blockIdx.x == 0 && threadIdx.x == 0) *a.n_freed = moves, *a.total = live;
}

// Counts move with their pages, and the tables get the new ids.
__global__ __launch_bounds__(256) void k_compact_apply(RefArgs a) {
  const uint32_t blocks = (uint32_t)(((uint64_t)a.n_pages + 255) / 256);
  if (blockIdx.x < blocks) {
    const uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= *a.n_freed) return;
    const uint32_t s = a.src[i], d = a.dst[i];
    a.refs_out[d] = a.refs_in[s];
    a.refs_out[s] = 0;
    return;
  }
  const uint32_t chunks = (a.s.max_pages + 255) / 256, x = blockIdx.x - blocks, b = x / chunks, i = x % chunks * 256 + threadIdx.x;
  uint32_t len;
  const uint32_t n = row_pages(a, b, len);
  if (i >= a.s.max_pages) return;
  uint32_t *to = a.out_table + (int64_t)b * a.out_stride + i;
  if (i >= n) {
    if (a.out_table != a.s.table) *to = kInvalid;
    return;
  }
  uint32_t id = a.s.table[(int64_t)b * a.s.table_stride + i];
  if (id >= a.n_pages) {
    cache_err(a.err, kCachePage, b);
  } else if (!(a.bits[id / 64] >> (id % 64) & 1)) {
    cache_err(a.err, kCacheRefs, id);  // named, though its count is 0
  } else {
    if (id >= *a.total) id = a.dst[a.rank[id]];
  }
  *to = id;
}

// ---------------------------------------------------------------- copies
// 1,024 pieces of 16 bytes a workgroup, of each entry the keys' first, then the values':
// `per` small pages, or a part of a large one.  Written past the caches: 185 MB of pages
// in 61 us, 6.1 TB/s of reads and writes; through them 78, read past them too 70.  (Pages of
// one slot, 4 KB of both, several a workgroup: half of a pool compacted in 97 us, a workgroup each 115;
// of two slots a workgroup each is better, 86 and 95.)
template <bool SMALL>
__global__ __launch_bounds__(256) void k_copy_pages(CopyArgs a, uint32_t per, uint32_t chunks) {
  const uint32_t both = 2 * a.pieces, t = threadIdx.x, line = a.row / 16;
  const uint32_t chunk = SMALL ? 0 : blockIdx.x % chunks;
  const uint64_t first = SMALL ? (uint64_t)blockIdx.x * per : blockIdx.x / chunks;
  const uint32_t n = SMALL ? (uint32_t)min((uint64_t)per, a.n - first) : 1;
  auto there = [&](uint32_t s, uint32_t d) { return s < a.pg.n_pages && d < a.pg.n_pages; };
  v4u x[4];
  uint32_t s[4], d[4], at[4];
  bool some[4], key[4];
#pragma unroll
  for (uint32_t j = 0; j < (SMALL ? 4 : 1); j++) {
    const uint32_t e = SMALL ? min((t + j * 256) / both, n - 1) : 0;
    s[j] = a.src[first + e], d[j] = a.dst[first + e];
  }
  if (!SMALL && !there(s[0], d[0])) {
    if (s[0] != kInvalid && d[0] != kInvalid) cache_err(a.err, kCacheList, (uint32_t)first);
    return;
  }
#pragma unroll
  for (uint32_t j = 0; j < 4; j++) {
    const uint32_t y = t + j * 256, e = SMALL ? y / both : 0, in = SMALL ? y - e * both : chunk * 1024 + y;
    if (!SMALL) s[j] = s[0], d[j] = d[0];
    some[j] = SMALL ? e < n && there(s[j], d[j]) : in < both;
    key[j] = in < a.pieces;
    const uint32_t z = key[j] ? in : in - a.pieces;
    at[j] = a.flat ? z * 16u : z / line / a.heads * a.pg.slot + z / line % a.heads * a.pg.head + z % line * 16;
  }
#pragma unroll
  for (uint32_t j = 0; j < 4; j++)
    if (some[j]) x[j] = *(const v4u *)((key[j] ? a.pg.k : a.pg.v) + (uint64_t)s[j] * a.pg.page + at[j]);
#pragma unroll
  for (uint32_t j = 0; j < 4; j++)
    if (some[j]) __builtin_nontemporal_store(x[j], (v4u *)(const_cast<uint8_t *>(key[j] ? a.pg.k : a.pg.v) + (uint64_t)d[j] * a.pg.page + at[j]));
  if (SMALL && t < n) {
    const uint32_t s0 = a.src[first + t], d0 = a.dst[first + t];
    if (s0 != kInvalid && d0 != kInvalid && !there(s0, d0)) cache_err(a.err, kCacheList, (uint32_t)(first + t));
  }
  if (!a.sc.k || chunk) return;
  // the entries' scales, a byte at a time
  const uint32_t bytes = a.slots * a.heads * a.scale_row;
  for (uint32_t y = t; y < n * bytes; y += 256) {
    const uint32_t e = y / bytes, in = y - e * bytes, r = in / a.scale_row;
    const uint32_t s0 = a.src[first + e], d0 = a.dst[first + e];
    if (!there(s0, d0)) continue;
    const uint64_t off = (uint64_t)(r / a.heads) * a.sc.slot + (uint64_t)(r % a.heads) * a.sc.head + in % a.scale_row;
    const_cast<uint8_t *>(a.sc.k)[(uint64_t)d0 * a.sc.page + off] = a.sc.k[(uint64_t)s0 * a.sc.page + off];
    const_cast<uint8_t *>(a.sc.v)[(uint64_t)d0 * a.sc.page + off] = a.sc.v[(uint64_t)s0 * a.sc.page + off];
  }
}

}  // namespace

static uint32_t groups(uint64_t n, uint32_t per) { return (uint32_t)((n + per - 1) / per); }

hipError_t launch_fork(const RefArgs &a, hipStream_t st) {
  if (a.refs_out != a.refs_in) k_copy_refs<<<groups(a.n_pages, 256), 256, 0, st>>>(a);
  const uint32_t chunks = a.s.max_pages ? groups(a.s.max_pages, 256) : 1;
  if (a.drop && a.s.n_seq) k_fork_drop<<<chunks * a.s.n_seq, 256, 0, st>>>(a);
  if (a.n_out) k_fork<<<chunks * a.n_out, 256, 0, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_grow(const RefArgs &a, hipStream_t st) {
  const uint32_t blocks = groups(a.n_pages, kRefPages), seqs = groups(a.s.n_seq, 256);
  if (!a.s.n_seq) {
    if (a.refs_out != a.refs_in) k_copy_refs<<<groups(a.n_pages, 256), 256, 0, st>>>(a);
    return hipGetLastError();
  }
  k_grow_need<<<blocks + seqs, 256, 0, st>>>(a);
  if (a.s.n_seq <= kFewSeqs) {
    k_grow_give<true><<<blocks + seqs, 256, 0, st>>>(a);
  } else {
    k_grow_start<<<1, 1024, 0, st>>>(a);
    k_grow_give<false><<<blocks + seqs, 256, 0, st>>>(a);
  }
  return hipGetLastError();
}

hipError_t launch_release(const RefArgs &a, hipStream_t st) {
  const uint32_t blocks = groups(a.n_pages, kRefPages);
  k_release_start<<<groups(a.n_pages, 256), 256, 0, st>>>(a);
  if (a.n_rows && a.width) k_release_names<<<groups(a.width, 256) * a.n_rows, 256, 0, st>>>(a);
  if (blocks > kFewBlocks) k_count_bits<<<blocks, 256, 0, st>>>(a);
  k_release_list<<<blocks, 256, 0, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_compact(const RefArgs &a, hipStream_t st) {
  const uint32_t blocks = groups(a.n_pages, kRefPages);
  k_compact_bits<<<blocks, 256, 0, st>>>(a);
  k_compact_lists<<<blocks, 256, 0, st>>>(a);
  k_compact_apply<<<groups(a.n_pages, 256) + groups(a.s.max_pages, 256) * a.s.n_seq, 256, 0, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_copy(const CopyArgs &a, hipStream_t st) {
  const uint32_t both = 2 * a.pieces, per = both < 512 ? 1024 / both : 1, chunks = per > 1 ? 1 : groups(both, 1024);
  const uint64_t wgs = per > 1 ? groups(a.n, per) : (uint64_t)a.n * chunks;
  if (per > 1) k_copy_pages<true><<<(uint32_t)wgs, 256, 0, st>>>(a, per, chunks);
  else k_copy_pages<false><<<(uint32_t)wgs, 256, 0, st>>>(a, per, chunks);
  return hipGetLastError();
}

}  // namespace gr
