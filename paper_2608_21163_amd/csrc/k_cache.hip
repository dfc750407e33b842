// k_cache.hip -- operators beside the cache's attention: attention over
// retrieved ids, the write of new tokens, eviction by accumulated weight.
#include "cache.h"
#include "wave.h"

namespace gr {
namespace {

typedef uint32_t v4u __attribute__((ext_vector_type(4)));
constexpr float kLn2 = 0.69314718055994531f;

__device__ __forceinline__ float neg_inf() { return -__builtin_inff(); }
__device__ __forceinline__ float ex2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float lg2(float x) { return __builtin_amdgcn_logf(x); }

struct Bf16 {
  static __device__ __forceinline__ void widen(v4u x, float *f) {
#pragma unroll
    for (int i = 0; i < 4; i++) {
      f[2 * i] = __uint_as_float(x[i] << 16);
      f[2 * i + 1] = __uint_as_float(x[i] & 0xFFFF0000u);
    }
  }
  typedef __bf16 T;
};
struct F16 {
  static __device__ __forceinline__ void widen(v4u x, float *f) {
    typedef _Float16 v8h __attribute__((ext_vector_type(8)));
    const v8h h = __builtin_bit_cast(v8h, x);
#pragma unroll
    for (int i = 0; i < 8; i++) f[i] = (float)h[i];
  }
  typedef _Float16 T;
};

// (m, l) of two parts of a softmax, in log2 units; m may be -inf (nothing).
__device__ __forceinline__ float part_scale(float m, float top) { return m == neg_inf() ? 1.f : ex2(m - top); }

// One workgroup per (sequence, query head); DP / 8 lanes read one row, each
// 16 bytes of it, and a lane group runs its own softmax over every
// (4 x groups)-th id; the groups are joined at the end.  Rows lie anywhere,
// so the time is that of their bytes: 256 x 32 lists of 256 ids (1.09 GB)
// 178 us, 6.1 TB/s; 8 x 32 lists of 100 take 6 us, launch and two dependent loads.
// Lists of a large pool that were found apart share few rows; where the heads of a
// group name one list, each of them reads its rows, through the caches.
template <class E, int DP>
__global__ __launch_bounds__(256) void k_attend_ids(IdsArgs a) {
  constexpr int LPR = DP / 8, GROUPS = 64 / LPR, U = 4;
  __shared__ float2 sml[4];
  __shared__ float sacc[4][DP];
  const uint32_t b = blockIdx.x / a.q_heads, head = blockIdx.x % a.q_heads, kvh = head / a.group;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6, g = lane / LPR, c = lane % LPR;
  const bool in = c * 8 < (int)a.dim;
  float q[8];
  {
    v4u x{0, 0, 0, 0};
    if (in) x = *(const v4u *)(a.q.p + (int64_t)b * a.q.token + (int64_t)head * a.q.head + c * 16);
    E::widen(x, q);
#pragma unroll
    for (int i = 0; i < 8; i++) q[i] *= a.c;
  }
  const uint32_t *ids = a.ids + (int64_t)b * a.ids_seq + (int64_t)head * a.ids_head;
  const uint64_t slots = (uint64_t)a.pg.n_pages << a.pg.shift;
  const uint32_t mask = (1u << a.pg.shift) - 1;
  float m = neg_inf(), l = 0.f, acc[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  for (uint32_t j0 = wave * GROUPS + g; j0 < a.k; j0 += 4 * GROUPS * U) {
    uint32_t id[U];
    v4u kx[U], vx[U];
#pragma unroll
    for (int u = 0; u < U; u++) {
      const uint32_t j = j0 + u * 4 * GROUPS;
      id[u] = j < a.k ? ids[j] : kInvalid;
      if (id[u] != kInvalid && id[u] >= slots) {
        cache_err(a.err, kCacheId, b);
        id[u] = kInvalid;
      }
    }
#pragma unroll
    for (int u = 0; u < U; u++) {
      kx[u] = vx[u] = v4u{0, 0, 0, 0};
      if (id[u] != kInvalid && in) {
        const uint64_t off = (uint64_t)(id[u] >> a.pg.shift) * a.pg.page + ((id[u] & mask) * a.pg.slot + kvh * a.pg.head + c * 16);
        kx[u] = *(const v4u *)(a.pg.k + off);
        vx[u] = *(const v4u *)(a.pg.v + off);
      }
    }
    float s[U], top = m;
#pragma unroll
    for (int u = 0; u < U; u++) {
      float f[8], x = 0.f;
      E::widen(kx[u], f);
#pragma unroll
      for (int i = 0; i < 8; i++) x = __builtin_fmaf(f[i], q[i], x);
#pragma unroll
      for (int j = LPR / 2; j; j >>= 1) x += xshfl(x, j);
      s[u] = id[u] == kInvalid ? neg_inf() : x;
      top = fmaxf(top, s[u]);
    }
    const float base = top == neg_inf() ? 0.f : top, scale = m == neg_inf() ? 1.f : ex2(m - base);
    m = top;
    l *= scale;
#pragma unroll
    for (int i = 0; i < 8; i++) acc[i] *= scale;
#pragma unroll
    for (int u = 0; u < U; u++) {
      const float p = id[u] == kInvalid ? 0.f : ex2(s[u] - base);
      float f[8];
      E::widen(vx[u], f);
      l += p;
#pragma unroll
      for (int i = 0; i < 8; i++) acc[i] = __builtin_fmaf(p, f[i], acc[i]);
    }
  }
  // lane groups of the wave, then the waves
  float top = m;
#pragma unroll
  for (int j = LPR; j < 64; j <<= 1) top = fmaxf(top, xshfl(top, j));
  const float f = part_scale(m, top);
  l *= f;
#pragma unroll
  for (int i = 0; i < 8; i++) acc[i] *= f;
#pragma unroll
  for (int j = LPR; j < 64; j <<= 1) {
    l += xshfl(l, j);
#pragma unroll
    for (int i = 0; i < 8; i++) acc[i] += xshfl(acc[i], j);
  }
  if (g == 0) {
#pragma unroll
    for (int i = 0; i < 8; i++) sacc[wave][c * 8 + i] = acc[i];
  }
  if (lane == 0) sml[wave] = make_float2(top, l);
  const size_t row = (size_t)b * a.q_heads + head;
  // read before the barrier: lse may be the same memory, and one thread writes it
  const float z0 = a.prior.p ? a.prior_lse[row] * (1.f / kLn2) : neg_inf();
  __syncthreads();
  if (t >= DP) return;
  float o0 = 0.f;
  if (a.prior.p) {
    if (t < (int)a.dim)
      o0 = (float)*(const typename E::T *)(a.prior.p + (int64_t)b * a.prior.token + (int64_t)head * a.prior.head + t * 2);
  }
  float mm = z0;
#pragma unroll
  for (int w = 0; w < 4; w++) mm = fmaxf(mm, sml[w].x);
  // the earlier result stands for one row of weight 1 at its lse
  float w0 = z0 == neg_inf() ? 0.f : ex2(z0 - mm);
  float sum = w0, o = w0 == 0.f ? 0.f : w0 * o0;
#pragma unroll
  for (int w = 0; w < 4; w++) {
    const float s = part_scale(sml[w].x, mm);
    sum += sml[w].y * s;
    o += sacc[w][t] * s;
  }
  const bool some = sum > 0.f || sum != sum;
  if (t < (int)a.dim)
    *(typename E::T *)(a.out.p + (int64_t)b * a.out.token + (int64_t)head * a.out.head + t * 2) =
        (typename E::T)(some ? o / sum : 0.f);
  if (t == 0 && a.lse) a.lse[row] = some ? (mm + lg2(sum)) * kLn2 : neg_inf();
}

// One thread per 16 bytes of a new token's keys and values: 8,192 tokens of
// 8 heads (67 MB) 11.8 us, 5.7 TB/s; 64 tokens are a launch.
__global__ __launch_bounds__(256) void k_append(AppendArgs a) {
  const uint32_t b = blockIdx.y, nch = a.dim / 8;
  const Chunk ch = chunk_of(a.s, b, a.err);
  const uint32_t x = blockIdx.x * 256 + threadIdx.x;
  const uint32_t c = x % nch, head = x / nch % a.kv_heads, i = x / nch / a.kv_heads;
  if (i >= ch.ql) return;
  const int64_t pos = (int64_t)ch.p0 + i;
  if (pos < 0) {  // a chunk longer than its cache
    cache_err(a.err, kCacheLen, b);
    return;
  }
  const uint32_t page = a.s.table[(int64_t)b * a.s.table_stride + (pos >> a.pg.shift)];
  if (page >= a.pg.n_pages) {
    cache_err(a.err, kCachePage, b);
    return;
  }
  const uint64_t to = (uint64_t)page * a.pg.page + ((uint32_t)(pos & ((1u << a.pg.shift) - 1)) * a.pg.slot + head * a.pg.head + c * 16);
  const int64_t tok = ch.r0 + i;
  *(v4u *)(const_cast<uint8_t *>(a.pg.k) + to) = *(const v4u *)(a.k.p + tok * a.k.token + (int64_t)head * a.k.head + c * 16);
  *(v4u *)(const_cast<uint8_t *>(a.pg.v) + to) = *(const v4u *)(a.v.p + tok * a.v.token + (int64_t)head * a.v.head + c * 16);
}

// ---------------------------------------------------------------- eviction
struct EvictSeq {
  uint32_t len, n, fixed, keep;  // tokens, pages, pages that must stay, pages that stay
  uint32_t tail0;                // first of the last pages that must stay
};
__device__ __forceinline__ EvictSeq evict_seq(const EvictArgs &a, uint32_t b) {
  EvictSeq e;
  e.len = a.s.lens[b];
  if (e.len > a.s.max_k) {
    cache_err(a.err, kCacheLen, b);
    e.len = a.s.max_k;
  }
  e.n = (e.len + a.page - 1) >> a.shift;
  const uint32_t recent = min(max(a.recent, (e.len & (a.page - 1)) ? 1u : 0u), e.n);
  e.tail0 = e.n - recent;
  e.fixed = recent + min(a.sinks, e.tail0);
  e.keep = max(min(e.n, a.budget[b]), e.fixed);
  return e;
}

// The order key of a score: larger keys are kept first.  Pages that must
// stay have the largest key; NaN counts as -inf, -0 as 0.
__device__ __forceinline__ uint32_t order_key(float s) {
  if (s != s) s = neg_inf();
  const uint32_t u = __float_as_uint(s + 0.f);
  return (u >> 31) ? ~u : u | 0x80000000u;
}

// A page's score, in the order of the definition: head by head, token by
// token.  A page's tokens lie side by side, so 16 bytes at a time where that
// is aligned (a.quads), 64 tokens' loads in flight: 64 sequences of 512 pages
// of 16 with 8 heads take 4.6 us, one float at a time 17.7.
__device__ __forceinline__ float page_score(const EvictArgs &a, uint32_t b, uint32_t p) {
  const float *w = a.win.p + (int64_t)b * a.win.seq + ((size_t)p << a.shift);
  float s = 0.f;
  if (!a.quads) {
    for (uint32_t h = 0; h < a.heads; h++)
#pragma unroll 4
      for (uint32_t i = 0; i < a.page; i++) s += w[(int64_t)h * a.win.head + i];
    return s;
  }
  const uint32_t heads_at_once = a.page <= 16 ? 4 : 1, quads = a.page / 4;
  for (uint32_t h0 = 0; h0 < a.heads; h0 += heads_at_once)
    for (uint32_t i0 = 0; i0 < quads; i0 += 16) {
      float4 x[16];
#pragma unroll
      for (uint32_t j = 0; j < 16; j++) {
        const uint32_t h = h0 + (heads_at_once == 4 ? j / 4 : 0), i = heads_at_once == 4 ? j % 4 : i0 + j;
        const bool ok = h < a.heads && i < quads;
        x[j] = ok ? *(const float4 *)(w + (int64_t)h * a.win.head + i * 4) : make_float4(0.f, 0.f, 0.f, 0.f);
      }
#pragma unroll
      for (uint32_t j = 0; j < 16; j++) {
        const uint32_t h = h0 + (heads_at_once == 4 ? j / 4 : 0), i = heads_at_once == 4 ? j % 4 : i0 + j;
        if (h < a.heads && i < quads) s = (((s + x[j].x) + x[j].y) + x[j].z) + x[j].w;
      }
    }
  return s;
}
__device__ __forceinline__ uint32_t page_key(const EvictArgs &a, const EvictSeq &e, uint32_t b, uint32_t p) {
  return p < a.sinks || p >= e.tail0 ? 0xFFFFFFFFu : order_key(page_score(a, b, p));
}

__global__ __launch_bounds__(64) void k_evict_score(EvictArgs a) {
  const uint32_t b = blockIdx.y, p = blockIdx.x * 64 + threadIdx.x;
  const EvictSeq e = evict_seq(a, b);
  if (p < e.n) a.keys[(size_t)b * a.s.max_pages + p] = page_key(a, e, b, p);
}

// The digit at which the number of larger digits reaches `left`: hist holds
// BINS counts, every thread of the workgroup calls.  left becomes the rank
// inside that digit.
template <int BINS, int NT>
__device__ __forceinline__ uint32_t find_digit(const uint32_t *hist, uint32_t &left, uint32_t *tmp) {
  constexpr int PER = (BINS + NT - 1) / NT;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  uint32_t own = 0;
  if (t * PER < BINS) {
#pragma unroll
    for (int i = 0; i < PER; i++) own += hist[t * PER + i];
  }
  uint32_t above = own;  // inclusive sum over the lanes from this one on
#pragma unroll
  for (int j = 1; j < 64; j <<= 1) {
    const uint32_t x = (uint32_t)__shfl_down((int)above, j, 64);
    if (lane + j < 64) above += x;
  }
  if (lane == 0) tmp[wave] = above;
  __syncthreads();
  for (int w = wave + 1; w < NT / 64; w++) above += tmp[w];
  above -= own;  // keys in later threads' digits
  if (own && above < left && above + own >= left) {
    uint32_t at = above;
    for (int i = PER - 1; i >= 0; i--) {
      const uint32_t h = hist[t * PER + i];
      if (at + h >= left) {
        tmp[NT / 64] = (uint32_t)(t * PER + i);
        tmp[NT / 64 + 1] = left - at;
        break;
      }
      at += h;
    }
  }
  __syncthreads();
  const uint32_t d = tmp[NT / 64];
  left = tmp[NT / 64 + 1];
  __syncthreads();
  return d;
}

// Pages [p0, p1) of a sequence: kept ones go to their places in the table,
// with their tokens' weights, freed ones to the list.  Keys above thr stay,
// and the first `left` equal to it; above0 and equal0 count such keys before
// p0.  512 threads.
template <class Keys>
__device__ void evict_slice(const EvictArgs &a, const EvictSeq &e, uint32_t b, uint32_t thr, uint32_t left, uint32_t p0, uint32_t p1,
                            uint32_t above0, uint32_t equal0, Keys keys) {
  __shared__ uint32_t list[512];
  __shared__ uint32_t wsum[8][2];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const uint32_t *table = a.s.table + (int64_t)b * a.s.table_stride;
  uint32_t *out = a.out_table + (int64_t)b * a.out_table_stride, *freed = a.freed + (int64_t)b * a.freed_stride;
  const bool all = e.keep >= e.n;
  for (uint32_t q0 = p0; q0 < p1; q0 += 512) {
    const uint32_t p = q0 + t;
    const bool live = p < p1;
    const uint32_t k = live ? keys(p) : 0;
    const uint32_t id = live ? table[p] : 0;
    const uint64_t am = ballot(live && (all || k > thr)), em = ballot(live && !all && k == thr);
    if (lane == 0) {
      wsum[wave][0] = popc(am);
      wsum[wave][1] = popc(em);
    }
    __syncthreads();
    uint32_t above = above0 + mbcnt(am), equal = equal0 + mbcnt(em), an = above0, en = equal0;
#pragma unroll
    for (int w = 0; w < 8; w++) {
      if (w < wave) {
        above += wsum[w][0];
        equal += wsum[w][1];
      }
      an += wsum[w][0];
      en += wsum[w][1];
    }
    const uint32_t kept0 = above0 + min(equal0, left), at = above + min(equal, left);  // kept before q0, before p
    if (live) {
      const bool keep = all || k > thr || (k == thr && equal < left);
      if (keep) {
        out[at] = id;
        list[at - kept0] = p;
      } else {
        freed[p - at] = id;
      }
    }
    above0 = an;
    equal0 = en;
    const uint32_t kept1 = above0 + min(equal0, left);
    __syncthreads();
    // the last page of the sequence may be partly filled
    const uint32_t first = kept0 << a.shift, n = min(kept1 << a.shift, e.len - ((e.n - e.keep) << a.shift));
    const float *win = a.win.p + (int64_t)b * a.win.seq;
    float *wout = a.wout.p + (int64_t)b * a.wout.seq;
    for (uint32_t j = first + t; j < n; j += 512) {
      const size_t from = ((size_t)list[(j >> a.shift) - kept0] << a.shift) + (j & (a.page - 1));
      for (uint32_t h0 = 0; h0 < a.heads; h0 += 8) {
        float x[8];
#pragma unroll
        for (uint32_t h = 0; h < 8; h++)
          if (h0 + h < a.heads) x[h] = win[(int64_t)(h0 + h) * a.win.head + from];
#pragma unroll
        for (uint32_t h = 0; h < 8; h++)
          if (h0 + h < a.heads) wout[(int64_t)(h0 + h) * a.wout.head + j] = x[h];
      }
    }
    __syncthreads();
  }
}

// What lies behind the kept pages, by `parts` workgroups of 512 threads.
__device__ __forceinline__ void evict_tails(const EvictArgs &a, const EvictSeq &e, uint32_t b, uint32_t part, uint32_t parts) {
  const uint32_t step = parts * 512, i0 = part * 512 + threadIdx.x, gone = e.n - e.keep, len = e.len - (gone << a.shift);
  uint32_t *out = a.out_table + (int64_t)b * a.out_table_stride, *freed = a.freed + (int64_t)b * a.freed_stride;
  for (uint32_t p = e.keep + i0; p < a.s.max_pages; p += step) out[p] = kInvalid;
  for (uint32_t p = gone + i0; p < a.s.max_pages; p += step) freed[p] = kInvalid;
  for (uint32_t h = 0; h < a.heads; h++) {
    float *wout = a.wout.p + (int64_t)b * a.wout.seq + (int64_t)h * a.wout.head;
    for (uint32_t j = len + i0; j < a.cap; j += step) wout[j] = 0.f;
  }
  if (i0 == 0) {
    a.out_lens[b] = len;
    a.n_freed[b] = gone;
  }
}

// Tables of up to kEvictSmall pages: every workgroup of a sequence takes all
// its keys into LDS, finds the threshold by four passes of eight bits, and
// moves its slice of the pages.  Finding it once per slice costs no launch.
// 64 histories of 512 pages of 16, 8 heads: 13 us (17 MB), of which the moves
// take 4; a chain of dependent loads and about 30 barriers bounds it.
__global__ __launch_bounds__(512) void k_evict_small(EvictArgs a) {
  extern __shared__ uint32_t keys[];
  __shared__ uint32_t hist[256], tmp[10];
  const uint32_t b = blockIdx.y, slice = (a.s.max_pages + gridDim.x - 1) / gridDim.x;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const EvictSeq e = evict_seq(a, b);
  evict_tails(a, e, b, blockIdx.x, gridDim.x);
  const uint32_t p0 = blockIdx.x * slice, p1 = min(e.n, p0 + slice);
  if (p0 >= p1) return;
  const uint32_t *src = a.keys + (size_t)b * a.s.max_pages;
  for (uint32_t p = t; p < e.n; p += 512) keys[p] = src[p];
  uint32_t thr = 0, left = e.keep;
  if (e.keep < e.n) {
    if (e.keep == 0) {
      thr = 0xFFFFFFFFu;  // no key is larger
      left = 0;
    } else {
      for (int shift = 24; shift >= 0; shift -= 8) {
        if (t < 256) hist[t] = 0;
        __syncthreads();
        for (uint32_t p = t; p < e.n; p += 512) {
          const uint32_t k = keys[p];
          if (shift == 24 || (k >> (shift + 8)) == (thr >> (shift + 8))) atomicAdd(&hist[(k >> shift) & 255], 1u);
        }
        __syncthreads();
        thr |= find_digit<256, 512>(hist, left, tmp) << shift;
      }
    }
  }
  __syncthreads();
  // keys above and at the threshold before the slice
  uint32_t above = 0, equal = 0;
  for (uint32_t p = t; p < p0; p += 512) {
    above += e.keep >= e.n || keys[p] > thr;
    equal += e.keep < e.n && keys[p] == thr;
  }
#pragma unroll
  for (int j = 32; j; j >>= 1) {
    above += (uint32_t)__shfl_xor((int)above, j, 64);
    equal += (uint32_t)__shfl_xor((int)equal, j, 64);
  }
  if (lane == 0) {
    hist[wave] = above;
    hist[8 + wave] = equal;
  }
  __syncthreads();
  above = equal = 0;
#pragma unroll
  for (int w = 0; w < 8; w++) {
    above += hist[w];
    equal += hist[8 + w];
  }
  evict_slice(a, e, b, thr, left, p0, p1, above, equal, [&](uint32_t p) { return keys[p]; });
}

// Longer tables, tiles of kEvictTile pages: digits of 11, 11 and 10 bits are
// counted by all workgroups together, one launch a digit, then each tile's
// keys above and at the threshold, then the tiles move.  A million pages of
// one slot, two heads: 14 us for the scores and the first digit (its counts meet
// in a few hundred words), 7, 5 and 6 for the others, 11 for the moves; one
// workgroup for it all took 2,290.
constexpr uint32_t kBins = 2048;
constexpr int kPerThread = kEvictTile / 512;  // pages of a tile a thread takes
__device__ __forceinline__ uint32_t *evict_hist(const EvictArgs &a, uint32_t b, int pass) { return a.hist + ((size_t)b * 3 + pass) * kBins; }

__global__ __launch_bounds__(512) void k_evict_clear(EvictArgs a) {
  const size_t i = (size_t)blockIdx.x * 512 + threadIdx.x;
  if (i < (size_t)a.s.n_seq * 3 * kBins) a.hist[i] = 0;
}

// The threshold's digits of the passes before `pass`.
__device__ __forceinline__ void evict_prefix(const EvictArgs &a, const EvictSeq &e, uint32_t b, int pass, uint32_t *tmp, uint32_t &thr,
                                             uint32_t &left) {
  thr = 0;
  left = e.keep;
  if (pass > 0) thr |= find_digit<2048, 512>(evict_hist(a, b, 0), left, tmp) << 21;
  if (pass > 1) thr |= find_digit<2048, 512>(evict_hist(a, b, 1), left, tmp) << 10;
  if (pass > 2) thr |= find_digit<1024, 512>(evict_hist(a, b, 2), left, tmp);
}

template <int PASS>
__global__ __launch_bounds__(512) void k_evict_digit(EvictArgs a) {
  __shared__ uint32_t hist[kBins], tmp[10];
  const uint32_t b = blockIdx.y, p0 = blockIdx.x * kEvictTile;
  const int t = threadIdx.x;
  const EvictSeq e = evict_seq(a, b);
  if (p0 >= e.n) return;
  const uint32_t p1 = min(e.n, p0 + kEvictTile);
  uint32_t *keys = a.keys + (size_t)b * a.s.max_pages;
  // all of a thread's pages are loaded before the first is counted
  uint32_t k[kPerThread];
#pragma unroll
  for (int i = 0; i < kPerThread; i++) {
    const uint32_t p = p0 + i * 512 + t;
    k[i] = p >= p1 ? 0 : PASS == 0 ? page_key(a, e, b, p) : keys[p];
  }
  uint32_t thr = 0, left = 0;
  if (e.keep > 0 && e.keep < e.n) evict_prefix(a, e, b, PASS, tmp, thr, left);
  for (int i = t; i < (int)kBins; i += 512) hist[i] = 0;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kPerThread; i++) {
    const uint32_t p = p0 + i * 512 + t;
    if (p >= p1) break;
    if (PASS == 0) {
      keys[p] = k[i];
      atomicAdd(&hist[k[i] >> 21], 1u);
    }
    if (PASS == 1 && (k[i] >> 21) == (thr >> 21)) atomicAdd(&hist[(k[i] >> 10) & 2047], 1u);
    if (PASS == 2 && (k[i] >> 10) == (thr >> 10)) atomicAdd(&hist[k[i] & 1023], 1u);
  }
  __syncthreads();
  uint32_t *sum = evict_hist(a, b, PASS);
  for (int i = t; i < (int)kBins; i += 512)
    if (hist[i]) atomicAdd(&sum[i], hist[i]);
}

__device__ __forceinline__ void evict_threshold(const EvictArgs &a, const EvictSeq &e, uint32_t b, uint32_t *tmp, uint32_t &thr, uint32_t &left) {
  if (e.keep >= e.n) {
    thr = 0;
    left = e.keep;
  } else if (e.keep == 0) {
    thr = 0xFFFFFFFFu;
    left = 0;
  } else {
    evict_prefix(a, e, b, 3, tmp, thr, left);
  }
}

__global__ __launch_bounds__(512) void k_evict_count(EvictArgs a) {
  __shared__ uint32_t tmp[10], sum[8][2];
  const uint32_t b = blockIdx.y, p0 = blockIdx.x * kEvictTile;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const EvictSeq e = evict_seq(a, b);
  if (p0 >= e.n) return;
  uint32_t thr, left, above = 0, equal = 0;
  const uint32_t *keys = a.keys + (size_t)b * a.s.max_pages, p1 = min(e.n, p0 + kEvictTile);
  uint32_t k[kPerThread];
#pragma unroll
  for (int i = 0; i < kPerThread; i++) k[i] = p0 + i * 512 + t < p1 ? keys[p0 + i * 512 + t] : 0;
  evict_threshold(a, e, b, tmp, thr, left);
#pragma unroll
  for (int i = 0; i < kPerThread; i++) {
    const bool live = p0 + i * 512 + t < p1;
    above += live && (e.keep >= e.n || k[i] > thr);
    equal += live && e.keep < e.n && k[i] == thr;
  }
#pragma unroll
  for (int j = 32; j; j >>= 1) {
    above += (uint32_t)__shfl_xor((int)above, j, 64);
    equal += (uint32_t)__shfl_xor((int)equal, j, 64);
  }
  if (lane == 0) {
    sum[wave][0] = above;
    sum[wave][1] = equal;
  }
  __syncthreads();
  if (t == 0) {
    above = equal = 0;
    for (int w = 0; w < 8; w++) {
      above += sum[w][0];
      equal += sum[w][1];
    }
    uint32_t *blk = a.blk + ((size_t)b * gridDim.x + blockIdx.x) * 2;
    blk[0] = above;
    blk[1] = equal;
    if (blockIdx.x == 0) {
      a.state[b * 2] = thr;
      a.state[b * 2 + 1] = left;
    }
  }
}

__global__ __launch_bounds__(512) void k_evict_move(EvictArgs a) {
  __shared__ uint32_t sum[8][2];
  const uint32_t b = blockIdx.y, p0 = blockIdx.x * kEvictTile;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const EvictSeq e = evict_seq(a, b);
  evict_tails(a, e, b, blockIdx.x, gridDim.x);
  if (p0 >= e.n) return;
  uint32_t above = 0, equal = 0;
  const uint32_t *blk = a.blk + (size_t)b * gridDim.x * 2;
  for (uint32_t i = t; i < blockIdx.x; i += 512) {
    above += blk[i * 2];
    equal += blk[i * 2 + 1];
  }
#pragma unroll
  for (int j = 32; j; j >>= 1) {
    above += (uint32_t)__shfl_xor((int)above, j, 64);
    equal += (uint32_t)__shfl_xor((int)equal, j, 64);
  }
  if (lane == 0) {
    sum[wave][0] = above;
    sum[wave][1] = equal;
  }
  __syncthreads();
  above = equal = 0;
#pragma unroll
  for (int w = 0; w < 8; w++) {
    above += sum[w][0];
    equal += sum[w][1];
  }
  const uint32_t *keys = a.keys + (size_t)b * a.s.max_pages;
  evict_slice(a, e, b, a.state[b * 2], a.state[b * 2 + 1], p0, min(e.n, p0 + kEvictTile), above, equal, [&](uint32_t p) { return keys[p]; });
}

template <class E>
hipError_t ids_type(const IdsArgs &a, hipStream_t st) {
  const dim3 grid(a.n_seq * a.q_heads);
  if (a.dim <= 64) k_attend_ids<E, 64><<<grid, 256, 0, st>>>(a);
  else if (a.dim <= 128) k_attend_ids<E, 128><<<grid, 256, 0, st>>>(a);
  else k_attend_ids<E, 256><<<grid, 256, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_attend_ids(bool f16, const IdsArgs &a, hipStream_t st) {
  return f16 ? ids_type<F16>(a, st) : ids_type<Bf16>(a, st);
}

hipError_t launch_append(const AppendArgs &a, hipStream_t st) {
  const uint64_t n = (uint64_t)a.s.max_q * a.kv_heads * (a.dim / 8);
  k_append<<<dim3((uint32_t)((n + 255) / 256), a.s.n_seq), 256, 0, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_evict(const EvictArgs &a, hipStream_t st) {
  if (a.s.max_pages <= kEvictSmall) {
    if (a.s.max_pages) k_evict_score<<<dim3((a.s.max_pages + 63) / 64, a.s.n_seq), 64, 0, st>>>(a);
    // enough slices to fill the chip, of 64 pages at least
    const uint32_t want = (512 + a.s.n_seq - 1) / a.s.n_seq, most = (a.s.max_pages + 63) / 64;
    const uint32_t slices = want < most ? want : most ? most : 1;
    k_evict_small<<<dim3(slices, a.s.n_seq), 512, a.s.max_pages * 4, st>>>(a);
    return hipGetLastError();
  }
  const dim3 grid((a.s.max_pages + kEvictTile - 1) / kEvictTile, a.s.n_seq);
  k_evict_clear<<<(uint32_t)(((size_t)a.s.n_seq * 3 * kBins + 511) / 512), 512, 0, st>>>(a);
  k_evict_digit<0><<<grid, 512, 0, st>>>(a);
  k_evict_digit<1><<<grid, 512, 0, st>>>(a);
  k_evict_digit<2><<<grid, 512, 0, st>>>(a);
  k_evict_count<<<grid, 512, 0, st>>>(a);
  k_evict_move<<<grid, 512, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace gr
