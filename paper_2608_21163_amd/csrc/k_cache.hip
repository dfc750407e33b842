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
// (4 x groups)-th id; the groups are joined at the end.
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
  __syncthreads();
  if (t >= DP) return;
  float z0 = neg_inf(), o0 = 0.f;
  const size_t row = (size_t)b * a.q_heads + head;
  if (a.prior.p) {
    z0 = a.prior_lse[row] * (1.f / kLn2);
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

// One thread per 16 bytes of a new token's keys and values.
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

__global__ __launch_bounds__(256) void k_evict_score(EvictArgs a) {
  const uint32_t b = blockIdx.y, p = blockIdx.x * 256 + threadIdx.x;
  const EvictSeq e = evict_seq(a, b);
  if (p >= e.n) return;
  uint32_t key = 0xFFFFFFFFu;
  if (p >= a.sinks && p < e.tail0) {
    float s = 0.f;
    for (uint32_t h = 0; h < a.heads; h++) {
      const float *w = a.win.p + (int64_t)b * a.win.seq + (int64_t)h * a.win.head + ((size_t)p << a.shift);
      for (uint32_t i = 0; i < a.page; i++) s += w[i];
    }
    key = order_key(s);
  }
  a.keys[(size_t)b * a.s.max_pages + p] = key;
}

// One workgroup per sequence: the threshold key by four passes of eight
// bits, then the kept and the freed pages in order.
__global__ __launch_bounds__(1024) void k_evict_select(EvictArgs a) {
  __shared__ uint32_t hist[256];
  __shared__ uint32_t sh[4];
  __shared__ uint32_t wsum[16][2];
  const uint32_t b = blockIdx.x;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const EvictSeq e = evict_seq(a, b);
  const uint32_t *keys = a.keys + (size_t)b * a.s.max_pages;
  uint32_t prefix = 0, left = e.keep;  // the left-th largest key among those with this prefix
  if (e.keep < e.n) {
    for (int shift = 24; shift >= 0; shift -= 8) {
      if (t < 256) hist[t] = 0;
      __syncthreads();
      for (uint32_t p = t; p < e.n; p += 1024) {
        const uint32_t k = keys[p];
        if (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&hist[(k >> shift) & 255], 1u);
      }
      __syncthreads();
      if (t == 0) {
        uint32_t above = 0;
        int d = 255;
        for (; d > 0 && above + hist[d] < left; d--) above += hist[d];
        sh[0] = prefix | ((uint32_t)d << shift);
        sh[1] = left - above;
      }
      __syncthreads();
      prefix = sh[0];
      left = sh[1];
      __syncthreads();
    }
  }
  // keys above `prefix` stay, and the first `left` equal to it
  const uint32_t *table = a.s.table + (int64_t)b * a.s.table_stride;
  uint32_t *out = a.out_table + (int64_t)b * a.out_table_stride, *freed = a.freed + (int64_t)b * a.freed_stride;
  uint32_t *map = a.map + (size_t)b * a.s.max_pages;
  uint32_t eq0 = 0, kept0 = 0;
  for (uint32_t p0 = 0; p0 < a.s.max_pages; p0 += 1024) {
    const uint32_t p = p0 + t;
    const bool live = p < e.n;
    const uint32_t k = live ? keys[p] : 0;
    const bool all = e.keep >= e.n, eq = live && !all && k == prefix;
    const uint64_t eqm = ballot(eq);
    if (lane == 0) wsum[wave][0] = popc(eqm);
    __syncthreads();
    uint32_t before = eq0;
    for (int w = 0; w < wave; w++) before += wsum[w][0];
    const bool keep = live && (all || k > prefix || (eq && before + mbcnt(eqm) < left));
    const uint64_t km = ballot(keep);
    if (lane == 0) wsum[wave][1] = popc(km);
    __syncthreads();
    uint32_t at = kept0, eqn = 0, kn = 0;
    for (int w = 0; w < 16; w++) {
      if (w < wave) at += wsum[w][1];
      eqn += wsum[w][0];
      kn += wsum[w][1];
    }
    at += mbcnt(km);  // pages kept before p
    if (live) {
      if (keep) {
        out[at] = table[p];
        map[at] = p;
      } else {
        freed[p - at] = table[p];
      }
    }
    eq0 += eqn;
    kept0 += kn;
    __syncthreads();
  }
  for (uint32_t p = kept0 + t; p < a.s.max_pages; p += 1024) out[p] = kInvalid;
  for (uint32_t p = e.n - kept0 + t; p < a.s.max_pages; p += 1024) freed[p] = kInvalid;
  if (t == 0) {
    a.out_lens[b] = e.len - ((e.n - kept0) << a.shift);
    a.n_freed[b] = e.n - kept0;
  }
}

// Weights of the kept tokens move to their new places; zeros behind them.
__global__ __launch_bounds__(256) void k_evict_pack(EvictArgs a) {
  const uint32_t b = blockIdx.z, h = blockIdx.y, j = blockIdx.x * 256 + threadIdx.x;
  if (j >= a.cap) return;
  float x = 0.f;
  if (j < a.out_lens[b]) {
    const uint32_t p = a.map[(size_t)b * a.s.max_pages + (j >> a.shift)];
    x = a.win.p[(int64_t)b * a.win.seq + (int64_t)h * a.win.head + ((size_t)p << a.shift) + (j & (a.page - 1))];
  }
  a.wout.p[(int64_t)b * a.wout.seq + (int64_t)h * a.wout.head + j] = x;
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
  k_evict_score<<<dim3((a.s.max_pages + 255) / 256, a.s.n_seq), 256, 0, st>>>(a);
  k_evict_select<<<a.s.n_seq, 1024, 0, st>>>(a);
  k_evict_pack<<<dim3((a.cap + 255) / 256, a.heads, a.s.n_seq), 256, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace gr
