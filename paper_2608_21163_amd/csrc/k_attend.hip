// k_attend.hip -- attention of chunks of new tokens over a paged cache.
//
// One wave holds 32 query rows as the columns of its products: S^T = K Q^T
// and O^T = V^T P^T, so a row's running maximum and sum stay in the lanes
// of its column (two lanes a row), and the probabilities leave the first
// product in the layout that the second one reads them in.  The new tokens
// of a sequence and the query heads that share a key/value head are packed
// into the rows (row = token * group + head in group): keys are read once
// for all of them.
#include "cache.h"

namespace gr {
namespace {

typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef short v8s __attribute__((ext_vector_type(8)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef float v4f __attribute__((ext_vector_type(4)));

constexpr float kLn2 = 0.69314718055994531f;

struct Bf16 {
  static constexpr uint32_t kExp = 0x7F807F80u, kExpLow = 0x00800080u, kInf = 0x7F80u;  // exponent bits of two elements, their lowest bits, of one
  typedef __bf16 T;
  typedef v8bf V;
  static __device__ __forceinline__ v16f mul(V a, V b, v16f c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};
struct F16 {
  static constexpr uint32_t kExp = 0x7C007C00u, kExpLow = 0x04000400u, kInf = 0x7C00u;
  typedef _Float16 T;
  typedef v8h V;
  static __device__ __forceinline__ v16f mul(V a, V b, v16f c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
};

__device__ __forceinline__ float neg_inf() { return -__builtin_inff(); }
__device__ __forceinline__ float ex2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float lg2(float x) { return __builtin_amdgcn_logf(x); }
__device__ __forceinline__ float other_half(float x) { return __shfl_xor(x, 32, 64); }

// The LDS writes of this workgroup (or wave) are visible after these; loads
// from global memory stay in flight.
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
__device__ __forceinline__ void lds_wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// Rows of LDS tiles: keys 16 bytes longer than their data, so that the 16
// bytes that consecutive rows read lie in consecutive banks; values a row
// length of 64 bytes modulo 128, so that the four rows of a transposing
// read cover all banks.
template <int DP> constexpr int k_row() { return DP * 2 + 16; }
template <int DP> constexpr int v_row() { return DP * 2 + ((DP * 2) % 128 == 0 ? 64 : 0); }
template <int DP, int KT> constexpr int tile_bytes() { return KT * (k_row<DP>() + v_row<DP>()); }

// Global loads of one tile of KT keys by NT threads into registers, and
// their way into LDS.  Keys at or past `end` repeat key end - 1.
template <int DP, int KT, int NT>
struct TileLoad {
  static constexpr int NCH = DP / 8;
  static constexpr int N = KT * NCH / NT;
  v4u k[N], v[N];
  uint32_t page[N];

  static __device__ __forceinline__ int row(int i, int t) { return (i * NT + t) / NCH; }
  static __device__ __forceinline__ int col(int i, int t) { return (i * NT + t) % NCH; }

  __device__ __forceinline__ void pages(const AttendArgs &a, const uint32_t *table, uint32_t key0, uint32_t end, int t) {
#pragma unroll
    for (int i = 0; i < N; i++) page[i] = table[min(key0 + row(i, t), end - 1) >> a.pg.shift];
  }
  // seq: where a page outside the pool is reported
  __device__ __forceinline__ void rows(const AttendArgs &a, uint32_t key0, uint32_t end, uint32_t kvh, int t, uint32_t seq) {
    const uint32_t mask = (1u << a.pg.shift) - 1;
    bool bad = false;
#pragma unroll
    for (int i = 0; i < N; i++) {
      const uint32_t slot = min(key0 + row(i, t), end - 1) & mask;
      bad |= page[i] >= a.pg.n_pages;
      const uint32_t p = min(page[i], a.pg.n_pages - 1);
      const int64_t off = (int64_t)p * a.pg.page + (int64_t)slot * a.pg.slot + (int64_t)kvh * a.pg.head + col(i, t) * 16;
      if (DP == 64 || col(i, t) * 8 < (int)a.dim || (DP & (DP - 1)) == 0) {
        const bool in = col(i, t) * 8 < (int)a.dim;
        const int64_t o = in ? off : off - col(i, t) * 16;
        k[i] = *(const v4u *)(a.pg.k + o);
        v[i] = *(const v4u *)(a.pg.v + o);
        if (!in) k[i] = v[i] = v4u{0, 0, 0, 0};
      } else {
        k[i] = v[i] = v4u{0, 0, 0, 0};
      }
    }
    if (bad) cache_err(a.err, kCachePage, seq);
  }
  __device__ __forceinline__ void store(uint8_t *lk, uint8_t *lv, int t) {
#pragma unroll
    for (int i = 0; i < N; i++) {
      *(v4u *)(lk + row(i, t) * k_row<DP>() + col(i, t) * 16) = k[i];
      *(v4u *)(lv + row(i, t) * v_row<DP>() + col(i, t) * 16) = v[i];
    }
  }
};

// The running state of a wave's 32 rows.
template <class E, int DP>
struct RowState {
  typename E::V q[DP / 16];
  v16f o[DP / 32];
  float m, l;  // maximum (raw score units) and this lane's share of the sum

  __device__ __forceinline__ void init(const AttendArgs &a, bool valid, uint32_t token, uint32_t head, int half) {
    m = neg_inf();
    l = 0.f;
#pragma unroll
    for (int d = 0; d < DP / 32; d++) o[d] = v16f{};
    const uint8_t *p = a.q.p + (int64_t)token * a.q.token + (int64_t)head * a.q.head;
#pragma unroll
    for (int s = 0; s < DP / 16; s++) {
      v4u x{0, 0, 0, 0};
      if (valid && (2 * s + half) * 8 < (int)a.dim) x = *(const v4u *)(p + (2 * s + half) * 16);
      q[s] = __builtin_bit_cast(typename E::V, x);
    }
  }
};

// The operand of O^T = V^T P^T for 16 keys (step t) and 32 elements (block d):
// two reads that transpose four keys by sixteen elements each.
template <class E, int DP>
__device__ __forceinline__ v8s v_operand(const uint8_t *lv, int t, int d, int lane) {
  const uint8_t *at = lv + (t * 16 + (lane >> 5) * 4 + (lane & 15) / 4) * v_row<DP>() + (d * 32 + ((lane >> 4) & 1) * 16 + (lane & 3) * 4) * 2;
  typedef __attribute__((address_space(3))) v4s *P;
  const v4s x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)at), y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(at + 8 * v_row<DP>()));
  return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
}

// Whether a value of the tile is infinite or NaN.  A hidden key's weight of
// zero would make NaN of it.
template <class E, int DP, int KT>
__device__ __forceinline__ bool has_non_finite(const uint8_t *lv, int lane) {
  uint32_t any = 0;
  constexpr int NCH = DP / 8;
#pragma unroll 4
  for (int i = 0; i < KT * NCH / 64; i++) {
    const int x = i * 64 + lane;
    const v4u v = *(const v4u *)(lv + x / NCH * v_row<DP>() + x % NCH * 16);
#pragma unroll
    for (int j = 0; j < 4; j++) any |= ((v[j] & E::kExp) + E::kExpLow) & 0x80008000u;
  }
  return __ballot(any != 0) != 0;
}

// One tile of KT keys: scores, running softmax, weighted values.
// pos: the row's position; keys past it (causal) or `window` before it are
// hidden, as are keys at or past end.  masked: some key of the tile is
// hidden from some row of the wave.  emit(kb, s): sees the scores of block kb.
template <class E, int DP, int KT, class F>
__device__ __forceinline__ void tile_step(RowState<E, DP> &st, const uint8_t *lk, const uint8_t *lv, float c, uint32_t key0,
                                          bool masked, int64_t first, int64_t last, int lane, F emit) {
  const int col = lane & 31, half = lane >> 5;
  v16f s[KT / 32];
#pragma unroll
  for (int kb = 0; kb < KT / 32; kb++) {
    v16f acc{};
#pragma unroll
    for (int x = 0; x < DP / 16; x++) {
      const v4u kk = *(const v4u *)(lk + (kb * 32 + col) * k_row<DP>() + (2 * x + half) * 16);
      acc = E::mul(__builtin_bit_cast(typename E::V, kk), st.q[x], acc);
    }
    s[kb] = acc;
  }
  if (masked) {
#pragma unroll
    for (int kb = 0; kb < KT / 32; kb++)
#pragma unroll
      for (int i = 0; i < 16; i++) {
        const int64_t key = (int64_t)key0 + kb * 32 + (i / 4) * 8 + half * 4 + i % 4;
        if (key < first || key > last) s[kb][i] = neg_inf();
      }
  }
  emit(s);
  float mx = st.m;
#pragma unroll
  for (int kb = 0; kb < KT / 32; kb++)
#pragma unroll
    for (int i = 0; i < 16; i++) mx = fmaxf(mx, s[kb][i]);
  mx = fmaxf(mx, other_half(mx));
  const float base = mx == neg_inf() ? 0.f : mx * c;
  const float scale = ex2(st.m == neg_inf() ? neg_inf() : st.m * c - base);
#pragma unroll
  for (int d = 0; d < DP / 32; d++)
#pragma unroll
    for (int i = 0; i < 16; i++) st.o[d][i] *= scale;
  st.m = mx;
  // a tile's sum first: the running sum then takes one rounding a tile
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int kb = 0; kb < KT / 32; kb++)
#pragma unroll
    for (int i = 0; i < 16; i++) {
      const float p = ex2(__builtin_fmaf(s[kb][i], c, -base));
      s[kb][i] = p;
      sum[i % 4] += p;
    }
  st.l = __builtin_fmaf(st.l, scale, (sum[0] + sum[1]) + (sum[2] + sum[3]));
  if (masked && has_non_finite<E, DP, KT>(lv, lane)) {
    // finite values as ever, then the infinities and NaN one key at a time,
    // to the rows that see it
#pragma unroll
    for (int t = 0; t < KT / 16; t++) {
      typename E::V p;
#pragma unroll
      for (int j = 0; j < 8; j++) p[j] = (typename E::T)s[t / 2][(t % 2) * 8 + j];
#pragma unroll
      for (int d = 0; d < DP / 32; d++) {
        v8s v = v_operand<E, DP>(lv, t, d, lane);
#pragma unroll
        for (int j = 0; j < 8; j++) v[j] = ((uint16_t)v[j] & E::kInf) == E::kInf ? (short)0 : v[j];
        st.o[d] = E::mul(__builtin_bit_cast(typename E::V, v), p, st.o[d]);
      }
    }
#pragma unroll 1
    for (int k = 0; k < KT; k++) {
      const bool see = (int64_t)key0 + k >= first && (int64_t)key0 + k <= last;
#pragma unroll
      for (int d = 0; d < DP / 32; d++)
#pragma unroll
        for (int i = 0; i < 16; i++) {
          const uint16_t u = *(const uint16_t *)(lv + k * v_row<DP>() + (d * 32 + (i / 4) * 8 + half * 4 + i % 4) * 2);
          if (see && (u & E::kInf) == E::kInf) st.o[d][i] += (float)__builtin_bit_cast(typename E::T, u);
        }
    }
    return;
  }
#pragma unroll
  for (int t = 0; t < KT / 16; t++) {
    // the probabilities enter the product in 16 bits, as the values are; the
    // sum l keeps them in 32
    typename E::V p;
#pragma unroll
    for (int j = 0; j < 8; j++) p[j] = (typename E::T)s[t / 2][(t % 2) * 8 + j];
#pragma unroll
    for (int d = 0; d < DP / 32; d++)
      st.o[d] = E::mul(__builtin_bit_cast(typename E::V, v_operand<E, DP>(lv, t, d, lane)), p, st.o[d]);
  }
}

// The keys that rows [first token, last token] of a chunk see.
__device__ __forceinline__ void key_range(const AttendArgs &a, const Chunk &c, uint32_t t0, uint32_t t1, uint32_t align,
                                          uint32_t &lo, uint32_t &hi) {
  int64_t l = 0, h = c.kl;
  if (a.causal) h = min(h, c.p0 + (int64_t)t1 + 1);
  if (a.window != 0xFFFFFFFFu) l = max((int64_t)0, c.p0 + (int64_t)t0 - (int64_t)a.window + 1);
  lo = (uint32_t)l / align * align;
  hi = (uint32_t)max(h, (int64_t)lo);
}

template <class E, int DP>
__device__ __forceinline__ void write_row(const AttendArgs &a, const v16f *o, float m, float l, uint32_t token, uint32_t head,
                                          uint32_t split, bool direct, int half) {
  const size_t row = (size_t)token * a.q_heads + head;
  if (direct) {
    const float inv = l > 0.f || l != l ? 1.f / l : 0.f;
    uint8_t *p = a.out.p + (int64_t)token * a.out.token + (int64_t)head * a.out.head;
#pragma unroll
    for (int d = 0; d < DP / 32; d++)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        const int at = d * 32 + (i / 4) * 8 + half * 4;
        if (at < (int)a.dim) {
          typename E::T x[4];
#pragma unroll
          for (int j = 0; j < 4; j++) x[j] = (typename E::T)(o[d][i + j] * inv);
          *(uint2 *)(p + at * 2) = *(uint2 *)x;
        }
      }
    if (half == 0) {
      const float z = l > 0.f || l != l ? m * a.c + lg2(l) : neg_inf();
      if (a.lse) a.lse[row] = z * kLn2;
      if (a.lse2) a.lse2[row] = z;
    }
  } else {
    float *p = a.part + (row * a.n_splits + split) * a.dim;
#pragma unroll
    for (int d = 0; d < DP / 32; d++)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        const int at = d * 32 + (i / 4) * 8 + half * 4;
        if (at < (int)a.dim) *(v4f *)(p + at) = v4f{o[d][i], o[d][i + 1], o[d][i + 2], o[d][i + 3]};
      }
    if (half == 0) a.part_ml[row * a.n_splits + split] = make_float2(l > 0.f || l != l ? m * a.c : neg_inf(), l);
  }
}

// Four waves of 32 rows each over shared tiles of KT keys.
template <class E, int DP, int KT>
__global__ __launch_bounds__(256, DP > 128 ? 1 : 2) void k_attend_rows(AttendArgs a) {
  extern __shared__ uint8_t smem[];
  const uint32_t kvh = blockIdx.x % a.kv_heads, rest = blockIdx.x / a.kv_heads;
  const uint32_t rt = rest % a.row_tiles, split = rest / a.row_tiles, b = blockIdx.y;
  const Chunk ch = chunk_of(a.s, b, a.err);
  const uint32_t rows = ch.ql * a.group, r0 = rt * kRowsTileRows;
  if (r0 >= rows) return;
  const uint32_t r1 = min(rows, r0 + kRowsTileRows) - 1;
  uint32_t lo, hi;
  key_range(a, ch, r0 / a.group, r1 / a.group, 32, lo, hi);
  const bool direct = a.n_splits == 1;
  const uint32_t begin = lo + split * a.split, end = min(hi, begin + a.split);
  if (split && begin >= hi) return;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6, half = lane >> 5;
  const uint32_t r = r0 + wave * 32 + (lane & 31), tok = min(r, r1) / a.group;
  const bool valid = r < rows;
  const uint32_t head = kvh * a.group + min(r, r1) % a.group;
  RowState<E, DP> st;
  st.init(a, valid, ch.r0 + tok, head, half);
  const int64_t pos = ch.p0 + tok;
  const int64_t last = a.causal ? min(pos, (int64_t)ch.kl - 1) : (int64_t)ch.kl - 1;
  const int64_t first = a.window != 0xFFFFFFFFu ? pos - (int64_t)a.window + 1 : 0;
  // positions of the wave's first and last row
  const uint32_t wr0 = min(r0 + wave * 32, r1), wr1 = min(r0 + wave * 32 + 31, r1);
  const int64_t wfirst = a.window != 0xFFFFFFFFu ? ch.p0 + wr1 / a.group - (int64_t)a.window + 1 : 0;
  const int64_t wlast = a.causal ? min(ch.p0 + wr0 / a.group, (int64_t)ch.kl - 1) : (int64_t)ch.kl - 1;
  if (begin < end) {
    const uint32_t *table = a.s.table + (int64_t)b * a.s.table_stride;
    TileLoad<DP, KT, 256> ld;
    ld.pages(a, table, begin, end, t);
    ld.rows(a, begin, end, kvh, t, b);
    ld.pages(a, table, min(begin + KT, end - 1), end, t);
    int buf = 0;
    for (uint32_t key0 = begin; key0 < end; key0 += KT, buf ^= 1) {
      uint8_t *lk = smem + buf * tile_bytes<DP, KT>(), *lv = lk + KT * k_row<DP>();
      ld.store(lk, lv, t);
      if (key0 + KT < end) {
        ld.rows(a, key0 + KT, end, kvh, t, b);
        ld.pages(a, table, min(key0 + 2 * KT, end - 1), end, t);
      }
      lds_barrier();
      const bool masked = (int64_t)key0 < wfirst || (int64_t)key0 + KT - 1 > wlast || key0 + KT > end;
      tile_step<E, DP, KT>(st, lk, lv, a.c, key0, masked, first, min(last, (int64_t)end - 1), lane, [](v16f *) {});
    }
  }
  st.l += other_half(st.l);
  if (valid) write_row<E, DP>(a, st.o, st.m, st.l, ch.r0 + tok, head, split, direct, half);
}

// Four waves of the same 32 rows, each over tiles of 32 keys of its own;
// their sums are joined at the end.
template <class E, int DP>
__global__ __launch_bounds__(256, DP > 128 ? 1 : 2) void k_attend_keys(AttendArgs a) {
  extern __shared__ uint8_t smem[];
  __shared__ float2 ml[4][32];
  const uint32_t kvh = blockIdx.x % a.kv_heads, rest = blockIdx.x / a.kv_heads;
  const uint32_t rt = rest % a.row_tiles, split = rest / a.row_tiles, b = blockIdx.y;
  const Chunk ch = chunk_of(a.s, b, a.err);
  const uint32_t rows = ch.ql * a.group, r0 = rt * kKeysTileRows;
  if (r0 >= rows) return;
  const uint32_t r1 = min(rows, r0 + kKeysTileRows) - 1;
  uint32_t lo, hi;
  key_range(a, ch, r0 / a.group, r1 / a.group, 32, lo, hi);
  const bool direct = a.n_splits == 1;
  const uint32_t begin = lo + split * a.split, end = min(hi, begin + a.split);
  if (split && begin >= hi) return;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6, half = lane >> 5;
  const uint32_t r = r0 + (lane & 31), tok = min(r, r1) / a.group;
  const bool valid = r < rows;
  const uint32_t head = kvh * a.group + min(r, r1) % a.group;
  RowState<E, DP> st;
  st.init(a, valid, ch.r0 + tok, head, half);
  const int64_t pos = ch.p0 + tok;
  const int64_t last = a.causal ? min(pos, (int64_t)ch.kl - 1) : (int64_t)ch.kl - 1;
  const int64_t first = a.window != 0xFFFFFFFFu ? pos - (int64_t)a.window + 1 : 0;
  const int64_t wfirst = a.window != 0xFFFFFFFFu ? ch.p0 + r1 / a.group - (int64_t)a.window + 1 : 0;
  const int64_t wlast = a.causal ? min(ch.p0 + r0 / a.group, (int64_t)ch.kl - 1) : (int64_t)ch.kl - 1;
  uint8_t *lk = smem + wave * tile_bytes<DP, 32>(), *lv = lk + 32 * k_row<DP>();
  uint32_t key0 = begin + wave * 32;
  if (key0 < end) {
    const uint32_t *table = a.s.table + (int64_t)b * a.s.table_stride;
    TileLoad<DP, 32, 64> ld;
    ld.pages(a, table, key0, end, lane);
    ld.rows(a, key0, end, kvh, lane, b);
    ld.pages(a, table, min(key0 + kKeysStep, end - 1), end, lane);
    for (; key0 < end; key0 += kKeysStep) {
      lds_wave_fence();
      ld.store(lk, lv, lane);
      if (key0 + kKeysStep < end) {
        ld.rows(a, key0 + kKeysStep, end, kvh, lane, b);
        ld.pages(a, table, min(key0 + 2 * kKeysStep, end - 1), end, lane);
      }
      lds_wave_fence();
      const bool masked = (int64_t)key0 < wfirst || (int64_t)key0 + 31 > wlast || key0 + 32 > end;
      tile_step<E, DP, 32>(st, lk, lv, a.c, key0, masked, first, min(last, (int64_t)end - 1), lane, [&](v16f *s) {
        if (a.scores && valid) {
          float *p = a.scores + (((size_t)b * a.kv_heads + kvh) * a.score_rows + r) * a.score_keys + key0 + half * 4;
#pragma unroll
          for (int i = 0; i < 16; i += 4)
            *(v4f *)(p + i * 2) = v4f{s[0][i] * a.c, s[0][i + 1] * a.c, s[0][i + 2] * a.c, s[0][i + 3] * a.c};
        }
      });
    }
  }
  st.l += other_half(st.l);
  if (half == 0) ml[wave][lane] = make_float2(st.m, st.l);
  __syncthreads();  // tiles are free, the waves' maxima known
  float m = neg_inf(), l = 0.f;
#pragma unroll
  for (int w = 0; w < 4; w++) m = fmaxf(m, ml[w][lane & 31].x);
#pragma unroll
  for (int w = 0; w < 4; w++) {
    const float2 x = ml[w][lane & 31];
    l += x.x == neg_inf() ? x.y : x.y * ex2((x.x - m) * a.c);
  }
  const float scale = st.m == neg_inf() ? 1.f : ex2((st.m - m) * a.c);
  // waves 3, 2, 1 add to one buffer in turn, wave 0 last
  float *sum = (float *)smem;
  constexpr int kStride = DP + 4;
  for (int w = 3; w >= 0; w--) {
    if (wave == w) {
      float *p = sum + (lane & 31) * kStride + half * 4;
#pragma unroll
      for (int d = 0; d < DP / 32; d++)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
          v4f x{st.o[d][i] * scale, st.o[d][i + 1] * scale, st.o[d][i + 2] * scale, st.o[d][i + 3] * scale};
          if (w < 3) {
            const v4f y = *(v4f *)(p + d * 32 + i * 2);
            x += y;
          }
          if (w > 0) {
            *(v4f *)(p + d * 32 + i * 2) = x;
          } else {
#pragma unroll
            for (int j = 0; j < 4; j++) st.o[d][i + j] = x[j];
          }
        }
    }
    if (w) __syncthreads();
  }
  if (wave == 0 && valid) write_row<E, DP>(a, st.o, m, l, ch.r0 + tok, head, split, direct, half);
}

// Joins the splits of one row: four waves, every fourth split each.
template <class E>
__global__ __launch_bounds__(256) void k_attend_join(AttendArgs a, uint32_t tile_rows) {
  __shared__ float2 ml[4];
  __shared__ float acc[4][256];
  const uint32_t b = blockIdx.y;
  const Chunk ch = chunk_of(a.s, b, a.err);
  const uint32_t kvh = blockIdx.x % a.kv_heads, r = blockIdx.x / a.kv_heads, rows = ch.ql * a.group;
  if (r >= rows) return;
  const uint32_t r0 = r / tile_rows * tile_rows, r1 = min(rows, r0 + tile_rows) - 1;
  uint32_t lo, hi;
  key_range(a, ch, r0 / a.group, r1 / a.group, 32, lo, hi);
  const uint32_t n = max(1u, (hi - lo + a.split - 1) / a.split);
  const uint32_t token = ch.r0 + r / a.group, head = kvh * a.group + r % a.group;
  const size_t row = (size_t)token * a.q_heads + head;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  float m = neg_inf(), l = 0.f;
  for (uint32_t s = wave * 64 + lane; s < n; s += 256) {
    const float2 x = a.part_ml[row * a.n_splits + s];
    const float mn = fmaxf(m, x.x);
    l = (m == neg_inf() ? l : l * ex2(m - mn)) + (x.x == neg_inf() ? x.y : x.y * ex2(x.x - mn));
    m = mn;
  }
#pragma unroll
  for (int j = 32; j; j >>= 1) {
    const float m2 = __shfl_xor(m, j, 64), l2 = __shfl_xor(l, j, 64), mn = fmaxf(m, m2);
    l = (m == neg_inf() ? l : l * ex2(m - mn)) + (m2 == neg_inf() ? l2 : l2 * ex2(m2 - mn));
    m = mn;
  }
  if (lane == 0) ml[wave] = make_float2(m, l);
  __syncthreads();
  m = neg_inf(), l = 0.f;
#pragma unroll
  for (int w = 0; w < 4; w++) m = fmaxf(m, ml[w].x);
#pragma unroll
  for (int w = 0; w < 4; w++) l += ml[w].x == neg_inf() ? ml[w].y : ml[w].y * ex2(ml[w].x - m);
  v4f o{0, 0, 0, 0};
  if (lane * 4 < (int)a.dim) {
    for (uint32_t s = wave; s < n; s += 4) {
      const float x = a.part_ml[row * a.n_splits + s].x;
      const float f = x == neg_inf() ? 1.f : ex2(x - m);
      o += *(const v4f *)(a.part + (row * a.n_splits + s) * a.dim + lane * 4) * f;
    }
  }
  *(v4f *)&acc[wave][lane * 4] = o;
  __syncthreads();
  const int d = threadIdx.x;
  const bool some = l > 0.f || l != l;
  if (d < (int)a.dim) {
    const float x = acc[0][d] + acc[1][d] + acc[2][d] + acc[3][d];
    *(typename E::T *)(a.out.p + (int64_t)token * a.out.token + (int64_t)head * a.out.head + d * 2) =
        (typename E::T)(some ? x / l : 0.f);
  }
  if (d == 0) {
    const float z = some ? m + lg2(l) : neg_inf();
    if (a.lse) a.lse[row] = z * kLn2;
    if (a.lse2) a.lse2[row] = z;
  }
}

// Weights from stored scores: a thread sums one key's weights over the rows.
__global__ __launch_bounds__(256) void k_weights_stored(AttendArgs a) {
  const uint32_t b = blockIdx.z, kvh = blockIdx.y;
  const Chunk ch = chunk_of(a.s, b, a.err);
  const uint32_t key = blockIdx.x * 256 + threadIdx.x;
  if (key >= ch.kl) return;
  float sum = a.win.p[(int64_t)b * a.win.seq + (int64_t)kvh * a.win.head + key];
  const uint32_t rows = ch.ql * a.group;
  for (uint32_t r0 = 0; r0 < rows; r0 += kKeysTileRows) {
    const uint32_t r1 = min(rows, r0 + kKeysTileRows);
    uint32_t lo, hi;
    key_range(a, ch, r0 / a.group, (r1 - 1) / a.group, 32, lo, hi);
    if (key < lo || key >= hi) continue;
    for (uint32_t r = r0; r < r1; r++) {
      const float z = a.lse2[(size_t)(ch.r0 + r / a.group) * a.q_heads + kvh * a.group + r % a.group];
      const float s = a.scores[(((size_t)b * a.kv_heads + kvh) * a.score_rows + r) * a.score_keys + key];
      sum += z == neg_inf() ? 0.f : ex2(s - z);
    }
  }
  a.wout.p[(int64_t)b * a.wout.seq + (int64_t)kvh * a.wout.head + key] = sum;
}

// Weights from scores computed again: a wave keeps 32 keys, the rows of the
// chunk pass by in tiles of 32.
template <class E, int DP>
__global__ __launch_bounds__(256, 2) void k_weights_again(AttendArgs a) {
  constexpr int kStride = DP * 2 + 16;
  __shared__ __align__(16) uint8_t lq[2][32 * kStride];
  __shared__ float lz[2][32];
  __shared__ float total[128];
  const uint32_t b = blockIdx.y, kvh = blockIdx.x % a.kv_heads, kt = blockIdx.x / a.kv_heads;
  const Chunk ch = chunk_of(a.s, b, a.err);
  const uint32_t key0 = kt * 128;
  if (key0 >= ch.kl) return;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6, half = lane >> 5, col = lane & 31;
  typename E::V k[DP / 16];
  {
    const uint32_t key = min(key0 + wave * 32 + col, ch.kl - 1);
    uint32_t p = a.s.table[(int64_t)b * a.s.table_stride + (key >> a.pg.shift)];
    p = min(p, a.pg.n_pages - 1);
    const uint8_t *at = a.pg.k + (int64_t)p * a.pg.page + (int64_t)(key & ((1u << a.pg.shift) - 1)) * a.pg.slot + (int64_t)kvh * a.pg.head;
#pragma unroll
    for (int s = 0; s < DP / 16; s++) {
      v4u x{0, 0, 0, 0};
      if ((2 * s + half) * 8 < (int)a.dim) x = *(const v4u *)(at + (2 * s + half) * 16);
      k[s] = __builtin_bit_cast(typename E::V, x);
    }
  }
  // rows that see a key of this tile
  const int64_t klast = min((int64_t)key0 + 127, (int64_t)ch.kl - 1);
  int64_t t_lo = a.causal ? max((int64_t)0, (int64_t)key0 - ch.p0) : 0;
  int64_t t_hi = a.window != 0xFFFFFFFFu ? min((int64_t)ch.ql, klast + (int64_t)a.window - ch.p0) : (int64_t)ch.ql;
  const uint32_t r_lo = (uint32_t)min(t_lo, (int64_t)ch.ql) * a.group, r_hi = (uint32_t)max(t_hi, (int64_t)0) * a.group;
  v16f acc{};
  constexpr int NCH = DP / 8, N = (32 * NCH + 255) / 256;
  v4u next[N];
  float nextz = 0.f;
  auto load = [&](uint32_t r0) {
#pragma unroll
    for (int i = 0; i < N; i++) {
      const int x = i * 256 + t;
      const uint32_t r = r0 + x / NCH;
      next[i] = v4u{0, 0, 0, 0};
      if (x < 32 * NCH && r < r_hi && (x % NCH) * 8 < (int)a.dim)
        next[i] = *(const v4u *)(a.q.p + (int64_t)(ch.r0 + r / a.group) * a.q.token + (int64_t)(kvh * a.group + r % a.group) * a.q.head + (x % NCH) * 16);
    }
    if (t < 32) {
      const uint32_t r = r0 + t;
      const float z = r < r_hi ? a.lse2[(size_t)(ch.r0 + r / a.group) * a.q_heads + kvh * a.group + r % a.group] : neg_inf();
      nextz = z == neg_inf() ? __builtin_inff() : z;
    }
  };
  if (r_lo < r_hi) load(r_lo);
  int buf = 0;
  for (uint32_t r0 = r_lo; r0 < r_hi; r0 += 32, buf ^= 1) {
#pragma unroll
    for (int i = 0; i < N; i++) {
      const int x = i * 256 + t;
      if (x < 32 * NCH) *(v4u *)(lq[buf] + (x / NCH) * kStride + (x % NCH) * 16) = next[i];
    }
    if (t < 32) lz[buf][t] = nextz;
    if (r0 + 32 < r_hi) load(r0 + 32);
    lds_barrier();
    v16f s{};
#pragma unroll
    for (int x = 0; x < DP / 16; x++) {
      const v4u q = *(const v4u *)(lq[buf] + col * kStride + (2 * x + half) * 16);
      s = E::mul(k[x], __builtin_bit_cast(typename E::V, q), s);
    }
    const float z = lz[buf][col];
    const int64_t p_lo = ch.p0 + r0 / a.group, p_hi = ch.p0 + min(r0 + 31, r_hi - 1) / a.group;
    const bool masked = (a.causal && (int64_t)key0 + wave * 32 + 31 > p_lo) ||
                        (a.window != 0xFFFFFFFFu && (int64_t)key0 + wave * 32 <= p_hi - (int64_t)a.window);
    if (masked) {
      const int64_t pos = ch.p0 + min(r0 + col, r_hi - 1) / a.group;
#pragma unroll
      for (int i = 0; i < 16; i++) {
        const int64_t key = (int64_t)key0 + wave * 32 + (i / 4) * 8 + half * 4 + i % 4;
        if ((a.causal && key > pos) || (a.window != 0xFFFFFFFFu && key <= pos - (int64_t)a.window)) s[i] = neg_inf();
      }
    }
#pragma unroll
    for (int i = 0; i < 16; i++) acc[i] += ex2(__builtin_fmaf(s[i], a.c, -z));
  }
#pragma unroll
  for (int i = 0; i < 16; i++) {
    float x = acc[i];
#pragma unroll
    for (int j = 16; j; j >>= 1) x += __shfl_xor(x, j, 64);
    if (col == 0) total[wave * 32 + (i / 4) * 8 + half * 4 + i % 4] = x;
  }
  __syncthreads();
  const uint32_t key = key0 + t;
  if (t < 128 && key < ch.kl)
    a.wout.p[(int64_t)b * a.wout.seq + (int64_t)kvh * a.wout.head + key] =
        a.win.p[(int64_t)b * a.win.seq + (int64_t)kvh * a.win.head + key] + total[t];
}

template <class E, int DP>
hipError_t attend_dim(int mode, const AttendArgs &a, hipStream_t st) {
  const dim3 grid(a.kv_heads * a.row_tiles * a.n_splits, a.s.n_seq);
  if (mode == kRows) {
    constexpr int KT = DP > 128 ? 32 : 64;
    k_attend_rows<E, DP, KT><<<grid, 256, 2 * tile_bytes<DP, KT>(), st>>>(a);
  } else {
    k_attend_keys<E, DP><<<grid, 256, 4 * tile_bytes<DP, 32>(), st>>>(a);
  }
  return hipGetLastError();
}

template <class E>
hipError_t attend_type(int mode, const AttendArgs &a, hipStream_t st) {
  if (a.dim <= 64) return attend_dim<E, 64>(mode, a, st);
  if (a.dim <= 128) return attend_dim<E, 128>(mode, a, st);
  return attend_dim<E, 256>(mode, a, st);
}

template <class E>
hipError_t weights_type(const AttendArgs &a, hipStream_t st) {
  const dim3 grid((a.s.max_k + 127) / 128 * a.kv_heads, a.s.n_seq);
  if (a.dim <= 64) k_weights_again<E, 64><<<grid, 256, 0, st>>>(a);
  else if (a.dim <= 128) k_weights_again<E, 128><<<grid, 256, 0, st>>>(a);
  else k_weights_again<E, 256><<<grid, 256, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_attend(int mode, bool f16, const AttendArgs &a, hipStream_t st) {
  return f16 ? attend_type<F16>(mode, a, st) : attend_type<Bf16>(mode, a, st);
}

hipError_t launch_attend_join(bool f16, const AttendArgs &a, uint32_t tile_rows, hipStream_t st) {
  const dim3 grid(a.s.max_q * a.q_heads, a.s.n_seq);
  if (f16) k_attend_join<F16><<<grid, 256, 0, st>>>(a, tile_rows);
  else k_attend_join<Bf16><<<grid, 256, 0, st>>>(a, tile_rows);
  return hipGetLastError();
}

hipError_t launch_attend_weights(bool f16, const AttendArgs &a, hipStream_t st) {
  if (a.scores) {
    k_weights_stored<<<dim3((a.s.max_k + 255) / 256, a.kv_heads, a.s.n_seq), 256, 0, st>>>(a);
    return hipGetLastError();
  }
  return f16 ? weights_type<F16>(a, st) : weights_type<Bf16>(a, st);
}

}  // namespace gr
