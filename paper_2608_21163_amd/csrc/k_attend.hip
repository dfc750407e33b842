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

// kUp, kLagUp: probabilities enter their product at 2^kUp times their size
// where the largest is 1, at 2^kLagUp times where it may reach 2^8 (tile_step).
// fp16 has steps of 2^-24 below 2^-14: the weight of tokens 2^-25 of the largest
// and less would be lost from the results, though not from the sum that divides
// them, however many they are.  Powers of two, taken back at the end.
struct Bf16 {
  static constexpr int kUp = 0, kLagUp = 0;
  static constexpr uint32_t kExp = 0x7F807F80u, kExpLow = 0x00800080u, kInf = 0x7F80u;  // exponent bits of two elements, their lowest bits, of one
  typedef __bf16 T;
  typedef v8bf V;
  static __device__ __forceinline__ v16f mul(V a, V b, v16f c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
  static __device__ __forceinline__ v4f mul16(V a, V b, v4f c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
struct F16 {
  static constexpr int kUp = 14, kLagUp = 7;
  static constexpr uint32_t kExp = 0x7C007C00u, kExpLow = 0x04000400u, kInf = 0x7C00u;
  typedef _Float16 T;
  typedef v8h V;
  static __device__ __forceinline__ v16f mul(V a, V b, v16f c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
  static __device__ __forceinline__ v4f mul16(V a, V b, v4f c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};

__device__ __forceinline__ float neg_inf() { return -__builtin_inff(); }
constexpr float down(int up) { return 1.f / (float)(1 << up); }
__device__ __forceinline__ float ex2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float lg2(float x) { return __builtin_amdgcn_logf(x); }

// Both halves of the wave (both rows of 16 of each half) in every lane.
template <class F> __device__ __forceinline__ float halves(float x, F f) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return f(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
template <class F> __device__ __forceinline__ float rows16(float x, F f) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return f(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float fmax2(float a, float b) { return fmaxf(a, b); }
__device__ __forceinline__ float fadd2(float a, float b) { return a + b; }

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

// Global loads of one tile of KT keys by 256 threads into registers, and
// their way into LDS.  LPR lanes load a row, 16 bytes each (some idle where
// rows are not a power of two long); a lane loads a piece of N consecutive
// keys, which mostly lie in one page.  A key at or past `end` reads some slot
// of the pool and is hidden.
template <int DP, int KT>
struct TileLoad {
  static constexpr int LPR = DP <= 64 ? 8 : DP <= 128 ? 16 : 32, N = KT * LPR / 256;
  v4u k[N], v[N];
  uint32_t page[N];
  int piece, krow;
  bool in, one_page;

  __device__ __forceinline__ TileLoad(const AttendArgs &a, int t) {
    piece = t % LPR;
    krow = t / LPR * N;
    in = piece * 8 < (int)a.dim;
    one_page = (1u << a.pg.shift) >= N;
  }
  __device__ __forceinline__ void pages(const AttendArgs &a, const uint32_t *table, uint32_t key0) {
    if (one_page) {
      page[0] = table[min((key0 + krow) >> a.pg.shift, a.s.max_pages - 1)];
    } else {
#pragma unroll
      for (int i = 0; i < N; i++) page[i] = table[min((key0 + krow + i) >> a.pg.shift, a.s.max_pages - 1)];
    }
  }
  // Of the keys from seen to end, a page outside the pool is reported of seq;
  // what lies before them is hidden, and a window's user may have freed it.
  __device__ __forceinline__ void rows(const AttendArgs &a, uint32_t key0, uint32_t seen, uint32_t end, uint32_t kvh, uint32_t seq) {
    const uint32_t mask = (1u << a.pg.shift) - 1, in_head = kvh * a.pg.head + (in ? piece * 16 : 0);
    bool bad = false;
    if (one_page) {
      bad = page[0] >= a.pg.n_pages && key0 + krow < end && key0 + krow + N > seen;
      const uint64_t off = (uint64_t)min(page[0], a.pg.n_pages - 1) * a.pg.page + (((key0 + krow) & mask) * a.pg.slot + in_head);
#pragma unroll
      for (int i = 0; i < N; i++) {
        k[i] = *(const v4u *)(a.pg.k + off + i * a.pg.slot);
        v[i] = *(const v4u *)(a.pg.v + off + i * a.pg.slot);
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; i++) {
        bad |= page[i] >= a.pg.n_pages && key0 + krow + i < end && key0 + krow + i >= seen;
        const uint64_t off = (uint64_t)min(page[i], a.pg.n_pages - 1) * a.pg.page + (((key0 + krow + i) & mask) * a.pg.slot + in_head);
        k[i] = *(const v4u *)(a.pg.k + off);
        v[i] = *(const v4u *)(a.pg.v + off);
      }
    }
    if (bad) cache_err(a.err, kCachePage, seq);
  }
  // Infinite and NaN values become 0; returns whether there were any among
  // the keys before end.
  template <class E>
  __device__ __forceinline__ bool clear_non_finite(uint32_t key0, uint32_t end) {
    uint32_t any = 0;
#pragma unroll
    for (int i = 0; i < N; i++)
#pragma unroll
      for (int j = 0; j < 4; j++) {
        const uint32_t odd = ((v[i][j] & E::kExp) + E::kExpLow) & 0x80008000u;  // the sign bits of such elements
        if (key0 + krow + i < end) any |= odd;
        v[i][j] &= ~((odd >> 15) * 0xFFFFu);
      }
    return any != 0;
  }
  // Elements past dim: the keys' are zeros, as the queries' are, the values'
  // are whatever was loaded, as their sums are not written.
  __device__ __forceinline__ void store(const AttendArgs &a, uint8_t *lk, uint8_t *lv) {
    if (a.dim != DP && !in) {
#pragma unroll
      for (int i = 0; i < N; i++) k[i] = v4u{0, 0, 0, 0};
    }
    if (LPR * 8 == DP || piece * 8 < DP) {
#pragma unroll
      for (int i = 0; i < N; i++) {
        *(v4u *)(lk + (krow + i) * k_row<DP>() + piece * 16) = k[i];
        *(v4u *)(lv + (krow + i) * v_row<DP>() + piece * 16) = v[i];
      }
    }
  }
};

// The running state of a wave's 32 rows.
template <class E, int DP>
struct RowState {
  typename E::V q[DP / 16];
  v16f o[DP / 32];
  // what scores are taken against (log2 units, kLagUp below a maximum; -inf: no key seen), this lane's share of the sum
  float m, l;

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

// Adds the infinite and NaN values of the keys [begin, end) to the rows that
// see them.  Tiles with a key that is hidden from some row hold zeros in their
// place, as a hidden key's weight of zero would make NaN of them; in other
// tiles the product took them already, and what is infinite or NaN stays so.
// (There a probability that 16 bits round to 0 makes NaN of an infinite value,
// where a tile with hidden keys gives the infinity.)
template <class E, int DP>
__device__ __forceinline__ void add_non_finite(const AttendArgs &a, const uint32_t *table, uint32_t kvh, uint32_t begin, uint32_t end,
                                               int first, int last, int half, v16f *o) {
  for (uint32_t key = begin; key < end; key++) {
    const uint32_t page = min(table[key >> a.pg.shift], a.pg.n_pages - 1), slot = key & ((1u << a.pg.shift) - 1);
    const uint8_t *p = a.pg.v + (uint64_t)page * a.pg.page + (slot * a.pg.slot + kvh * a.pg.head);
    const bool see = (int)key >= first && (int)key <= last;
#pragma unroll
    for (int d = 0; d < DP / 32; d++)
#pragma unroll
      for (int i = 0; i < 16; i++) {
        const int at = d * 32 + (i / 4) * 8 + half * 4 + i % 4;
        if (at < (int)a.dim) {
          const uint16_t u = *(const uint16_t *)(p + at * 2);
          if (see && (u & E::kInf) == E::kInf) o[d][i] += (float)__builtin_bit_cast(typename E::T, u);
        }
      }
  }
}

// One tile of KT keys: scores, running softmax, weighted values.
// pos: the row's position; keys past it (causal) or `window` before it are
// hidden, as are keys at or past end.  masked: some key of the tile is
// hidden from some row of the wave.
template <class E, int DP, int KT>
__device__ __forceinline__ void tile_step(RowState<E, DP> &st, const uint8_t *lk, const uint8_t *lv, float c, uint32_t key0,
                                          bool masked, int first, int last, int lane) {
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
    // (opaque, or the compiler computes every comparison in every tile)
    uint32_t k0 = key0;
    asm volatile("" : "+s"(k0));
#pragma unroll
    for (int kb = 0; kb < KT / 32; kb++)
#pragma unroll
      for (int i = 0; i < 16; i++) {
        const int key = (int)k0 + kb * 32 + (i / 4) * 8 + half * 4 + i % 4;
        if (key < first || key > last) s[kb][i] = neg_inf();
      }
  }
  float mx = s[0][0];
#pragma unroll
  for (int kb = 0; kb < KT / 32; kb++)
#pragma unroll
    for (int i = 0; i < 16; i++) mx = fmaxf(mx, s[kb][i]);
  mx = halves(mx, fmax2);
  // The maximum that scores are taken against follows the true one only
  // when that passes it by 2^8 for some row: sums and values then stay below
  // 2^8 times what they would be, and most tiles need no rescaling.  The
  // largest probability is then rounded too, not 1: bf16 results are 0.0023 off
  // on average instead of 0.0020 (their own rounding is 0.0017); following the
  // true maximum costs 1 to 6%.
  const float top = mx * c - E::kLagUp;
  if (__ballot(top > st.m + 8.f)) {
    const float mn = fmaxf(st.m, top);
    const float scale = st.m == neg_inf() ? 0.f : ex2(st.m - mn);
#pragma unroll
    for (int d = 0; d < DP / 32; d++)
#pragma unroll
      for (int i = 0; i < 16; i++) st.o[d][i] *= scale;
    st.l *= scale;
    st.m = mn;
  }
  const float base = st.m == neg_inf() ? 0.f : st.m;
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
  st.l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
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

// The keys that rows [first token, last token] of a chunk see: from the result
// on, lo is that rounded down to `align`, to before hi.
__device__ __forceinline__ uint32_t key_range(const AttendArgs &a, const Chunk &c, uint32_t t0, uint32_t t1, uint32_t align,
                                              uint32_t &lo, uint32_t &hi) {
  int l = 0, h = (int)c.kl;
  if (a.causal) h = min(h, c.p0 + (int)t1 + 1);
  if (a.window) l = max(0, c.p0 + (int)t0 - (int)a.window + 1);
  lo = (uint32_t)l / align * align;
  hi = (uint32_t)max(h, (int)lo);
  return (uint32_t)l;
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
      const float z = l > 0.f || l != l ? m + lg2(l) : neg_inf();
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
    if (half == 0) a.part_ml[row * a.n_splits + split] = make_float2(l > 0.f || l != l ? m : neg_inf(), l);
  }
}

// Four waves of 32 rows each over shared tiles of KT keys: chunks.  A wave
// reads each tile's keys and values once from LDS for 32 rows, 32 cycles of
// the matrix unit a 1 KB operand.  2,048 tokens of 32 heads over 32,768 cached
// ones take 1.13 to 1.20 ms, 0.89 to 0.94 PFLOP/s, where a large library product
// reaches 1.23; the matrix unit is busy 45% of the time, the vector unit
// (exponentials, sums, maxima, rounding) 55%, LDS 36%.  Tiles of 32 keys are 5%
// slower, 256 rows a workgroup 5%, the next block's scores beside this one's
// softmax 3%, operands read ahead of the products 0 to 3%; splits read the
// keys again through L2.
template <class E, int DP, int KT>
__global__ __launch_bounds__(256, DP > 128 ? 1 : 2) void k_attend_rows(AttendArgs a) {
  extern __shared__ uint8_t smem[];
  const uint32_t kvh = blockIdx.x % a.kv_heads, rest = blockIdx.x / a.kv_heads;
  const uint32_t rt = rest % a.row_tiles, split = rest / a.row_tiles, b = blockIdx.y;
  const Chunk ch = chunk_of(a.s, b, a.err);
  const uint32_t rows = ch.ql * a.group, r0 = rt * kManyRows;
  if (r0 >= rows) return;
  const uint32_t r1 = min(rows, r0 + kManyRows) - 1;
  uint32_t lo, hi;
  const uint32_t seen = key_range(a, ch, r0 / a.group, r1 / a.group, 32, lo, hi);
  const bool direct = a.n_splits == 1;
  const uint32_t begin = lo + split * a.split, end = min(hi, begin + a.split);
  if (split && begin >= hi) return;
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), half = lane >> 5;
  const uint32_t r = r0 + wave * 32 + (lane & 31), tok = min(r, r1) / a.group;
  const bool valid = r < rows;
  const uint32_t head = kvh * a.group + min(r, r1) % a.group;
  RowState<E, DP> st;
  st.init(a, valid, ch.r0 + tok, head, half);
  const int pos = ch.p0 + (int)tok;
  const int last = a.causal ? min(pos, (int)ch.kl - 1) : (int)ch.kl - 1;
  const int first = a.window ? pos - (int)a.window + 1 : 0;
  // positions of the wave's first and last row
  const uint32_t wr0 = min(r0 + wave * 32, r1), wr1 = min(r0 + wave * 32 + 31, r1);
  const int wfirst = a.window ? ch.p0 + (int)(wr1 / a.group) - (int)a.window + 1 : 0;
  const int wlast = a.causal ? min(ch.p0 + (int)(wr0 / a.group), (int)ch.kl - 1) : (int)ch.kl - 1;
  if (begin < end) {
    const uint32_t *table = a.s.table + (int64_t)b * a.s.table_stride;
    // the whole workgroup's rows see every key from all0 to all1
    const int all0 = a.window ? ch.p0 + (int)(r1 / a.group) - (int)a.window + 1 : 0;
    const int all1 = min(a.causal ? min(ch.p0 + (int)(r0 / a.group), (int)ch.kl - 1) : (int)ch.kl - 1, (int)end - 1);
    bool odd = false;
    TileLoad<DP, KT> ld(a, t);
    ld.pages(a, table, begin);
    ld.rows(a, begin, seen, end, kvh, b);
    ld.pages(a, table, begin + KT);
    int buf = 0;
    for (uint32_t key0 = begin; key0 < end; key0 += KT, buf ^= 1) {
      uint8_t *lk = smem + buf * tile_bytes<DP, KT>(), *lv = lk + KT * k_row<DP>();
      if ((int)key0 < all0 || (int)key0 + KT - 1 > all1) odd |= ld.template clear_non_finite<E>(key0, end);
      ld.store(a, lk, lv);
      if (key0 + KT < end) {
        ld.rows(a, key0 + KT, seen, end, kvh, b);
        ld.pages(a, table, key0 + 2 * KT);
      }
      lds_barrier();
      const bool masked = (int)key0 < wfirst || (int)key0 + KT - 1 > min(wlast, (int)end - 1);
      tile_step<E, DP, KT>(st, lk, lv, a.c, key0, masked, first, min(last, (int)end - 1), lane);
    }
    if (__syncthreads_or(odd)) add_non_finite<E, DP>(a, table, kvh, begin, end, first, last, half, st.o);
  }
  st.l = halves(st.l, fadd2) * down(E::kLagUp);
  st.m += E::kLagUp;
#pragma unroll
  for (int d = 0; d < DP / 32; d++) st.o[d] *= down(E::kLagUp);
  if (valid) write_row<E, DP>(a, st.o, st.m, st.l, ch.r0 + tok, head, split, direct, half);
}

// Four waves of the same 16 NB rows, each over every fourth tile of 32 keys;
// their sums are joined at the end.  For the few rows of single tokens and
// short chunks: the time is that of the cache's bytes, so what counts is how
// many loads are in flight and that each takes whole cache lines, past which
// the caches are told not to keep them (an instruction reads whole rows of 2
// to 8 keys).  A tile's keys, then its values pass through the same LDS.
// 64 tokens over 1 to 8,192 cached ones, 1.15 GB: 196 to 205 us, 5.6 to 5.9
// TB/s, where a plain read of as much takes 174 (past the caches) to 195.  The
// whole call takes 210 to 213 us, 239 with loads that the caches keep, 258
// with 64 bytes of 16 rows an instruction.
template <class E, int DP, int NB>
__global__ __launch_bounds__(256, DP > 192 || (DP > 128 && NB > 1) ? 1 : DP > 128 || NB > 1 ? 2 : 3) void k_attend_few(AttendArgs a) {
  typedef typename E::V V;
  constexpr int NS = DP / 32, KROW = k_row<DP>(), VROW = v_row<DP>(), ROWS = 16 * NB;
  constexpr int LPR = DP <= 64 ? 8 : DP <= 128 ? 16 : 32;  // lanes that load a row, 16 bytes each (96, 192: some idle)
  constexpr int N = LPR / 2;                               // consecutive keys of a tile that a lane loads a piece of
  constexpr int kSum = DP + 4;  // floats of a row of the waves' sums
  constexpr int kTiles = 4 * 32 * (VROW > KROW ? VROW : KROW), kSums = 4 * 16 * kSum * 4;
  __shared__ __align__(16) uint8_t smem[kTiles > kSums ? kTiles : kSums];
  __shared__ float2 ml[4][16];
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), g = lane >> 4, c = lane & 15;
  // Workgroups go to the eight XCDs in turn.  A unit (sequence, row tile,
  // split) has all its heads on one of them, one after the other: a slot's
  // heads lie side by side, and an XCD that had one head only would read
  // through an eighth of its L2 channels.
  const uint32_t unit = blockIdx.x / (8 * a.kv_heads) * 8 + blockIdx.x % 8, kvh = blockIdx.x / 8 % a.kv_heads;
  const uint32_t b = unit % a.s.n_seq, rt = unit / a.s.n_seq % a.row_tiles, split = unit / a.s.n_seq / a.row_tiles;
  if (split >= a.n_splits) return;
  const uint32_t *table = a.s.table + (int64_t)b * a.s.table_stride;
  const int piece = lane % LPR, krow = lane / LPR * N;
  const bool in = piece * 8 < (int)a.dim;
  // pages of at least N slots hold all N keys
  const bool one_page = a.pg.shift >= (DP <= 64 ? 2 : DP <= 128 ? 3 : 4);
  // the first page ids are asked for together with the lengths where the
  // split's first key does not depend on them
  uint32_t page[N];
  auto pages = [&](uint32_t key0) {
    if (one_page) {
      page[0] = table[min((key0 + krow) >> a.pg.shift, a.s.max_pages - 1)];
    } else {
#pragma unroll
      for (int i = 0; i < N; i++) page[i] = table[min((key0 + krow + i) >> a.pg.shift, a.s.max_pages - 1)];
    }
  };
  if (a.s.max_pages) pages(split * a.split + wave * 32);
  const Chunk ch = chunk_of(a.s, b, a.err);
  const uint32_t rows = ch.ql * a.group, r0 = rt * ROWS;
  if (r0 >= rows) return;
  const uint32_t r1 = min(rows, r0 + ROWS) - 1;
  uint32_t lo, hi;
  const uint32_t seen = key_range(a, ch, r0 / a.group, r1 / a.group, 32, lo, hi);
  const uint32_t begin = lo + split * a.split, end = min(hi, begin + a.split);
  if (split && begin >= hi) return;
  if (lo) pages(begin + wave * 32);

  V q[NB][NS];
  int first[NB], last[NB];
#pragma unroll
  for (int nb = 0; nb < NB; nb++) {
    const uint32_t r = min(r0 + nb * 16 + c, r1), tok = r / a.group;
    const uint8_t *p = a.q.p + (int64_t)(ch.r0 + tok) * a.q.token + (int64_t)(kvh * a.group + r % a.group) * a.q.head;
#pragma unroll
    for (int s = 0; s < NS; s++) {
      v4u x{0, 0, 0, 0};
      if ((s * 4 + g) * 8 < (int)a.dim) x = *(const v4u *)(p + (s * 4 + g) * 16);
      q[nb][s] = __builtin_bit_cast(V, x);
    }
    const int pos = ch.p0 + (int)tok;
    last[nb] = min(a.causal ? min(pos, (int)ch.kl - 1) : (int)ch.kl - 1, (int)end - 1);
    first[nb] = a.window ? pos - (int)a.window + 1 : 0;
  }
  // every row sees the keys from all0 to all1
  const int all0 = a.window ? ch.p0 + (int)(r1 / a.group) - (int)a.window + 1 : 0;
  const int all1 = a.causal ? min(ch.p0 + (int)(r0 / a.group), (int)ch.kl - 1) : (int)ch.kl - 1;

  v4f o[NB][DP / 16];
  float m[NB], l[NB];
#pragma unroll
  for (int nb = 0; nb < NB; nb++) {
    m[nb] = neg_inf();
    l[nb] = 0.f;
#pragma unroll
    for (int d = 0; d < DP / 16; d++) o[nb][d] = v4f{0, 0, 0, 0};
  }
  // keys and values of the lane's N keys of a tile; a key at or past `end`
  // reads some slot of the pool and is hidden
  v4u kx[N], vx[N];
  uint64_t off[N];
  bool odd = false;
  auto offsets = [&](uint32_t key0) {
    bool bad = false;
    const uint32_t mask = (1u << a.pg.shift) - 1, in_head = kvh * a.pg.head + (in ? piece * 16 : 0);
    if (one_page) {
      bad = page[0] >= a.pg.n_pages && key0 + krow < end && key0 + krow + N > seen;
      off[0] = (uint64_t)min(page[0], a.pg.n_pages - 1) * a.pg.page + (((key0 + krow) & mask) * a.pg.slot + in_head);
#pragma unroll
      for (int i = 1; i < N; i++) off[i] = off[i - 1] + a.pg.slot;
    } else {
#pragma unroll
      for (int i = 0; i < N; i++) {
        bad |= page[i] >= a.pg.n_pages && key0 + krow + i < end && key0 + krow + i >= seen;
        off[i] = (uint64_t)min(page[i], a.pg.n_pages - 1) * a.pg.page + (((key0 + krow + i) & mask) * a.pg.slot + in_head);
      }
    }
    if (bad) cache_err(a.err, kCachePage, b);
  };
  auto load_k = [&] {
#pragma unroll
    for (int i = 0; i < N; i++) kx[i] = __builtin_nontemporal_load((const v4u *)(a.pg.k + off[i]));
  };
  auto load_v = [&] {
#pragma unroll
    for (int i = 0; i < N; i++) vx[i] = __builtin_nontemporal_load((const v4u *)(a.pg.v + off[i]));
  };
  uint8_t *lt = smem + wave * (kTiles / 4);
  uint32_t key0 = begin + wave * 32;
  if (key0 < end) {
    offsets(key0);
    load_k();
    load_v();
    pages(key0 + kKeysStep);
    for (; key0 < end; key0 += kKeysStep) {
      const bool masked = (int)key0 < all0 || (int)key0 + 31 > min(all1, (int)end - 1), more = key0 + kKeysStep < end;
      if (a.dim != DP && !in) {
#pragma unroll
        for (int i = 0; i < N; i++) kx[i] = v4u{0, 0, 0, 0};
      }
      lds_wave_fence();
      if (LPR * 8 == DP || piece * 8 < DP) {
#pragma unroll
        for (int i = 0; i < N; i++) *(v4u *)(lt + (krow + i) * KROW + piece * 16) = kx[i];
      }
      lds_wave_fence();
      v4f sc[NB][2];
#pragma unroll
      for (int kb = 0; kb < 2; kb++) {
#pragma unroll
        for (int nb = 0; nb < NB; nb++) sc[nb][kb] = v4f{0, 0, 0, 0};
#pragma unroll
        for (int s = 0; s < NS; s++) {
          const v4u x = *(const v4u *)(lt + (kb * 16 + c) * KROW + (s * 4 + g) * 16);
#pragma unroll
          for (int nb = 0; nb < NB; nb++) sc[nb][kb] = E::mul16(__builtin_bit_cast(V, x), q[nb][s], sc[nb][kb]);
        }
      }
      if (masked) {
        uint32_t any = 0;
#pragma unroll
        for (int i = 0; i < N; i++)
#pragma unroll
          for (int j = 0; j < 4; j++) {
            const uint32_t bits = ((vx[i][j] & E::kExp) + E::kExpLow) & 0x80008000u;
            if (key0 + krow + i < end) any |= bits;
            vx[i][j] &= ~((bits >> 15) * 0xFFFFu);
          }
        odd |= any != 0;
      }
      lds_wave_fence();
      if (LPR * 8 == DP || piece * 8 < DP) {
#pragma unroll
        for (int i = 0; i < N; i++) *(v4u *)(lt + (krow + i) * VROW + piece * 16) = vx[i];
      }
      if (more) {
        offsets(key0 + kKeysStep);
        load_k();
        load_v();
        pages(key0 + 2 * kKeysStep);
      }
      lds_wave_fence();
      if (masked) {
        uint32_t k0 = key0;
        asm volatile("" : "+s"(k0));
#pragma unroll
        for (int nb = 0; nb < NB; nb++)
#pragma unroll
          for (int kb = 0; kb < 2; kb++)
#pragma unroll
            for (int i = 0; i < 4; i++) {
              const int key = (int)k0 + kb * 16 + g * 4 + i;
              if (key < first[nb] || key > last[nb]) sc[nb][kb][i] = neg_inf();
            }
      }
      V p[NB];
#pragma unroll
      for (int nb = 0; nb < NB; nb++) {
        if (a.scores && r0 + nb * 16 + c <= r1) {
          float *to = a.scores + (((size_t)b * a.kv_heads + kvh) * a.score_rows + r0 + nb * 16 + c) * a.score_keys + key0 + g * 4;
          *(v4f *)to = sc[nb][0] * a.c;
          *(v4f *)(to + 16) = sc[nb][1] * a.c;
        }
        float mx = fmaxf(fmaxf(fmaxf(sc[nb][0][0], sc[nb][0][1]), fmaxf(sc[nb][0][2], sc[nb][0][3])),
                         fmaxf(fmaxf(sc[nb][1][0], sc[nb][1][1]), fmaxf(sc[nb][1][2], sc[nb][1][3])));
        mx = halves(rows16(mx, fmax2), fmax2) * a.c - E::kUp;
        // the true maximum (unlike tile_step's): the largest probability is
        // then a power of two, which 16 bits hold, and the loads hide the rescaling
        if (__ballot(mx > m[nb])) {
          const float mn = fmaxf(m[nb], mx), scale = m[nb] == neg_inf() ? 0.f : ex2(m[nb] - mn);
#pragma unroll
          for (int d = 0; d < DP / 16; d++) o[nb][d] *= scale;
          l[nb] *= scale;
          m[nb] = mn;
        }
        const float base = m[nb] == neg_inf() ? 0.f : m[nb];
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < 8; j++) {
          const float x = ex2(__builtin_fmaf(sc[nb][j / 4][j % 4], a.c, -base));
          sum += x;
          p[nb][j] = (typename E::T)x;
        }
        l[nb] += sum;
      }
#pragma unroll
      for (int d = 0; d < DP / 16; d++) {
        typedef __attribute__((address_space(3))) v4s *P;
        const uint8_t *at = lt + (g * 4 + (c >> 2)) * VROW + (d * 16 + (c & 3) * 4) * 2;
        const v4s x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)at), y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(at + 16 * VROW));
        const V v = __builtin_bit_cast(V, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
        for (int nb = 0; nb < NB; nb++) o[nb][d] = E::mul16(v, p[nb], o[nb][d]);
      }
    }
    if (__ballot(odd)) {  // as add_non_finite
      for (uint32_t k0 = begin + wave * 32; k0 < end; k0 += kKeysStep)
        for (uint32_t key = k0; key < min(k0 + 32, end); key++) {
          const uint32_t pg = min(table[key >> a.pg.shift], a.pg.n_pages - 1), slot = key & ((1u << a.pg.shift) - 1);
          const uint8_t *p = a.pg.v + (uint64_t)pg * a.pg.page + (slot * a.pg.slot + kvh * a.pg.head);
#pragma unroll
          for (int d = 0; d < DP / 16; d++) {
            if (d * 16 + g * 4 < (int)a.dim) {
              const uint2 x = *(const uint2 *)(p + (d * 16 + g * 4) * 2);
#pragma unroll
              for (int i = 0; i < 4; i++) {
                const uint16_t u = (uint16_t)((i < 2 ? x.x : x.y) >> (i % 2 * 16));
                if ((u & E::kInf) == E::kInf) {
#pragma unroll
                  for (int nb = 0; nb < NB; nb++)
                    if ((int)key >= first[nb] && (int)key <= last[nb]) o[nb][d][i] += (float)__builtin_bit_cast(typename E::T, u);
                }
              }
            }
          }
        }
    }
  }
  float *sum = (float *)smem;
#pragma unroll
  for (int nb = 0; nb < NB; nb++) {
    __syncthreads();  // the tiles, or the sums of the rows before, are free
    l[nb] = halves(rows16(l[nb], fadd2), fadd2);
    if (g == 0) ml[wave][c] = make_float2(m[nb], l[nb]);
    if (r0 + nb * 16 + c <= r1) {
#pragma unroll
      for (int d = 0; d < DP / 16; d++) *(v4f *)(sum + (wave * 16 + c) * kSum + d * 16 + g * 4) = o[nb][d];
    }
    __syncthreads();
    const uint32_t quads = a.dim / 4, rb = r0 + nb * 16, n = rb > r1 ? 0 : (min(r1, rb + 15) - rb + 1) * quads;
    for (uint32_t x = t; x < n; x += 256) {
      const uint32_t row = x / quads, d = x % quads * 4, r = rb + row;
      float mm = neg_inf(), ll = 0.f;
#pragma unroll
      for (int w = 0; w < 4; w++) mm = fmaxf(mm, ml[w][row].x);
      v4f v{0, 0, 0, 0};
#pragma unroll
      for (int w = 0; w < 4; w++) {
        const float2 y = ml[w][row];
        const float f = y.x == neg_inf() ? 1.f : ex2(y.x - mm) * down(E::kUp);
        ll += y.y * f;
        v += *(const v4f *)(sum + (w * 16 + row) * kSum + d) * f;
      }
      mm += E::kUp;
      const bool some = ll > 0.f || ll != ll;
      const uint32_t token = ch.r0 + r / a.group, head = kvh * a.group + r % a.group;
      const size_t at = (size_t)token * a.q_heads + head;
      if (a.n_splits == 1) {
        const float inv = some ? 1.f / ll : 0.f;
        typename E::T y[4];
#pragma unroll
        for (int j = 0; j < 4; j++) y[j] = (typename E::T)(v[j] * inv);
        *(uint2 *)(a.out.p + (int64_t)token * a.out.token + (int64_t)head * a.out.head + d * 2) = *(uint2 *)y;
        if (d == 0) {
          const float z = some ? mm + lg2(ll) : neg_inf();
          if (a.lse) a.lse[at] = z * kLn2;
          if (a.lse2) a.lse2[at] = z;
        }
      } else {
        *(v4f *)(a.part + (at * a.n_splits + split) * a.dim + d) = v;
        if (d == 0) a.part_ml[at * a.n_splits + split] = make_float2(some ? mm : neg_inf(), ll);
      }
    }
  }
}

// Joins the splits of one row: LQ lanes read one split's sums, 16 bytes each.
// A launch of its own (7 us at 9 to 257 splits): with the last workgroup of a row's splits
// joining them, the fences that carry sums between XCDs made a token over
// 1,000 cached ones 14 us instead of 7 + 4, a step of 64 sequences 820 instead
// of 210.
template <class E, int LQ>
__global__ __launch_bounds__(256) void k_attend_join(AttendArgs a, uint32_t tile_rows) {
  constexpr int G = 256 / LQ, CHUNK = 1024;
  __shared__ float2 ml[4];
  __shared__ float factor[CHUNK];
  __shared__ v4f acc[256];
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
  const float2 *parts = a.part_ml + row * a.n_splits;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  float m = neg_inf(), l = 0.f;
  for (uint32_t s = t; s < n; s += 256) {
    const float2 x = parts[s];
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
  const int g = t / LQ, c = t % LQ;
  for (uint32_t s0 = 0; s0 < n; s0 += CHUNK) {
    const uint32_t m1 = min(n - s0, (uint32_t)CHUNK);
    if (s0) __syncthreads();
    for (uint32_t s = t; s < m1; s += 256) {
      const float x = parts[s0 + s].x;
      factor[s] = x == neg_inf() ? 1.f : ex2(x - m);
    }
    __syncthreads();
    if (c * 4 < (int)a.dim) {
      const float *p = a.part + (row * a.n_splits + s0) * a.dim + c * 4;
#pragma unroll 4
      for (uint32_t s = g; s < m1; s += G) o += *(const v4f *)(p + (size_t)s * a.dim) * factor[s];
    }
  }
  acc[t] = o;
  __syncthreads();
  const bool some = l > 0.f || l != l;
  if (t < LQ && t * 4 < (int)a.dim) {
    for (int i = 1; i < G; i++) o += acc[i * LQ + t];
    const float inv = some ? 1.f / l : 0.f;
    typename E::T y[4];
#pragma unroll
    for (int j = 0; j < 4; j++) y[j] = (typename E::T)(o[j] * inv);
    *(uint2 *)(a.out.p + (int64_t)token * a.out.token + (int64_t)head * a.out.head + t * 8) = *(uint2 *)y;
  }
  if (t == 0) {
    const float z = some ? m + lg2(l) : neg_inf();
    if (a.lse) a.lse[row] = z * kLn2;
    if (a.lse2) a.lse2[row] = z;
  }
}

// The same for few splits and many rows: LQ lanes a row.  Seven chunks of up
// to 300 tokens, 12 heads, in up to five splits: 4.3 to 5.1 us, a workgroup a row 26.
constexpr uint32_t kShortSplits = 8;
template <class E, int LQ>
__global__ __launch_bounds__(256) void k_attend_join_short(AttendArgs a, uint32_t tile_rows) {
  const uint32_t b = blockIdx.y;
  const Chunk ch = chunk_of(a.s, b, a.err);
  const uint32_t x = blockIdx.x * (256 / LQ) + threadIdx.x / LQ, c = threadIdx.x % LQ, rows = ch.ql * a.group;
  const uint32_t kvh = x % a.kv_heads, r = x / a.kv_heads;
  if (r >= rows || c * 4 >= a.dim) return;
  const uint32_t r0 = r / tile_rows * tile_rows, r1 = min(rows, r0 + tile_rows) - 1;
  uint32_t lo, hi;
  key_range(a, ch, r0 / a.group, r1 / a.group, 32, lo, hi);
  const uint32_t n = min(max(1u, (hi - lo + a.split - 1) / a.split), kShortSplits);
  const uint32_t token = ch.r0 + r / a.group, head = kvh * a.group + r % a.group;
  const size_t row = (size_t)token * a.q_heads + head;
  float2 ml[kShortSplits];
  v4f part[kShortSplits];
  float m = neg_inf(), l = 0.f;
#pragma unroll
  for (uint32_t s = 0; s < kShortSplits; s++) {
    ml[s] = s < n ? a.part_ml[row * a.n_splits + s] : make_float2(neg_inf(), 0.f);
    part[s] = s < n ? *(const v4f *)(a.part + (row * a.n_splits + s) * a.dim + c * 4) : v4f{0, 0, 0, 0};
  }
#pragma unroll
  for (uint32_t s = 0; s < kShortSplits; s++) m = fmaxf(m, ml[s].x);
  v4f o{0, 0, 0, 0};
#pragma unroll
  for (uint32_t s = 0; s < kShortSplits; s++) {
    const float f = ml[s].x == neg_inf() ? 1.f : ex2(ml[s].x - m);
    l += ml[s].y * f;
    o += part[s] * f;
  }
  const bool some = l > 0.f || l != l;
  const float inv = some ? 1.f / l : 0.f;
  typename E::T y[4];
#pragma unroll
  for (int j = 0; j < 4; j++) y[j] = (typename E::T)(o[j] * inv);
  *(uint2 *)(a.out.p + (int64_t)token * a.out.token + (int64_t)head * a.out.head + c * 8) = *(uint2 *)y;
  if (c == 0) {
    const float z = some ? m + lg2(l) : neg_inf();
    if (a.lse) a.lse[row] = z * kLn2;
    if (a.lse2) a.lse2[row] = z;
  }
}

// Weights from stored scores: a thread sums four keys' weights over the rows.
// 50 MB of scores and weights in 12 us; computing the scores again would read
// half of the cache.
__global__ __launch_bounds__(256) void k_weights_stored(AttendArgs a) {
  __shared__ float z[kFewRows];
  const uint32_t b = blockIdx.z, kvh = blockIdx.y, key0 = blockIdx.x * 1024 + threadIdx.x;
  const Chunk ch = chunk_of(a.s, b, a.err);
  if (blockIdx.x * 1024 >= ch.kl) return;
  const uint32_t rows = ch.ql * a.group;  // one tile: at most kFewRows
  if (threadIdx.x < rows) {
    const float x = a.lse2[(size_t)(ch.r0 + threadIdx.x / a.group) * a.q_heads + kvh * a.group + threadIdx.x % a.group];
    z[threadIdx.x] = x == neg_inf() ? __builtin_inff() : x;  // a row that sees nothing gives nothing
  }
  const float *win = a.win.p + (int64_t)b * a.win.seq + (int64_t)kvh * a.win.head;
  // the rows' weights first: the running sum takes one rounding a call
  float sum[4] = {0.f, 0.f, 0.f, 0.f}, old[4];
#pragma unroll
  for (int j = 0; j < 4; j++) old[j] = key0 + j * 256 < ch.kl ? win[key0 + j * 256] : 0.f;
  __syncthreads();
  if (rows) {
    uint32_t lo, hi;
    key_range(a, ch, 0, (rows - 1) / a.group, 32, lo, hi);
    const float *sc = a.scores + ((size_t)b * a.kv_heads + kvh) * a.score_rows * a.score_keys;
#pragma unroll 4
    for (uint32_t r = 0; r < rows; r++)
#pragma unroll
      for (int j = 0; j < 4; j++) {
        const uint32_t key = key0 + j * 256;
        if (key >= lo && key < hi) {
          const float x = sc[(size_t)r * a.score_keys + key];
          sum[j] += x == neg_inf() ? 0.f : ex2(x - z[r]);  // hidden: nothing, though the row's sum be NaN
        }
      }
  }
  float *wout = a.wout.p + (int64_t)b * a.wout.seq + (int64_t)kvh * a.wout.head;
#pragma unroll
  for (int j = 0; j < 4; j++)
    if (key0 + j * 256 < ch.kl) wout[key0 + j * 256] = old[j] + sum[j];
}

// Weights from scores computed again: a wave keeps 64 keys in registers, the
// rows of the chunk pass by in tiles of 64 (32 where rows are long).  Every score costs an
// exponential, a product and a sum, about 23 cycles of a SIMD for 64 scores,
// against 16 for its matrix product: the vector unit bounds it.  2,048 tokens
// of 32 heads over 32,768: 0.60 to 0.65 ms (beside 0.65 to 0.70 in the same
// runs: 32 keys a wave 0.80, tiles of 32 rows 0.70 to 0.75).
// Where that gives too few workgroups the rows are split, and their sums are
// added by another launch.
struct AgainRows {
  uint32_t lo, hi, per, n;  // rows that see a key of the tile, rows of a split, splits that have any
};
__device__ __forceinline__ AgainRows again_rows(const AttendArgs &a, const Chunk &ch, uint32_t key0) {
  AgainRows r;
  const int klast = (int)min(key0 + kAgainKeys, ch.kl) - 1;
  const int t_lo = a.causal ? max(0, (int)key0 - ch.p0) : 0;
  const int t_hi = a.window ? min((int)ch.ql, klast + (int)a.window - ch.p0) : (int)ch.ql;
  r.lo = (uint32_t)min(t_lo, (int)ch.ql) * a.group;
  r.hi = max((uint32_t)max(t_hi, 0) * a.group, r.lo);
  const uint32_t tiles = (r.hi - r.lo + 63) / 64;
  r.per = max((tiles + a.row_splits - 1) / a.row_splits, 1u) * 64;
  r.n = (r.hi - r.lo + r.per - 1) / r.per;
  return r;
}

template <class E, int DP>
__global__ __launch_bounds__(256, DP > 128 ? 1 : 2) void k_weights_again(AttendArgs a) {
  constexpr int kStride = DP * 2 + 16, RT = DP > 128 ? 32 : 64;  // rows of a tile
  __shared__ __align__(16) uint8_t lq[2][RT * kStride];
  __shared__ float lz[2][RT];
  __shared__ float total[kAgainKeys];
  const uint32_t b = blockIdx.y, kvh = blockIdx.x % a.kv_heads, rest = blockIdx.x / a.kv_heads;
  const uint32_t part = rest % a.row_splits, kt = rest / a.row_splits;
  const Chunk ch = chunk_of(a.s, b, a.err);
  const uint32_t key0 = kt * kAgainKeys;
  if (key0 >= ch.kl) return;
  const AgainRows range = again_rows(a, ch, key0);
  const float *win = a.win.p + (int64_t)b * a.win.seq + (int64_t)kvh * a.win.head;
  float *wout = a.wout.p + (int64_t)b * a.wout.seq + (int64_t)kvh * a.wout.head;
  if (part >= range.n) {
    if (a.row_splits == 1 && key0 + threadIdx.x < ch.kl) wout[key0 + threadIdx.x] = win[key0 + threadIdx.x];
    return;
  }
  const uint32_t r_lo = range.lo + part * range.per, r_hi = min(range.hi, r_lo + range.per);
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), half = lane >> 5, col = lane & 31;
  const int wkey = (int)key0 + wave * 64;  // the wave's first key
  typename E::V k[2][DP / 16];
#pragma unroll
  for (int kb = 0; kb < 2; kb++) {
    const uint32_t key = min((uint32_t)wkey + kb * 32 + col, ch.kl - 1);
    const uint32_t page = min(a.s.table[(int64_t)b * a.s.table_stride + (key >> a.pg.shift)], a.pg.n_pages - 1);
    const uint8_t *at = a.pg.k + (uint64_t)page * a.pg.page + ((key & ((1u << a.pg.shift) - 1)) * a.pg.slot + kvh * a.pg.head);
#pragma unroll
    for (int s = 0; s < DP / 16; s++) {
      v4u x{0, 0, 0, 0};
      if ((2 * s + half) * 8 < (int)a.dim) x = *(const v4u *)(at + (2 * s + half) * 16);
      k[kb][s] = __builtin_bit_cast(typename E::V, x);
    }
  }
  v16f acc[2] = {v16f{}, v16f{}};
  constexpr int NCH = DP / 8, N = (RT * NCH + 255) / 256;
  // places of the rows that this thread loads: RT rows on is some tokens and
  // some heads on, a pointer's step and another where the heads wrap around
  const uint32_t step_t = RT / a.group, step_g = RT % a.group;
  const int64_t q_step = step_t * a.q.token + step_g * a.q.head, q_wrap = a.q.token - (int64_t)a.group * a.q.head;
  const int64_t z_step = (int64_t)step_t * a.q_heads + step_g, z_wrap = (int64_t)a.q_heads - a.group;
  const uint8_t *qp[N];
  const float *zp;
  uint32_t gr[N + 1];
#pragma unroll
  for (int i = 0; i < N; i++) {
    const uint32_t r = r_lo + (i * 256 + t) / NCH;
    gr[i] = r % a.group;
    qp[i] = a.q.p + (int64_t)(ch.r0 + r / a.group) * a.q.token + (int64_t)(kvh * a.group + gr[i]) * a.q.head + (i * 256 + t) % NCH * 16;
  }
  gr[N] = (r_lo + t % RT) % a.group;
  zp = a.lse2 + (size_t)(ch.r0 + (r_lo + t % RT) / a.group) * a.q_heads + kvh * a.group + gr[N];
  uint32_t first_tok = r_lo / a.group, first_g = r_lo % a.group;
  v4u next[N];
  float nextz = 0.f;
  auto load = [&](uint32_t r0) {
#pragma unroll
    for (int i = 0; i < N; i++) {
      const int x = i * 256 + t;
      next[i] = v4u{0, 0, 0, 0};
      if (x < RT * NCH && r0 + x / NCH < r_hi && (x % NCH) * 8 < (int)a.dim) next[i] = *(const v4u *)qp[i];
      qp[i] += q_step;
      gr[i] += step_g;
      if (gr[i] >= a.group) {
        gr[i] -= a.group;
        qp[i] += q_wrap;
      }
    }
    if (t < RT) {
      const float z = r0 + t < r_hi ? *zp : neg_inf();
      nextz = z == neg_inf() ? __builtin_inff() : z;  // a row that sees nothing gives nothing
      zp += z_step;
      gr[N] += step_g;
      if (gr[N] >= a.group) {
        gr[N] -= a.group;
        zp += z_wrap;
      }
    }
  };
  load(r_lo);
  int buf = 0;
  for (uint32_t r0 = r_lo; r0 < r_hi; r0 += RT, buf ^= 1) {
#pragma unroll
    for (int i = 0; i < N; i++) {
      const int x = i * 256 + t;
      if (x < RT * NCH) *(v4u *)(lq[buf] + (x / NCH) * kStride + (x % NCH) * 16) = next[i];
    }
    if (t < RT) lz[buf][t] = nextz;
    if (r0 + RT < r_hi) load(r0 + RT);
    lds_barrier();
    // (the last row's token is at most (RT - 1) / group + 1 on)
    const int p_lo = ch.p0 + (int)first_tok, p_hi = p_lo + (int)((RT - 1) / a.group) + 1;
    // (rows past the last are zeros, which an infinite key makes NaN of)
    const bool masked = (a.causal && wkey + 63 > p_lo) || (a.window && wkey <= p_hi - (int)a.window) || r0 + RT > r_hi;
#pragma unroll
    for (int rb = 0; rb < RT / 32; rb++) {
      v16f s[2] = {v16f{}, v16f{}};
#pragma unroll
      for (int x = 0; x < DP / 16; x++) {
        const v4u q = *(const v4u *)(lq[buf] + (rb * 32 + col) * kStride + (2 * x + half) * 16);
#pragma unroll
        for (int kb = 0; kb < 2; kb++) s[kb] = E::mul(k[kb][x], __builtin_bit_cast(typename E::V, q), s[kb]);
      }
      const float z = lz[buf][rb * 32 + col];
      if (masked) {
        int k0 = wkey;
        asm volatile("" : "+s"(k0));
        const uint32_t row = r0 + rb * 32 + col;
        const int pos = ch.p0 + (int)(min(row, r_hi - 1) / a.group);
#pragma unroll
        for (int kb = 0; kb < 2; kb++)
#pragma unroll
          for (int i = 0; i < 16; i++) {
            const int key = k0 + kb * 32 + (i / 4) * 8 + half * 4 + i % 4;
            const bool hidden = row >= r_hi || (a.causal && key > pos) || (a.window && key <= pos - (int)a.window);
            acc[kb][i] += hidden ? 0.f : ex2(__builtin_fmaf(s[kb][i], a.c, -z));
          }
      } else {
#pragma unroll
        for (int kb = 0; kb < 2; kb++)
#pragma unroll
          for (int i = 0; i < 16; i++) acc[kb][i] += ex2(__builtin_fmaf(s[kb][i], a.c, -z));
      }
    }
    first_tok += step_t;
    first_g += step_g;
    if (first_g >= a.group) {
      first_g -= a.group;
      first_tok++;
    }
  }
#pragma unroll
  for (int kb = 0; kb < 2; kb++)
#pragma unroll
    for (int i = 0; i < 16; i++) {
      float x = acc[kb][i];
#pragma unroll
      for (int j = 16; j; j >>= 1) x += __shfl_xor(x, j, 64);
      if (col == 0) total[wave * 64 + kb * 32 + (i / 4) * 8 + half * 4 + i % 4] = x;
    }
  __syncthreads();
  const uint32_t key = key0 + t;
  if (key < ch.kl) {
    if (a.row_splits == 1) wout[key] = win[key] + total[t];
    else a.row_sums[(((size_t)part * a.s.n_seq + b) * a.kv_heads + kvh) * a.score_keys + key] = total[t];
  }
}

__global__ __launch_bounds__(256) void k_weights_add(AttendArgs a) {
  const uint32_t b = blockIdx.y, kvh = blockIdx.x % a.kv_heads, key0 = blockIdx.x / a.kv_heads * kAgainKeys, key = key0 + threadIdx.x;
  const Chunk ch = chunk_of(a.s, b, a.err);
  if (key >= ch.kl) return;
  const AgainRows range = again_rows(a, ch, key0);
  const float old = a.win.p[(int64_t)b * a.win.seq + (int64_t)kvh * a.win.head + key];
  float sum = 0.f;
#pragma unroll 4
  for (uint32_t i = 0; i < range.n; i++) sum += a.row_sums[(((size_t)i * a.s.n_seq + b) * a.kv_heads + kvh) * a.score_keys + key];
  a.wout.p[(int64_t)b * a.wout.seq + (int64_t)kvh * a.wout.head + key] = old + sum;
}

template <class E, int DP>
hipError_t rows_dim(const AttendArgs &a, hipStream_t st) {
  constexpr int KT = DP > 128 ? 32 : 64;
  k_attend_rows<E, DP, KT><<<dim3(a.kv_heads * a.row_tiles * a.n_splits, a.s.n_seq), 256, 2 * tile_bytes<DP, KT>(), st>>>(a);
  return hipGetLastError();
}

template <class E, int DP>
hipError_t few_dim(const AttendArgs &a, uint32_t tile_rows, hipStream_t st) {
  const uint32_t units = (a.row_tiles * a.n_splits * a.s.n_seq + 7) / 8 * 8;
  const dim3 grid(units * a.kv_heads);
  if (tile_rows == 16) k_attend_few<E, DP, 1><<<grid, 256, 0, st>>>(a);
  else k_attend_few<E, DP, 2><<<grid, 256, 0, st>>>(a);
  return hipGetLastError();
}

template <class E>
hipError_t attend_type(uint32_t tile_rows, const AttendArgs &a, hipStream_t st) {
  if (tile_rows == kManyRows) {
    if (a.dim <= 64) return rows_dim<E, 64>(a, st);
    if (a.dim <= 96) return rows_dim<E, 96>(a, st);
    if (a.dim <= 128) return rows_dim<E, 128>(a, st);
    if (a.dim <= 192) return rows_dim<E, 192>(a, st);
    return rows_dim<E, 256>(a, st);
  }
  if (a.dim <= 64) return few_dim<E, 64>(a, tile_rows, st);
  if (a.dim <= 96) return few_dim<E, 96>(a, tile_rows, st);
  if (a.dim <= 128) return few_dim<E, 128>(a, tile_rows, st);
  if (a.dim <= 192) return few_dim<E, 192>(a, tile_rows, st);
  return few_dim<E, 256>(a, tile_rows, st);
}

template <class E>
hipError_t weights_type(const AttendArgs &a, hipStream_t st) {
  const uint32_t tiles = (a.s.max_k + kAgainKeys - 1) / kAgainKeys;
  const dim3 grid(tiles * a.row_splits * a.kv_heads, a.s.n_seq);
  if (a.dim <= 64) k_weights_again<E, 64><<<grid, 256, 0, st>>>(a);
  else if (a.dim <= 96) k_weights_again<E, 96><<<grid, 256, 0, st>>>(a);
  else if (a.dim <= 128) k_weights_again<E, 128><<<grid, 256, 0, st>>>(a);
  else if (a.dim <= 192) k_weights_again<E, 192><<<grid, 256, 0, st>>>(a);
  else k_weights_again<E, 256><<<grid, 256, 0, st>>>(a);
  if (a.row_splits > 1) k_weights_add<<<dim3(tiles * a.kv_heads, a.s.n_seq), 256, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_attend(uint32_t tile_rows, bool f16, const AttendArgs &a, hipStream_t st) {
  return f16 ? attend_type<F16>(tile_rows, a, st) : attend_type<Bf16>(tile_rows, a, st);
}

template <class E>
static hipError_t join_type(const AttendArgs &a, uint32_t tile_rows, hipStream_t st) {
  const uint32_t rows = a.s.max_q * a.q_heads;
  if (a.n_splits <= kShortSplits) {
    if (a.dim <= 64) k_attend_join_short<E, 16><<<dim3((rows + 15) / 16, a.s.n_seq), 256, 0, st>>>(a, tile_rows);
    else if (a.dim <= 128) k_attend_join_short<E, 32><<<dim3((rows + 7) / 8, a.s.n_seq), 256, 0, st>>>(a, tile_rows);
    else k_attend_join_short<E, 64><<<dim3((rows + 3) / 4, a.s.n_seq), 256, 0, st>>>(a, tile_rows);
    return hipGetLastError();
  }
  const dim3 grid(rows, a.s.n_seq);
  if (a.dim <= 64) k_attend_join<E, 16><<<grid, 256, 0, st>>>(a, tile_rows);
  else if (a.dim <= 128) k_attend_join<E, 32><<<grid, 256, 0, st>>>(a, tile_rows);
  else k_attend_join<E, 64><<<grid, 256, 0, st>>>(a, tile_rows);
  return hipGetLastError();
}
hipError_t launch_attend_join(bool f16, const AttendArgs &a, uint32_t tile_rows, hipStream_t st) {
  return f16 ? join_type<F16>(a, tile_rows, st) : join_type<Bf16>(a, tile_rows, st);
}

hipError_t launch_attend_weights(bool f16, const AttendArgs &a, hipStream_t st) {
  if (a.scores) {
    k_weights_stored<<<dim3((a.s.max_k + 1023) / 1024, a.kv_heads, a.s.n_seq), 256, 0, st>>>(a);
    return hipGetLastError();
  }
  return f16 ? weights_type<F16>(a, st) : weights_type<Bf16>(a, st);
}

}  // namespace gr
