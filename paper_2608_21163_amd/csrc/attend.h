// attend.h -- attention of chunks of new tokens over a paged cache: what the
// kernels for 16-bit pages (k_attend.hip), for 16-bit pages with first tokens
// that every row sees (k_attend_sinks.hip) and for packed pages
// (k_attend_packed.hip) are made of.
//
// One wave holds 32 query rows as the columns of its products: S^T = K Q^T
// and O^T = V^T P^T, so a row's running maximum and sum stay in the lanes
// of its column (two lanes a row), and the probabilities leave the first
// product in the layout that the second one reads them in.  The new tokens
// of a sequence and the query heads that share a key/value head are packed
// into the rows (row = token * group + head in group): keys are read once
// for all of them.
#pragma once
#include "cache.h"
#include "packed.h"
#include "wave.h"

namespace gr {
namespace {

typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef short v8s __attribute__((ext_vector_type(8)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef float v4f __attribute__((ext_vector_type(4)));

constexpr float kLn2 = 0.69314718055994531f;

// kUp, kLagUp: probabilities enter their product at 2^kUp times their size
// where the largest is 1, at 2^kLagUp times where it may reach 2^8 (tile_step).
// fp16 has steps of 2^-24 below 2^-14: the weight of tokens 2^-25 of the largest
// and less would be lost from the results, though not from the sum that divides
// them, however many they are.  Powers of two, taken back at the end.
struct Bf16 : PackBf16 {
  static constexpr int kUp = 0, kLagUp = 0;
  static constexpr uint32_t kExp = 0x7F807F80u, kExpLow = 0x00800080u, kInf = 0x7F80u;  // exponent bits of two elements, their lowest bits, of one
  typedef __bf16 T;
  typedef v8bf V;
  static __device__ __forceinline__ v16f mul(V a, V b, v16f c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
  static __device__ __forceinline__ v4f mul16(V a, V b, v4f c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
struct F16 : PackF16 {
  static constexpr int kUp = 14, kLagUp = 7;
  static constexpr uint32_t kExp = 0x7C007C00u, kExpLow = 0x04000400u, kInf = 0x7C00u;
  typedef _Float16 T;
  typedef v8h V;
  static __device__ __forceinline__ v16f mul(V a, V b, v16f c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
  static __device__ __forceinline__ v4f mul16(V a, V b, v4f c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};

// What a kernel reads: 16-bit pages; those with first tokens that every row
// sees beside its window; packed pages, with or without such tokens.
struct Whole { static constexpr bool kSinks = false, kPacked = false; };
struct Sinks { static constexpr bool kSinks = true, kPacked = false; };
struct Packed { static constexpr bool kSinks = true, kPacked = true; };

// A key before a row's window that is none of the first tokens.
template <class V> __device__ __forceinline__ bool before_window(int key, int first, int sinks) {
  return key < first && (!V::kSinks || key >= sinks);
}

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
// (values that are unpacked: 16 bytes a lane of eight rows in consecutive lanes, which start 32 bytes apart)
template <int DP> constexpr int packed_v_row() { return DP * 2 + 32; }
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
  // Of the keys before sinks and from seen to end, a page outside the pool is reported
  // of seq; what lies between them is hidden, and a window's user may have freed it.
  __device__ __forceinline__ void rows(const AttendArgs &a, uint32_t key0, uint32_t sinks, uint32_t seen, uint32_t end, uint32_t kvh, uint32_t seq) {
    const uint32_t mask = (1u << a.pg.shift) - 1, in_head = kvh * a.pg.head + (in ? piece * 16 : 0);
    bool bad = false;
    if (one_page) {
      bad = page[0] >= a.pg.n_pages && key0 + krow < end && (key0 + krow + N > seen || key0 + krow < sinks);
      const uint64_t off = (uint64_t)min(page[0], a.pg.n_pages - 1) * a.pg.page + (((key0 + krow) & mask) * a.pg.slot + in_head);
#pragma unroll
      for (int i = 0; i < N; i++) {
        k[i] = *(const v4u *)(a.pg.k + off + i * a.pg.slot);
        v[i] = *(const v4u *)(a.pg.v + off + i * a.pg.slot);
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; i++) {
        bad |= page[i] >= a.pg.n_pages && key0 + krow + i < end && (key0 + krow + i >= seen || key0 + krow + i < sinks);
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
  template <class E>
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

// The same of packed pages: a thread loads one block of a key and of its
// value, 16 bytes of codes and a scale each, and 16-bit rows enter LDS.
template <int DP, int KT>
struct PackedLoad {
  static constexpr int BLOCKS = DP / 32;
  static_assert(KT * BLOCKS <= 256, "a block a thread");
  v4u k, v;
  uint32_t ks, vs, page;
  int key, block;
  bool in;

  __device__ __forceinline__ PackedLoad(const AttendArgs &a, int t) {
    key = t / BLOCKS;
    block = t % BLOCKS;
    in = key < KT && block * 32 < (int)a.dim;
  }
  __device__ __forceinline__ void pages(const AttendArgs &a, const uint32_t *table, uint32_t key0) {
    page = table[min((key0 + key) >> a.pg.shift, a.s.max_pages - 1)];
  }
  __device__ __forceinline__ void rows(const AttendArgs &a, uint32_t key0, uint32_t sinks, uint32_t seen, uint32_t end, uint32_t kvh, uint32_t seq) {
    k = v = v4u{0, 0, 0, 0};
    ks = vs = 127;
    if (!in) return;
    if (page >= a.pg.n_pages && key0 + key < end && (key0 + key >= seen || key0 + key < sinks)) cache_err(a.err, kCachePage, seq);
    const uint64_t pg = min(page, a.pg.n_pages - 1);
    const uint32_t slot = (key0 + key) & ((1u << a.pg.shift) - 1);
    const uint64_t off = pg * a.pg.page + (slot * a.pg.slot + kvh * a.pg.head + block * 16);
    const uint64_t sc = pg * a.sc.page + (slot * a.sc.slot + kvh * a.sc.head + block);
    k = *(const v4u *)(a.pg.k + off);
    v = *(const v4u *)(a.pg.v + off);
    ks = a.sc.k[sc];
    vs = a.sc.v[sc];
  }
  // A block of NaN among the values becomes zeros.
  template <class E>
  __device__ __forceinline__ bool clear_non_finite(uint32_t key0, uint32_t end) {
    if (vs <= (uint32_t)E::kMaxScale) return false;
    v = v4u{0, 0, 0, 0};
    vs = 127;
    return key0 + key < end;
  }
  // (what codes past dim stand for meets zeros of the queries, or is not written)
  template <class E>
  __device__ __forceinline__ void store(const AttendArgs &, uint8_t *lk, uint8_t *lv) {
    if (key >= KT) return;
    const float kf = pack_factor<E>(ks), vf = pack_factor<E>(vs);
#pragma unroll
    for (int w = 0; w < 4; w++) {
      *(v4u *)(lk + key * k_row<DP>() + block * 64 + w * 16) = unpack8<E>(k[w], kf);
      *(v4u *)(lv + key * v_row<DP>() + block * 64 + w * 16) = unpack8<E>(v[w], vf);
    }
  }
};
template <class V, int DP, int KT> struct TileLoadOf { typedef TileLoad<DP, KT> T; };
template <int DP, int KT> struct TileLoadOf<Packed, DP, KT> { typedef PackedLoad<DP, KT> T; };

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

// One tile of KT keys: scores, running softmax, weighted values.
// A row sees the keys from first to last, and those before sinks up to last.
// masked: some key of the tile is hidden from some row of the wave.
template <class E, int DP, int KT, class V>
__device__ __forceinline__ void tile_step(RowState<E, DP> &st, const uint8_t *lk, const uint8_t *lv, float c, uint32_t key0,
                                          bool masked, int sinks, int first, int last, int lane) {
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
        if (before_window<V>(key, first, sinks) || key > last) s[kb][i] = neg_inf();
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

// The keys that rows [first token, last token] of a chunk see, on a line of
// places from lo to before hi, lo a multiple of 32.  Without first tokens
// (a.sinks) a place is a key.  With them the places before a.sink_keys (which is
// sinks rounded up to a tile) are the first keys, and where the window begins
// further on, a gap follows: later places are the window's keys.  So splits are
// equal shares of what is read, and no tile holds keys from both sides.
template <class V>
struct KeyLine {
  uint32_t lo, hi;
  uint32_t seen;   // no row sees the keys from a.sinks to before it
  uint32_t gap;

  __device__ __forceinline__ KeyLine(const AttendArgs &a, const Chunk &c, uint32_t t0, uint32_t t1) {
    int l = 0, h = (int)c.kl;
    if (a.causal) h = min(h, c.p0 + (int)t1 + 1);
    if (a.window) l = max(0, c.p0 + (int)t0 - (int)a.window + 1);
    seen = (uint32_t)l;
    lo = (uint32_t)l / 32 * 32;
    hi = (uint32_t)max(h, (int)lo);
    gap = 0;
    if constexpr (V::kSinks) {
      if (lo > a.sink_keys) {
        gap = lo - a.sink_keys;
        hi -= gap;
      }
      lo = 0;
    }
  }
  // the key at a place
  __device__ __forceinline__ uint32_t key(const AttendArgs &a, uint32_t at) const {
    return V::kSinks && at >= a.sink_keys ? at + gap : at;
  }
  // the key before which a tile that begins at this place ends, in a split that ends at place `end`
  __device__ __forceinline__ uint32_t end_of(const AttendArgs &a, uint32_t at, uint32_t end) const {
    if constexpr (!V::kSinks) return end;
    return gap && at < a.sink_keys ? min(end, a.sink_keys) : end + gap;
  }
};

// The first keys that every row sees.
template <class V>
__device__ __forceinline__ int sinks_of(const AttendArgs &a) { return V::kSinks ? (int)a.sinks : 0; }

// Adds the infinite and NaN values of the keys at places [begin, end) to the rows that
// see them.  Tiles with a key that is hidden from some row hold zeros in their
// place, as a hidden key's weight of zero would make NaN of them; in other
// tiles the product took them already, and what is infinite or NaN stays so.
// (There a probability that 16 bits round to 0 makes NaN of an infinite value,
// where a tile with hidden keys gives the infinity.)
template <class E, int DP, class V>
__device__ __forceinline__ void add_non_finite(const AttendArgs &a, const uint32_t *table, const KeyLine<V> &line, uint32_t kvh,
                                               uint32_t begin, uint32_t end, int first, int last, int half, v16f *o) {
  for (uint32_t at0 = begin; at0 < end; at0++) {
    const uint32_t key = line.key(a, at0);
    const uint32_t page = min(table[key >> a.pg.shift], a.pg.n_pages - 1), slot = key & ((1u << a.pg.shift) - 1);
    if constexpr (V::kPacked) {
      const uint8_t *p = a.sc.v + (uint64_t)page * a.sc.page + (slot * a.sc.slot + kvh * a.sc.head);
      if (((int)key >= first || (int)key < (int)a.sinks) && (int)key <= last) {
#pragma unroll
        for (int d = 0; d < DP / 32; d++)
          if (d * 32 < (int)a.dim && p[d] > E::kMaxScale) o[d] += __builtin_nanf("");
      }
      continue;
    }
    const uint8_t *p = a.pg.v + (uint64_t)page * a.pg.page + (slot * a.pg.slot + kvh * a.pg.head);
    const bool see = ((int)key >= first || (int)key < sinks_of<V>(a)) && (int)key <= last;
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
template <class E, int DP, int KT, class V>
__global__ __launch_bounds__(256, DP > 128 ? 1 : 2) void k_attend_rows(AttendArgs a) {
  typedef typename TileLoadOf<V, DP, KT>::T Load;
  extern __shared__ uint8_t smem[];
  const uint32_t kvh = blockIdx.x % a.kv_heads, rest = blockIdx.x / a.kv_heads;
  const uint32_t rt = rest % a.row_tiles, split = rest / a.row_tiles, b = blockIdx.y;
  const Chunk ch = chunk_of(a.s, b, a.err);
  const uint32_t rows = ch.ql * a.group, r0 = rt * kManyRows;
  if (r0 >= rows) return;
  const uint32_t r1 = min(rows, r0 + kManyRows) - 1;
  const KeyLine<V> line(a, ch, r0 / a.group, r1 / a.group);
  const bool direct = a.n_splits == 1;
  const uint32_t begin = line.lo + split * a.split, end = min(line.hi, begin + a.split);
  if (split && begin >= line.hi) return;
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
    const int all1 = a.causal ? min(ch.p0 + (int)(r0 / a.group), (int)ch.kl - 1) : (int)ch.kl - 1;
    const int sinks = sinks_of<V>(a);
    bool odd = false;
    Load ld(a, t);
    ld.pages(a, table, line.key(a, begin));
    ld.rows(a, line.key(a, begin), sinks, line.seen, line.end_of(a, begin, end), kvh, b);
    ld.pages(a, table, line.key(a, begin + KT));
    int buf = 0;
    for (uint32_t at = begin; at < end; at += KT, buf ^= 1) {
      const uint32_t key0 = line.key(a, at);
      const int tile_end = (int)line.end_of(a, at, end);
      uint8_t *lk = smem + buf * tile_bytes<DP, KT>(), *lv = lk + KT * k_row<DP>();
      if ((int)key0 < all0 || (int)key0 + KT - 1 > min(all1, tile_end - 1)) odd |= ld.template clear_non_finite<E>(key0, tile_end);
      ld.template store<E>(a, lk, lv);
      if (at + KT < end) {
        ld.rows(a, line.key(a, at + KT), sinks, line.seen, line.end_of(a, at + KT, end), kvh, b);
        ld.pages(a, table, line.key(a, at + 2 * KT));
      }
      lds_barrier();
      const bool masked = (int)key0 < wfirst || (int)key0 + KT - 1 > min(wlast, tile_end - 1);
      tile_step<E, DP, KT, V>(st, lk, lv, a.c, key0, masked, sinks, first, min(last, tile_end - 1), lane);
    }
    if (__syncthreads_or(odd)) add_non_finite<E, DP, V>(a, table, line, kvh, begin, end, first, last, half, st.o);
  }
  st.l = halves(st.l, fadd2) * down(E::kLagUp);
  st.m += E::kLagUp;
#pragma unroll
  for (int d = 0; d < DP / 32; d++) st.o[d] *= down(E::kLagUp);
  if (valid) write_row<E, DP>(a, st.o, st.m, st.l, ch.r0 + tok, head, split, direct, half);
}

// The end of a kernel whose four waves took different keys of the same 16 NB
// rows: their sums meet in LDS, and leave as results (direct) or at place
// part(row of the results, row of the chunk) among the parts.
template <int DP> constexpr int few_sum() { return DP + 4; }  // floats of a row
template <class E, int DP, int NB, class Part>
__device__ __forceinline__ void few_finish(const AttendArgs &a, const Chunk &ch, uint8_t *smem, float2 (*ml)[16], const v4f (*o)[DP / 16],
                                           const float *m, float *l, uint32_t kvh, uint32_t r0, uint32_t r1, bool direct, Part part) {
  constexpr int kSum = few_sum<DP>();
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), g = lane >> 4, c = lane & 15;
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
      if (direct) {
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
        const size_t to = part(at, r);
        *(v4f *)(a.part + to * a.dim + d) = v;
        if (d == 0) a.part_ml[to] = make_float2(some ? mm : neg_inf(), ll);
      }
    }
  }
}

// One tile's softmax step of a row of k_attend_few: lane (c, g) has 8 of row
// c's 32 scores.
template <class E, int DP>
__device__ __forceinline__ void few_softmax(const v4f *sc, float c, float &m, float &l, v4f *o, typename E::V &p) {
  float mx = fmaxf(fmaxf(fmaxf(sc[0][0], sc[0][1]), fmaxf(sc[0][2], sc[0][3])),
                   fmaxf(fmaxf(sc[1][0], sc[1][1]), fmaxf(sc[1][2], sc[1][3])));
  mx = halves(rows16(mx, fmax2), fmax2) * c - E::kUp;
  // the true maximum (unlike tile_step's): the largest probability is
  // then a power of two, which 16 bits hold, and the loads hide the rescaling
  if (__ballot(mx > m)) {
    const float mn = fmaxf(m, mx), scale = m == neg_inf() ? 0.f : ex2(m - mn);
#pragma unroll
    for (int d = 0; d < DP / 16; d++) o[d] *= scale;
    l *= scale;
    m = mn;
  }
  const float base = m == neg_inf() ? 0.f : m;
  float sum = 0.f;
#pragma unroll
  for (int j = 0; j < 8; j++) {
    const float x = ex2(__builtin_fmaf(sc[j / 4][j % 4], c, -base));
    sum += x;
    p[j] = (typename E::T)x;
  }
  l += sum;
}

// O^T += V^T P^T of a tile of 32 keys in LDS.
template <class E, int DP, int NB, int VROW>
__device__ __forceinline__ void few_values(const uint8_t *lt, int g, int c, const typename E::V *p, v4f (*o)[DP / 16]) {
  typedef typename E::V Op;
#pragma unroll
  for (int d = 0; d < DP / 16; d++) {
    typedef __attribute__((address_space(3))) v4s *P;
    const uint8_t *at = lt + (g * 4 + (c >> 2)) * VROW + (d * 16 + (c & 3) * 4) * 2;
    const v4s x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)at), y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(at + 16 * VROW));
    const Op v = __builtin_bit_cast(Op, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
    for (int nb = 0; nb < NB; nb++) o[nb][d] = E::mul16(v, p[nb], o[nb][d]);
  }
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
template <class E, int DP, int NB, class V>
__global__ __launch_bounds__(256, DP > 192 || (DP > 128 && NB > 1) ? 1 : DP > 128 || NB > 1 ? 2 : 3) void k_attend_few(AttendArgs a) {
  typedef typename E::V Op;
  constexpr int NS = DP / 32, KROW = k_row<DP>(), VROW = v_row<DP>(), ROWS = 16 * NB;
  constexpr int LPR = DP <= 64 ? 8 : DP <= 128 ? 16 : 32;  // lanes that load a row, 16 bytes each (96, 192: some idle)
  constexpr int N = LPR / 2;                               // consecutive keys of a tile that a lane loads a piece of
  constexpr int kTiles = 4 * 32 * (VROW > KROW ? VROW : KROW), kSums = 4 * 16 * few_sum<DP>() * 4;
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
  const KeyLine<V> line(a, ch, r0 / a.group, r1 / a.group);
  const uint32_t begin = line.lo + split * a.split, end = min(line.hi, begin + a.split);
  if (split && begin >= line.hi) return;
  if (line.lo || line.gap) pages(line.key(a, begin + wave * 32));

  Op q[NB][NS];
  int first[NB], last[NB];
#pragma unroll
  for (int nb = 0; nb < NB; nb++) {
    const uint32_t r = min(r0 + nb * 16 + c, r1), tok = r / a.group;
    const uint8_t *p = a.q.p + (int64_t)(ch.r0 + tok) * a.q.token + (int64_t)(kvh * a.group + r % a.group) * a.q.head;
#pragma unroll
    for (int s = 0; s < NS; s++) {
      v4u x{0, 0, 0, 0};
      if ((s * 4 + g) * 8 < (int)a.dim) x = *(const v4u *)(p + (s * 4 + g) * 16);
      q[nb][s] = __builtin_bit_cast(Op, x);
    }
    const int pos = ch.p0 + (int)tok;
    last[nb] = a.causal ? min(pos, (int)ch.kl - 1) : (int)ch.kl - 1;
    if constexpr (!V::kSinks) last[nb] = min(last[nb], (int)end - 1);
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
  const int sinks = sinks_of<V>(a);
  auto offsets = [&](uint32_t at) {
    const uint32_t key0 = line.key(a, at), tile_end = line.end_of(a, at, end);
    bool bad = false;
    const uint32_t mask = (1u << a.pg.shift) - 1, in_head = kvh * a.pg.head + (in ? piece * 16 : 0);
    if (one_page) {
      bad = page[0] >= a.pg.n_pages && key0 + krow < tile_end && (key0 + krow + N > line.seen || (int)(key0 + krow) < sinks);
      off[0] = (uint64_t)min(page[0], a.pg.n_pages - 1) * a.pg.page + (((key0 + krow) & mask) * a.pg.slot + in_head);
#pragma unroll
      for (int i = 1; i < N; i++) off[i] = off[i - 1] + a.pg.slot;
    } else {
#pragma unroll
      for (int i = 0; i < N; i++) {
        bad |= page[i] >= a.pg.n_pages && key0 + krow + i < tile_end && (key0 + krow + i >= line.seen || (int)(key0 + krow + i) < sinks);
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
  uint32_t at0 = begin + wave * 32;
  if (at0 < end) {
    offsets(at0);
    load_k();
    load_v();
    pages(line.key(a, at0 + kKeysStep));
    for (; at0 < end; at0 += kKeysStep) {
      const uint32_t key0 = line.key(a, at0);
      const int tile_end = (int)line.end_of(a, at0, end);
      const bool masked = (int)key0 < all0 || (int)key0 + 31 > min(all1, tile_end - 1), more = at0 + kKeysStep < end;
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
          for (int nb = 0; nb < NB; nb++) sc[nb][kb] = E::mul16(__builtin_bit_cast(Op, x), q[nb][s], sc[nb][kb]);
        }
      }
      if (masked) {
        uint32_t any = 0;
#pragma unroll
        for (int i = 0; i < N; i++)
#pragma unroll
          for (int j = 0; j < 4; j++) {
            const uint32_t bits = ((vx[i][j] & E::kExp) + E::kExpLow) & 0x80008000u;
            if ((int)(key0 + krow) + i < tile_end) any |= bits;
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
        offsets(at0 + kKeysStep);
        load_k();
        load_v();
        pages(line.key(a, at0 + 2 * kKeysStep));
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
              if (before_window<V>(key, first[nb], sinks) || key > (V::kSinks ? min(last[nb], tile_end - 1) : last[nb])) sc[nb][kb][i] = neg_inf();
            }
      }
      Op p[NB];
#pragma unroll
      for (int nb = 0; nb < NB; nb++) {
        if (a.scores && r0 + nb * 16 + c <= r1) {
          float *to = a.scores + (((size_t)b * a.kv_heads + kvh) * a.score_rows + r0 + nb * 16 + c) * a.score_keys + key0 + g * 4;
          *(v4f *)to = sc[nb][0] * a.c;
          *(v4f *)(to + 16) = sc[nb][1] * a.c;
        }
        few_softmax<E, DP>(sc[nb], a.c, m[nb], l[nb], o[nb], p[nb]);
      }
      few_values<E, DP, NB, VROW>(lt, g, c, p, o);
    }
    if (__ballot(odd)) {  // as add_non_finite
      for (uint32_t k0 = begin + wave * 32; k0 < end; k0 += kKeysStep)
        for (uint32_t at1 = k0; at1 < min(k0 + 32, end); at1++) {
          const uint32_t key = line.key(a, at1), pg = min(table[key >> a.pg.shift], a.pg.n_pages - 1), slot = key & ((1u << a.pg.shift) - 1);
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
                    if (((int)key >= first[nb] || (int)key < sinks) && (int)key <= last[nb]) o[nb][d][i] += (float)__builtin_bit_cast(typename E::T, u);
                }
              }
            }
          }
        }
    }
  }
  few_finish<E, DP, NB>(a, ch, smem, ml, o, m, l, kvh, r0, r1, a.n_splits == 1, [&](size_t at, uint32_t) { return at * a.n_splits + split; });
}

// Shares of the work of few rows: the keys that a sequence's rows see, in steps of
// kKeysStep, one sequence after the other, are one line of `total` steps, and
// unit u takes those from u * per on.  Lengths lie on the GPU, so every
// workgroup adds them up itself.
struct Share {
  uint32_t total, per;
  uint32_t seq, before;  // a sequence, and the steps before it
};
__device__ __forceinline__ uint32_t steps_of(const AttendArgs &a, uint32_t b) {
  const Chunk ch = chunk_of(a.s, b, a.err);
  if (!ch.ql) return 0;
  const KeyLine<Sinks> line(a, ch, 0, ch.ql - 1);
  return max((line.hi - line.lo + kKeysStep - 1) / kKeysStep, 1u);
}
// The sequence that has step find(per) of the line, or that is find(per).
template <class F>
__device__ __forceinline__ Share share_of(const AttendArgs &a, bool by_step, F find) {
  Share s{};
  const uint32_t lane = threadIdx.x & 63;
  uint32_t steps = 0, sum = 0;
  for (uint32_t b0 = 0; b0 < a.s.n_seq; b0 += 64) {
    steps = b0 + lane < a.s.n_seq ? steps_of(a, b0 + lane) : 0;
    sum += steps;
  }
#pragma unroll
  for (int j = 32; j; j >>= 1) sum += (uint32_t)__shfl_xor((int)sum, j, 64);
  s.total = (uint32_t)__builtin_amdgcn_readfirstlane((int)sum);
  s.per = (uint32_t)__builtin_amdgcn_readfirstlane((int)max((sum + a.units - 1) / a.units, 1u));
  const uint32_t want = find(s.per);
  uint32_t base = 0;
  for (uint32_t b0 = 0; b0 < a.s.n_seq; b0 += 64) {
    if (a.s.n_seq > 64) steps = b0 + lane < a.s.n_seq ? steps_of(a, b0 + lane) : 0;
    uint32_t x = steps;
#pragma unroll
    for (int j = 1; j < 64; j <<= 1) {
      const uint32_t y = (uint32_t)__shfl_up((int)x, j, 64);
      if ((int)lane >= j) x += y;
    }
    const uint64_t at = __ballot(by_step ? base + x > want && base + x - steps <= want : b0 + lane == want);
    if (at) {
      const int l = __ffsll((unsigned long long)at) - 1;
      s.seq = (uint32_t)__builtin_amdgcn_readfirstlane((int)b0 + l);
      s.before = base + (uint32_t)__builtin_amdgcn_readlane((int)(x - steps), l);
      break;
    }
    base += (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
  }
  return s;
}

// The same over packed pages.  A row's codes are a quarter of its bytes, so a
// key's 64 bytes (128 elements) go to four lanes as the product wants them: lane
// (c, g) holds block g of key c, 32 elements with one scale, which are the
// operands of four steps (queries are read in that order of elements).  No
// LDS for the keys; values pass through it as 16 bits for their transposition.
// A wave takes tiles of 32 keys; the next one (4 KB at 128 elements) is in flight
// while one is computed (with the one after it, too, 69.8 us become 78).
// WIDE: pages of 16 slots or more, and whole rows of DP elements whose scales are
// aligned.  Sixteen keys of a tile then lie in one page: a lane's part of an address
// never changes, a wave looks up the places of 64 such runs at once, and the
// scales of 64 keys are one load, a row a lane.
// A workgroup takes a split of one sequence's keys, or (a.units) a share of all
// sequences' keys, which lie behind each other.
template <class E, int DP, int NB, bool WIDE>
__global__ __launch_bounds__(256, packed_groups(DP, NB)) void k_attend_few_packed(AttendArgs a) {
  typedef typename E::V Op;
  constexpr int KT = 32, R = 2, STEP = kKeysStep;  // keys of a tile, runs of 16 of them
  constexpr int W = DP == 64 ? 2 : 4, LD = DP / 32 / W;  // words of eight codes a load, loads of a row's share
  constexpr int VROW = packed_v_row<DP>(), ROWS = 16 * NB;
  constexpr int kTiles = 4 * KT * VROW, kSums = 4 * 16 * few_sum<DP>() * 4;
  typedef uint32_t vw __attribute__((ext_vector_type(W)));
  __shared__ __align__(16) uint8_t smem[kTiles > kSums ? kTiles : kSums];
  __shared__ float2 ml[4][16];
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), g = lane >> 4, c = lane & 15;
  // (as k_attend_few's)
  const uint32_t unit = blockIdx.x / (8 * a.kv_heads) * 8 + blockIdx.x % 8, kvh = blockIdx.x / 8 % a.kv_heads;
  uint32_t b, rt = 0, split = 0, pos, left;  // the sequence, the segment's first step and the steps that are left
  if (a.units) {
    if (unit >= a.units) return;
    const Share s = share_of(a, true, [&](uint32_t per) { return unit * per; });
    if (unit * s.per >= s.total) return;
    b = s.seq;
    pos = unit * s.per - s.before;
    left = min(s.per, s.total - unit * s.per);
  } else {
    b = unit % a.s.n_seq, rt = unit / a.s.n_seq % a.row_tiles, split = unit / a.s.n_seq / a.row_tiles;
    if (split >= a.n_splits) return;
    pos = split * (a.split / STEP);
    left = a.n_splits > 1 ? a.split / STEP : ~0u;
  }
  const uint32_t mask = (1u << a.pg.shift) - 1;
  const int blocks = ((int)a.dim + 31) / 32;
  // bytes from a slot's row to the lane's blocks and their scales (past a row's
  // last block that one again: its elements meet zeros of the queries, or are
  // not written)
  uint32_t in_row[LD], in_scales[LD];
#pragma unroll
  for (int j = 0; j < LD; j++) {
    const int block = (j * 4 + g) * W / 4;
    in_row[j] = kvh * a.pg.head + (block < blocks ? (j * 4 + g) * W * 4 : (blocks - 1) * 16);
    in_scales[j] = kvh * a.sc.head + min(block, blocks - 1);
    if constexpr (WIDE) in_row[j] += c * a.pg.slot;
  }
  if constexpr (WIDE) in_scales[0] = kvh * a.sc.head + c * a.sc.slot;  // a whole row: of key, or value, `lane`
  uint8_t *lt = smem + wave * (kTiles / 4);
  const int sinks = (int)a.sinks;
  // Codes of consecutive keys side by side pass by the caches; where other heads'
  // lie between them, a line is several workgroups' (64 single tokens over up to
  // 8,192, two over 131,072 with weights: side by side 69.8 us past the caches, 74.3
  // through them, slots of all heads 87.9 and 83.0, 114 and 100.5).
  const bool stream = DP >= 128 && a.pg.slot == DP / 2;

  for (bool first_seg = true; left && b < a.s.n_seq; first_seg = false) {
    const uint32_t *table = a.s.table + (int64_t)b * a.s.table_stride;
    const Chunk ch = chunk_of(a.s, b, a.err);
    const uint32_t rows = ch.ql * a.group, r0 = rt * ROWS;
    if (r0 >= rows) {
      if (!a.units) return;
      b++;
      continue;
    }
    const uint32_t r1 = min(rows, r0 + ROWS) - 1;
    const KeyLine<Packed> line(a, ch, r0 / a.group, r1 / a.group);
    const uint32_t steps = (uint32_t)__builtin_amdgcn_readfirstlane((int)max((line.hi - line.lo + STEP - 1) / STEP, 1u));
    const uint32_t n = min(steps - min(pos, steps), left);
    if (!a.units && split && !n) return;
    const uint32_t begin = line.lo + pos * STEP, end = min(line.hi, begin + n * STEP);
    // Where runs of 16 keys lie, in bytes of codes and of scales: WIDE lane r % R of
    // tile r / R from here on; else keys c of the next tile's runs.
    constexpr int P = WIDE ? 1 : R;
    uint64_t code_at[P], scale_at[P];
    auto places = [&](uint32_t at) {
      bool bad = false;
#pragma unroll
      for (int r = 0; r < P; r++) {
        const uint32_t from = WIDE ? at + lane / R * STEP + lane % R * 16 : at, to = from + (WIDE ? 0 : r * 16 + c);
        const uint32_t key = line.key(a, from) + (to - from), run = line.end_of(a, from, end);
        const uint32_t id = table[min(key >> a.pg.shift, a.s.max_pages - 1)];
        bad |= id >= a.pg.n_pages && from < end && key < run && (key + (WIDE ? 16 : 1) > line.seen || (int)key < sinks);
        const uint64_t pg = min(id, a.pg.n_pages - 1);
        code_at[r] = pg * a.pg.page + (key & mask) * a.pg.slot;
        scale_at[r] = pg * a.sc.page + (key & mask) * a.sc.slot;
      }
      if (bad) cache_err(a.err, kCachePage, b);
    };
    uint32_t at0 = begin + wave * KT, tile = 0;
    if (at0 < end) places(at0);

    Op q[NB][DP / 32];
    int first[NB], last[NB];
#pragma unroll
    for (int nb = 0; nb < NB; nb++) {
      const uint32_t r = min(r0 + nb * 16 + c, r1), tok = r / a.group;
      const uint8_t *p = a.q.p + (int64_t)(ch.r0 + tok) * a.q.token + (int64_t)(kvh * a.group + r % a.group) * a.q.head;
#pragma unroll
      for (int s = 0; s < DP / 32; s++) {
        const int at = ((s / W * 4 + g) * W + s % W) * 8;
        v4u x{0, 0, 0, 0};
        if (at < (int)a.dim) x = *(const v4u *)(p + at * 2);
        q[nb][s] = __builtin_bit_cast(Op, x);
      }
      const int p0 = ch.p0 + (int)tok;
      last[nb] = a.causal ? min(p0, (int)ch.kl - 1) : (int)ch.kl - 1;
      first[nb] = a.window ? p0 - (int)a.window + 1 : 0;
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
    // A lane's blocks of the keys c of a tile's runs and of their values; a key
    // at or past the end reads some slot of the pool and is hidden.
    constexpr int S = WIDE ? 1 : 2 * R;  // scales: WIDE a row, else of each run's keys and values
    struct Tile {
      vw k[R][LD], v[R][LD];
      uint32_t s[S][LD];
    } next;
    auto load = [&](uint32_t i) {  // i: the tile among those whose places are known
#pragma unroll
      for (int r = 0; r < R; r++) {
        uint64_t at;
        if constexpr (WIDE) {
          const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)code_at[0], R * i + r);
          const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(code_at[0] >> 32), R * i + r);
          at = (uint64_t)hi << 32 | lo;
        } else {
          at = code_at[r];
        }
#pragma unroll
        for (int j = 0; j < LD; j++) {
          const vw *k = (const vw *)(a.pg.k + at + in_row[j]), *v = (const vw *)(a.pg.v + at + in_row[j]);
          if (stream) {
            next.k[r][j] = __builtin_nontemporal_load(k);
            next.v[r][j] = __builtin_nontemporal_load(v);
          } else {
            next.k[r][j] = *k;
            next.v[r][j] = *v;
          }
          if constexpr (!WIDE) {
            next.s[r][j] = a.sc.k[scale_at[r] + in_scales[j]];
            next.s[R + r][j] = a.sc.v[scale_at[r] + in_scales[j]];
          }
        }
      }
      if constexpr (WIDE) {
        // the lower lanes keys, the upper ones values
        const int from = (R * (int)i + g % R) * 4;
        const uint32_t lo = (uint32_t)__builtin_amdgcn_ds_bpermute(from, (int)(uint32_t)scale_at[0]);
        const uint32_t hi = (uint32_t)__builtin_amdgcn_ds_bpermute(from, (int)(uint32_t)(scale_at[0] >> 32));
        const uint8_t *p = (g >= R ? a.sc.v : a.sc.k) + (((uint64_t)hi << 32 | lo) + in_scales[0]);
        if constexpr (DP == 64) {
          next.s[0][0] = *(const uint16_t *)p;
        } else {
#pragma unroll
          for (int j = 0; j < LD; j++) next.s[0][j] = *(const uint32_t *)(p + j * 4);
        }
      }
    };
    bool odd = false;
    if (at0 < end) {
      load(0);
      if constexpr (!WIDE) places(at0 + STEP);
      for (; at0 < end; at0 += STEP) {
        const uint32_t key0 = line.key(a, at0);
        const int tile_end = (int)line.end_of(a, at0, end);
        const bool masked = (int)key0 < all0 || (int)key0 + KT - 1 > min(all1, tile_end - 1);
        Tile x = next;
        if (at0 + STEP < end) {
          if constexpr (WIDE) {
            tile = (tile + 1) % (64 / R);
            if (tile == 0) places(at0 + STEP);
          }
          load(tile);
          if constexpr (!WIDE) places(at0 + 2 * STEP);
        }
        // the scales of the lane's blocks of the runs' keys, and values
        uint32_t scale[2 * R][LD];
#pragma unroll
        for (int y = 0; y < 2 * R; y++)
#pragma unroll
          for (int j = 0; j < LD; j++)
            scale[y][j] = WIDE ? (uint32_t)__builtin_amdgcn_ds_bpermute((y * 16 + c) * 4, (int)x.s[0][j]) : x.s[y][j];
        if constexpr (WIDE) {
          // all on their way before the first is waited for
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int y = 0; y < 2 * R; y++)
#pragma unroll
            for (int j = 0; j < LD; j++) scale[y][j] = scale[y][j] >> (DP == 64 ? g / 2 * 8 : g * 8) & 255;
        }
        if (masked) {
#pragma unroll
          for (int r = 0; r < R; r++)
#pragma unroll
            for (int j = 0; j < LD; j++)
              if (scale[R + r][j] > (uint32_t)E::kMaxScale) {  // a block of NaN becomes zeros
                odd |= (int)key0 + r * 16 + c < tile_end;
                x.v[r][j] = vw(0);
                scale[R + r][j] = 127;
              }
        }
        v4f sc[NB][R];
#pragma unroll
        for (int r = 0; r < R; r++) {
#pragma unroll
          for (int nb = 0; nb < NB; nb++) sc[nb][r] = v4f{0, 0, 0, 0};
#pragma unroll
          for (int j = 0; j < LD; j++) {
            const float f = pack_factor<E>(scale[r][j]);
#pragma unroll
            for (int w = 0; w < W; w++) {
              const Op k = __builtin_bit_cast(Op, unpack8<E>(x.k[r][j][w], f));
#pragma unroll
              for (int nb = 0; nb < NB; nb++) sc[nb][r] = E::mul16(k, q[nb][j * W + w], sc[nb][r]);
            }
          }
        }
        lds_wave_fence();
#pragma unroll
        for (int r = 0; r < R; r++)
#pragma unroll
          for (int j = 0; j < LD; j++) {
            const float f = pack_factor<E>(scale[R + r][j]);
#pragma unroll
            for (int w = 0; w < W; w++) *(v4u *)(lt + (r * 16 + c) * VROW + ((j * 4 + g) * W + w) * 16) = unpack8<E>(x.v[r][j][w], f);
          }
        lds_wave_fence();
        if (masked) {
          uint32_t k0 = key0;
          asm volatile("" : "+s"(k0));
#pragma unroll
          for (int nb = 0; nb < NB; nb++)
#pragma unroll
            for (int r = 0; r < R; r++)
#pragma unroll
              for (int i = 0; i < 4; i++) {
                const int key = (int)k0 + r * 16 + g * 4 + i;
                if ((key < first[nb] && key >= sinks) || key > min(last[nb], tile_end - 1)) sc[nb][r][i] = neg_inf();
              }
        }
        Op p[NB];
#pragma unroll
        for (int nb = 0; nb < NB; nb++) {
          if (a.scores && r0 + nb * 16 + c <= r1) {
            float *to = a.scores + (((size_t)b * a.kv_heads + kvh) * a.score_rows + r0 + nb * 16 + c) * a.score_keys + key0 + g * 4;
            *(v4f *)to = sc[nb][0] * a.c;
            *(v4f *)(to + 16) = sc[nb][1] * a.c;
          }
          few_softmax<E, DP>(sc[nb], a.c, m[nb], l[nb], o[nb], p[nb]);
        }
        few_values<E, DP, NB, VROW>(lt, g, c, p, o);
      }
      if (__ballot(odd)) {  // as add_non_finite
        for (uint32_t k0 = begin + wave * KT; k0 < end; k0 += STEP)
          for (uint32_t at1 = k0; at1 < min(k0 + KT, end); at1++) {
            const uint32_t key = line.key(a, at1), pg = min(table[key >> a.pg.shift], a.pg.n_pages - 1), slot = key & mask;
            const uint8_t *p = a.sc.v + (uint64_t)pg * a.sc.page + (slot * a.sc.slot + kvh * a.sc.head);
#pragma unroll
            for (int d = 0; d < DP / 16; d++)
              if (d * 16 < (int)a.dim && p[d / 2] > E::kMaxScale) {
#pragma unroll
                for (int nb = 0; nb < NB; nb++)
                  if (((int)key >= first[nb] || (int)key < sinks) && (int)key <= last[nb]) o[nb][d] += __builtin_nanf("");
              }
          }
      }
    }
    if (a.units) {
      // a unit's parts: the one that it begins with, and the one that it ends with
      const size_t to = (((size_t)unit * 2 + (first_seg ? 0 : 1)) * a.kv_heads + kvh) * ROWS;
      few_finish<E, DP, NB>(a, ch, smem, ml, o, m, l, kvh, r0, r1, n == steps, [&](size_t, uint32_t r) { return to + r; });
    } else {
      few_finish<E, DP, NB>(a, ch, smem, ml, o, m, l, kvh, r0, r1, a.n_splits == 1, [&](size_t at, uint32_t) { return at * a.n_splits + split; });
      return;
    }
    left -= n;
    pos = 0;
    b++;
    __syncthreads();  // the waves' sums have been read
  }
}

// Weights from scores computed again: a wave keeps 64 keys in registers, the
// rows of the chunk pass by in tiles of 64 (32 where rows are long).  Every score costs an
// exponential, a product and a sum, about 23 cycles of a SIMD for 64 scores,
// against 16 for its matrix product: the vector unit bounds it.  2,048 tokens
// of 32 heads over 32,768: 0.60 to 0.65 ms (beside 0.65 to 0.70 in the same
// runs: 32 keys a wave 0.80, tiles of 32 rows 0.70 to 0.75).
// Where that gives too few workgroups the rows are split, and their sums are
// added by another launch (which a window needs too, for the tiles without rows).
struct AgainRows {
  uint32_t lo, hi, per, n;  // rows that see a key of the tile, rows of a split, splits that have any
};
template <class V>
__device__ __forceinline__ AgainRows again_rows(const AttendArgs &a, const Chunk &ch, uint32_t key0) {
  AgainRows r;
  const int klast = (int)min(key0 + kAgainKeys, ch.kl) - 1;
  const int t_lo = a.causal ? max(0, (int)key0 - ch.p0) : 0;
  const int t_hi = a.window && (int)key0 >= sinks_of<V>(a) ? min((int)ch.ql, klast + (int)a.window - ch.p0) : (int)ch.ql;
  r.lo = (uint32_t)min(t_lo, (int)ch.ql) * a.group;
  r.hi = max((uint32_t)max(t_hi, 0) * a.group, r.lo);
  const uint32_t tiles = (r.hi - r.lo + 63) / 64;
  r.per = max((tiles + a.row_splits - 1) / a.row_splits, 1u) * 64;
  r.n = (r.hi - r.lo + r.per - 1) / r.per;
  return r;
}

// The keys of workgroup i's tile.  With a window only the tiles that it reaches
// from some row, and those of the first tokens, have workgroups (again_tiles):
// seven chunks of up to 300 tokens, 12 heads of 64 elements, windows of 1,000 over up to
// 5,000, 1,300 workgroups instead of 3,400, 40 us -> 38.
template <class V>
__device__ __forceinline__ uint32_t again_key(const AttendArgs &a, const Chunk &ch, uint32_t i) {
  if (!a.window) return i * kAgainKeys;
  const uint32_t front = ((uint32_t)sinks_of<V>(a) + kAgainKeys - 1) / kAgainKeys, base = (uint32_t)max(0, ch.p0 - (int)a.window + 1) / kAgainKeys;
  return (i < front || base <= front ? i : base + i - front) * kAgainKeys;
}
// The other way round, for a tile that some row sees.
template <class V>
__device__ __forceinline__ uint32_t again_tile(const AttendArgs &a, const Chunk &ch, uint32_t key0) {
  const uint32_t i = key0 / kAgainKeys;
  if (!a.window) return i;
  const uint32_t front = ((uint32_t)sinks_of<V>(a) + kAgainKeys - 1) / kAgainKeys, base = (uint32_t)max(0, ch.p0 - (int)a.window + 1) / kAgainKeys;
  return i < front || base <= front ? i : i - base + front;
}

template <class E, int DP, class V>
__global__ __launch_bounds__(256, DP > 128 ? 1 : DP > 64 ? 2 : 3) void k_weights_again(AttendArgs a) {
  constexpr int kStride = DP * 2 + 16, RT = DP > 128 ? 32 : 64;  // rows of a tile
  __shared__ __align__(16) uint8_t lq[2][RT * kStride];
  __shared__ float lz[2][RT];
  __shared__ float total[kAgainKeys];
  const uint32_t b = blockIdx.y, kvh = blockIdx.x % a.kv_heads, rest = blockIdx.x / a.kv_heads;
  const uint32_t part = rest % a.row_splits;
  const Chunk ch = chunk_of(a.s, b, a.err);
  const uint32_t key0 = again_key<V>(a, ch, rest / a.row_splits);
  if (key0 >= ch.kl) return;
  const AgainRows range = again_rows<V>(a, ch, key0);
  const float *win = a.win.p + (int64_t)b * a.win.seq + (int64_t)kvh * a.win.head;
  float *wout = a.wout.p + (int64_t)b * a.wout.seq + (int64_t)kvh * a.wout.head;
  if (part >= range.n) {
    if (!a.row_sums && key0 + threadIdx.x < ch.kl) wout[key0 + threadIdx.x] = win[key0 + threadIdx.x];
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
    if constexpr (V::kPacked) {
      const uint8_t *sc = a.sc.k + (uint64_t)page * a.sc.page + ((key & ((1u << a.pg.shift) - 1)) * a.sc.slot + kvh * a.sc.head);
#pragma unroll
      for (int j = 0; j < DP / 32; j++) {
        v4u x{0, 0, 0, 0};
        uint32_t f = 127;
        if (j * 32 < (int)a.dim) {
          x = *(const v4u *)(at + j * 16);
          f = sc[j];
        }
        k[kb][2 * j] = __builtin_bit_cast(typename E::V, unpack8<E>(half ? x[1] : x[0], pack_factor<E>(f)));
        k[kb][2 * j + 1] = __builtin_bit_cast(typename E::V, unpack8<E>(half ? x[3] : x[2], pack_factor<E>(f)));
      }
    } else {
#pragma unroll
      for (int s = 0; s < DP / 16; s++) {
        v4u x{0, 0, 0, 0};
        if ((2 * s + half) * 8 < (int)a.dim) x = *(const v4u *)(at + (2 * s + half) * 16);
        k[kb][s] = __builtin_bit_cast(typename E::V, x);
      }
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
    // (no row sees a key of the wave: most of a tile of first tokens)
    const bool none = V::kSinks && ((a.causal && wkey > p_hi) || (a.window && wkey + 63 <= p_lo - (int)a.window && wkey >= sinks_of<V>(a)));
#pragma unroll
    for (int rb = 0; rb < RT / 32 && !none; rb++) {
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
            const bool hidden = row >= r_hi || (a.causal && key > pos) || (a.window && before_window<V>(key, pos - (int)a.window + 1, sinks_of<V>(a)));
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
  // Sums over the 32 columns of 32 values, each half of the wave its own: at every
  // step a lane hands on the half of its values that it does not keep, and ends
  // with the sum of value `col` (all sums by themselves: 160 trips through LDS, 9 us).
  float y[16];
#pragma unroll
  for (int i = 0; i < 16; i++) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(acc[0][i]), __float_as_uint(acc[1][i]), false, false);
    y[i] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
#pragma unroll
  for (int j = 8; j; j >>= 1)
#pragma unroll
    for (int i = 0; i < j; i++) {
      const bool upper = lane & j;
      const float keep = upper ? y[i + j] : y[i], give = upper ? y[i] : y[i + j];
      y[i] = keep + xshfl(give, j);
    }
  total[wave * 64 + col / 16 * 32 + (col % 16 / 4) * 8 + half * 4 + col % 4] = y[0];
  __syncthreads();
  const uint32_t key = key0 + t;
  if (key < ch.kl) {
    if (!a.row_sums) wout[key] = win[key] + total[t];
    else a.row_sums[(((size_t)part * a.s.n_seq + b) * a.kv_heads + kvh) * a.sum_keys + rest / a.row_splits * kAgainKeys + t] = total[t];
  }
}

template <class E, int DP, class V>
hipError_t rows_dim(const AttendArgs &a, hipStream_t st) {
  constexpr int KT = rows_tile(DP);
  k_attend_rows<E, DP, KT, V><<<dim3(a.kv_heads * a.row_tiles * a.n_splits, a.s.n_seq), 256, 2 * tile_bytes<DP, KT>(), st>>>(a);
  return hipGetLastError();
}

template <class E, int DP, class V>
hipError_t few_dim(const AttendArgs &a, uint32_t tile_rows, hipStream_t st) {
  const uint32_t units = ((a.units ? a.units : a.row_tiles * a.n_splits * a.s.n_seq) + 7) / 8 * 8;
  const dim3 grid(units * a.kv_heads);
  if constexpr (V::kPacked) {
    const bool wide = packed_wide(a);
    if (tile_rows == 16 && wide) k_attend_few_packed<E, DP, 1, true><<<grid, 256, 0, st>>>(a);
    else if (tile_rows == 16) k_attend_few_packed<E, DP, 1, false><<<grid, 256, 0, st>>>(a);
    else if (wide) k_attend_few_packed<E, DP, 2, true><<<grid, 256, 0, st>>>(a);
    else k_attend_few_packed<E, DP, 2, false><<<grid, 256, 0, st>>>(a);
  } else {
    if (tile_rows == 16) k_attend_few<E, DP, 1, V><<<grid, 256, 0, st>>>(a);
    else k_attend_few<E, DP, 2, V><<<grid, 256, 0, st>>>(a);
  }
  return hipGetLastError();
}

template <class E, class V>
hipError_t attend_type(uint32_t tile_rows, const AttendArgs &a, hipStream_t st) {
  if (tile_rows == kManyRows) {
    if (a.dim <= 64) return rows_dim<E, 64, V>(a, st);
    if (a.dim <= 96) return rows_dim<E, 96, V>(a, st);
    if (a.dim <= 128) return rows_dim<E, 128, V>(a, st);
    if (a.dim <= 192) return rows_dim<E, 192, V>(a, st);
    return rows_dim<E, 256, V>(a, st);
  }
  if (a.dim <= 64) return few_dim<E, 64, V>(a, tile_rows, st);
  // (four lanes share a packed row: its kernel has no rows of 96 and 192)
  if (!V::kPacked && a.dim <= 96) return few_dim<E, V::kPacked ? 128 : 96, V>(a, tile_rows, st);
  if (a.dim <= 128) return few_dim<E, 128, V>(a, tile_rows, st);
  if (!V::kPacked && a.dim <= 192) return few_dim<E, V::kPacked ? 256 : 192, V>(a, tile_rows, st);
  return few_dim<E, 256, V>(a, tile_rows, st);
}

template <class E, class V>
hipError_t weights_type(const AttendArgs &a, hipStream_t st) {
  const dim3 grid(again_tiles(a) * a.row_splits * a.kv_heads, a.s.n_seq);
  if (a.dim <= 64) k_weights_again<E, 64, V><<<grid, 256, 0, st>>>(a);
  else if (a.dim <= 96) k_weights_again<E, 96, V><<<grid, 256, 0, st>>>(a);
  else if (a.dim <= 128) k_weights_again<E, 128, V><<<grid, 256, 0, st>>>(a);
  else if (a.dim <= 192) k_weights_again<E, 192, V><<<grid, 256, 0, st>>>(a);
  else k_weights_again<E, 256, V><<<grid, 256, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace
}  // namespace gr
