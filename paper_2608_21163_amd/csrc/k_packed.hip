// k_packed.hip -- packed pages beside the attention of chunks: the write of new
// tokens, attention over retrieved ids, and rows read back.
#include "cache.h"
#include "packed.h"
#include "wave.h"

namespace gr {
namespace {

typedef float v2f __attribute__((ext_vector_type(2)));
constexpr float kLn2 = 0.69314718055994531f;

__device__ __forceinline__ float neg_inf() { return -__builtin_inff(); }
__device__ __forceinline__ float ex2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float lg2(float x) { return __builtin_amdgcn_logf(x); }

struct Bf16 : PackBf16 {
  typedef __bf16 T;
  // the fp32 bits of the magnitude with these 15 bits
  static __device__ __forceinline__ uint32_t magnitude(uint32_t u) { return u << 16; }
  // two products and a sum, in 32 bits
  static __device__ __forceinline__ float dot2(uint32_t a, uint32_t b, float c) {
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(v2bf, a), __builtin_bit_cast(v2bf, b), c, false);
  }
};
struct F16 : PackF16 {
  typedef _Float16 T;
  static __device__ __forceinline__ uint32_t magnitude(uint32_t u) {
    return __float_as_uint((float)__builtin_bit_cast(_Float16, (uint16_t)u));
  }
  static __device__ __forceinline__ float dot2(uint32_t a, uint32_t b, float c) {
    return __builtin_amdgcn_fdot2(__builtin_bit_cast(v2h, a), __builtin_bit_cast(v2h, b), c, false);
  }
};
// 32 codes as fp32 values, small ones that the 16-bit type would round among them.
template <class E> __device__ __forceinline__ void unpack32(v4u x, float factor, float *f) {
#pragma unroll
  for (int w = 0; w < 4; w++) {
    const v2f a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(x[w], factor, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(x[w], factor, 1);
    const v2f c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(x[w], factor, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(x[w], factor, 3);
    f[8 * w] = a[0], f[8 * w + 1] = a[1], f[8 * w + 2] = b[0], f[8 * w + 3] = b[1];
    f[8 * w + 4] = c[0], f[8 * w + 5] = c[1], f[8 * w + 6] = d[0], f[8 * w + 7] = d[1];
  }
}

// One row's eight elements of a lane, four lanes a block: their codes and the
// block's scale.  The scale is the smallest power of two 2^e with every element
// below 7 * 2^e = 1.75 * 2^(e + 2): a quarter added to the mantissa of the largest
// magnitude carries into its exponent from 1.75 on.
template <class E>
__device__ __forceinline__ void pack_block(v4u x, uint32_t &codes, uint32_t &scale) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 4; i++) top = max(top, max(x[i] & 0x7FFFu, (x[i] >> 16) & 0x7FFFu));
  top = max(top, xshfl(top, 1));
  top = max(top, xshfl(top, 2));
  const uint32_t bits = E::magnitude(top);
  scale = (uint32_t)min(max((int)((bits + 0x200000u) >> 23) - 2, E::kMinScale), E::kMaxScale);
  const float f = __uint_as_float(scale << 23);
  codes = E::template code<0>(0u, x[0], f);
  codes = E::template code<1>(codes, x[1], f);
  codes = E::template code<2>(codes, x[2], f);
  codes = E::template code<3>(codes, x[3], f);
  if (bits >= 0x7F800000u) codes = 0, scale = 255;
}

// Four lanes a block of a new token's keys and of its values.
template <class E>
__global__ __launch_bounds__(256) void k_append_packed(AppendArgs a) {
  const uint32_t b = blockIdx.y, lanes = (a.dim + 31) / 32 * 4;
  const Chunk ch = chunk_of(a.s, b, a.err);
  const uint32_t x = blockIdx.x * 256 + threadIdx.x;
  const uint32_t c = x % lanes, head = x / lanes % a.kv_heads, i = x / lanes / a.kv_heads;
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
  v4u k{0, 0, 0, 0}, v{0, 0, 0, 0};
  if (c * 8 < a.dim) {
    const int64_t tok = ch.r0 + i;
    k = *(const v4u *)(a.k.p + tok * a.k.token + (int64_t)head * a.k.head + c * 16);
    v = *(const v4u *)(a.v.p + tok * a.v.token + (int64_t)head * a.v.head + c * 16);
  }
  uint32_t kc, ks, vc, vs;
  pack_block<E>(k, kc, ks);
  pack_block<E>(v, vc, vs);
  const uint32_t slot = (uint32_t)(pos & ((1u << a.pg.shift) - 1));
  const uint64_t to = (uint64_t)page * a.pg.page + (slot * a.pg.slot + head * a.pg.head + c * 4);
  *(uint32_t *)(const_cast<uint8_t *>(a.pg.k) + to) = kc;
  *(uint32_t *)(const_cast<uint8_t *>(a.pg.v) + to) = vc;
  if (c % 4 == 0) {
    const uint64_t sc = (uint64_t)page * a.sc.page + (slot * a.sc.slot + head * a.sc.head + c / 4);
    const_cast<uint8_t *>(a.sc.k)[sc] = (uint8_t)ks;
    const_cast<uint8_t *>(a.sc.v)[sc] = (uint8_t)vs;
  }
}

// A thread per eight elements of a listed slot's keys and values.
template <class E>
__global__ __launch_bounds__(256) void k_read(ReadArgs a) {
  const uint32_t nch = a.dim / 8;
  const uint64_t x = (uint64_t)blockIdx.x * 256 + threadIdx.x;
  const uint32_t c = x % nch, head = x / nch % a.kv_heads;
  const uint64_t i = x / nch / a.kv_heads;
  if (i >= a.n) return;
  const uint32_t id = a.slots[i];
  const bool there = id != kInvalid && id < (uint64_t)a.pg.n_pages << a.pg.shift;
  if (!there && id != kInvalid) cache_err(a.err, kCacheList, (uint32_t)i);
  const uint64_t page = there ? id >> a.pg.shift : 0;
  const uint32_t slot = id & ((1u << a.pg.shift) - 1);
  const uint64_t at = page * a.pg.page + (slot * a.pg.slot + head * a.pg.head + c * 4);
  const uint64_t sc = page * a.sc.page + (slot * a.sc.slot + head * a.sc.head + c / 4);
  v4u k{0, 0, 0, 0}, v{0, 0, 0, 0};
  if (there) {
    if (a.k.p) k = unpack8<E>(*(const uint32_t *)(a.pg.k + at), pack_factor<E>(a.sc.k[sc]));
    if (a.v.p) v = unpack8<E>(*(const uint32_t *)(a.pg.v + at), pack_factor<E>(a.sc.v[sc]));
  }
  v4u *to_k = (v4u *)(a.k.p + (int64_t)i * a.k.token + (int64_t)head * a.k.head + c * 16);
  v4u *to_v = (v4u *)(a.v.p + (int64_t)i * a.v.token + (int64_t)head * a.v.head + c * 16);
  // more than the caches could keep for who takes them: past them (67 MB of keys and as much of values,
  // written by an append and read back, 58 us, through them 68; 17 MB 22 both ways)
  if ((uint64_t)a.n * a.kv_heads * a.dim >= 1 << 24) {
    if (a.k.p) __builtin_nontemporal_store(k, to_k);
    if (a.v.p) __builtin_nontemporal_store(v, to_v);
  } else {
    if (a.k.p) *to_k = k;
    if (a.v.p) *to_v = v;
  }
}

// (m, l) of two parts of a softmax, in log2 units; m may be -inf (nothing).
__device__ __forceinline__ float part_scale(float m, float top) { return m == neg_inf() ? 1.f : ex2(m - top); }

// Attention over listed slots, as for 16-bit pages, here a lane per block of a row, so
// that DP / 32 lanes read one.  WAVES share a (sequence, query head)'s list: four, or
// one where there are many lists that would not fill a workgroup's first loads, or whose
// pool the caches hold: the start and the end of a list then count for more than its
// rows.  256 x 32 lists, one wave and four: of 64 ids 45 us, 82; of 256 in a pool
// of 16,384 slots of eight heads (18 MB) 58, 88; of 65,536 106, 113; of 131,072 129, 129; of 262,144 159, 150.
// Rows in a pool above the caches are bound by their number: 155, 150 and
// 159 us at 64, 128 and 256 elements, 57 lines a ns (keys and values are two
// places each, codes and scales), and as long with rows asked for ahead of the sums.
template <class E, int DP, int WAVES>
__global__ __launch_bounds__(256) void k_ids_packed(IdsArgs a) {
  constexpr int LPR = DP / 32, GROUPS = 64 / LPR, U = 4, STEP = WAVES * GROUPS;
  __shared__ float2 sml[4];
  __shared__ float sacc[4][DP];
  const int t = threadIdx.x, lane = t & 63, wave = t / 64 % WAVES, g = lane / LPR, c = lane % LPR;
  const uint32_t list = blockIdx.x * (4 / WAVES) + __builtin_amdgcn_readfirstlane(t / 64 / WAVES);
  if (list >= a.n_seq * a.q_heads) return;
  const uint32_t b = list / a.q_heads, head = list % a.q_heads, kvh = head / a.group;
  const bool in = c * 32 < (int)a.dim;
  v4u q[4];
#pragma unroll
  for (int w = 0; w < 4; w++) {
    q[w] = v4u{0, 0, 0, 0};
    if (c * 32 + w * 8 < (int)a.dim) q[w] = *(const v4u *)(a.q.p + (int64_t)b * a.q.token + (int64_t)head * a.q.head + c * 64 + w * 16);
  }
  const uint32_t *ids = a.ids + (int64_t)b * a.ids_seq + (int64_t)head * a.ids_head;
  const uint64_t slots = (uint64_t)a.pg.n_pages << a.pg.shift;
  const uint32_t mask = (1u << a.pg.shift) - 1;
  float m = neg_inf(), l = 0.f, acc[32];
#pragma unroll
  for (int i = 0; i < 32; i++) acc[i] = 0.f;
  const uint32_t j0 = wave * GROUPS + g;
  uint32_t next[U];
#pragma unroll
  for (int u = 0; u < U; u++) next[u] = j0 + u * STEP < a.k ? ids[j0 + u * STEP] : kInvalid;
  for (uint32_t j1 = 0; j1 < a.k; j1 += STEP * U) {
    uint32_t id[U], ks[U], vs[U];
    v4u kx[U], vx[U];
#pragma unroll
    for (int u = 0; u < U; u++) {
      id[u] = next[u];
      if (id[u] != kInvalid && id[u] >= slots) {
        cache_err(a.err, kCacheId, b);
        id[u] = kInvalid;
      }
    }
#pragma unroll
    for (int u = 0; u < U; u++) {
      kx[u] = vx[u] = v4u{0, 0, 0, 0};
      ks[u] = vs[u] = 127;
      if (id[u] != kInvalid && in) {
        const uint64_t page = id[u] >> a.pg.shift;
        const uint64_t off = page * a.pg.page + ((id[u] & mask) * a.pg.slot + kvh * a.pg.head + c * 16);
        const uint64_t sc = page * a.sc.page + ((id[u] & mask) * a.sc.slot + kvh * a.sc.head + c);
        kx[u] = *(const v4u *)(a.pg.k + off);
        vx[u] = *(const v4u *)(a.pg.v + off);
        ks[u] = a.sc.k[sc];
        vs[u] = a.sc.v[sc];
      }
    }
#pragma unroll
    for (int u = 0; u < U; u++) next[u] = j1 + j0 + (U + u) * STEP < a.k ? ids[j1 + j0 + (U + u) * STEP] : kInvalid;
    float s[U], top = m;
#pragma unroll
    for (int u = 0; u < U; u++) {
      float x = 0.f, y = 0.f;
      const float f = pack_factor<E>(ks[u]);
#pragma unroll
      for (int w = 0; w < 4; w++) {
        const v4u k = unpack8<E>(kx[u][w], f);
        x = E::dot2(k[0], q[w][0], x);
        y = E::dot2(k[1], q[w][1], y);
        x = E::dot2(k[2], q[w][2], x);
        y = E::dot2(k[3], q[w][3], y);
      }
      x += y;
#pragma unroll
      for (int j = LPR / 2; j; j >>= 1) x += xshfl(x, j);
      s[u] = id[u] == kInvalid ? neg_inf() : x * a.c;
      top = fmaxf(top, s[u]);
    }
    const float base = top == neg_inf() ? 0.f : top, scale = m == neg_inf() ? 1.f : ex2(m - base);
    m = top;
    l *= scale;
#pragma unroll
    for (int i = 0; i < 32; i++) acc[i] *= scale;
#pragma unroll
    for (int u = 0; u < U; u++) {
      const float p = id[u] == kInvalid ? 0.f : ex2(s[u] - base);
      float f[32];
      unpack32<E>(vx[u], pack_factor<E>(vs[u]), f);
      l += p;
#pragma unroll
      for (int i = 0; i < 32; i++) acc[i] = __builtin_fmaf(p, f[i], acc[i]);
    }
  }
  // lane groups of the wave, then the waves
  float top = m;
#pragma unroll
  for (int j = LPR; j < 64; j <<= 1) top = fmaxf(top, xshfl(top, j));
  const float f = part_scale(m, top);
  l *= f;
#pragma unroll
  for (int i = 0; i < 32; i++) acc[i] *= f;
#pragma unroll
  for (int j = LPR; j < 64; j <<= 1) l += xshfl(l, j);
  // at every step a lane hands on the half of its values that it does not keep,
  // and ends with the wave's sums of 32 / GROUPS elements of its block
#pragma unroll
  for (int i = 0; i < 16; i++) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(acc[i]), __float_as_uint(acc[i + 16]), false, false);
    acc[i] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
#pragma unroll
  for (int i = 0; i < 8; i++) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(acc[i]), __float_as_uint(acc[i + 8]), false, false);
    acc[i] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  int first = lane / 32 * 16 + lane / 16 % 2 * 8;
#pragma unroll
  for (int j = 8, n = 4; j >= LPR; j >>= 1, n >>= 1) {
    const bool upper = lane & j;
    if (upper) first += n;
#pragma unroll
    for (int i = 0; i < n; i++) {
      const float keep = upper ? acc[i + n] : acc[i], give = upper ? acc[i] : acc[i + n];
      acc[i] = keep + xshfl(give, j);
    }
  }
  const size_t row = (size_t)b * a.q_heads + head;
  const uint8_t *prior = a.prior.p + (int64_t)b * a.prior.token + (int64_t)head * a.prior.head;
  typename E::T *out = (typename E::T *)(a.out.p + (int64_t)b * a.out.token + (int64_t)head * a.out.head);
  // the earlier result stands for one row of weight 1 at its lse
  // (read before a barrier, or by the wave that writes: lse may be the same memory)
  const float z0 = a.prior.p ? a.prior_lse[row] * (1.f / kLn2) : neg_inf();
  if constexpr (WAVES == 1) {
    const float mm = fmaxf(top, z0), w0 = z0 == neg_inf() ? 0.f : ex2(z0 - mm), w = part_scale(top, mm), sum = w0 + l * w;
    const bool some = sum > 0.f || sum != sum;
#pragma unroll
    for (int i = 0; i < 32 / GROUPS; i++) {
      const int at = c * 32 + first + i;
      if (at < (int)a.dim) {
        const float o0 = a.prior.p ? (float)((const typename E::T *)prior)[at] : 0.f;
        const float o = (w0 == 0.f ? 0.f : w0 * o0) + acc[i] * w;
        out[at] = (typename E::T)(some ? o / sum : 0.f);
      }
    }
    if (lane == 0 && a.lse) a.lse[row] = some ? (mm + lg2(sum)) * kLn2 : neg_inf();
    return;
  }
#pragma unroll
  for (int i = 0; i < 32 / GROUPS; i++) sacc[wave][c * 32 + first + i] = acc[i];
  if (lane == 0) sml[wave] = make_float2(top, l);
  __syncthreads();
  if (t >= DP) return;
  const float o0 = a.prior.p && t < (int)a.dim ? (float)((const typename E::T *)prior)[t] : 0.f;
  float mm = z0;
#pragma unroll
  for (int w = 0; w < 4; w++) mm = fmaxf(mm, sml[w].x);
  const float w0 = z0 == neg_inf() ? 0.f : ex2(z0 - mm);
  float sum = w0, o = w0 == 0.f ? 0.f : w0 * o0;
#pragma unroll
  for (int w = 0; w < 4; w++) {
    const float s = part_scale(sml[w].x, mm);
    sum += sml[w].y * s;
    o += sacc[w][t] * s;
  }
  const bool some = sum > 0.f || sum != sum;
  if (t < (int)a.dim) out[t] = (typename E::T)(some ? o / sum : 0.f);
  if (t == 0 && a.lse) a.lse[row] = some ? (mm + lg2(sum)) * kLn2 : neg_inf();
}

template <class E, int WAVES>
hipError_t ids_type(const IdsArgs &a, hipStream_t st) {
  const uint32_t lists = a.n_seq * a.q_heads;
  const dim3 grid((lists + 4 / WAVES - 1) / (4 / WAVES));
  if (a.dim <= 64) k_ids_packed<E, 64, WAVES><<<grid, 256, 0, st>>>(a);
  else if (a.dim <= 128) k_ids_packed<E, 128, WAVES><<<grid, 256, 0, st>>>(a);
  else k_ids_packed<E, 256, WAVES><<<grid, 256, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_ids_packed(bool f16, const IdsArgs &a, hipStream_t st) {
  const uint32_t pass = a.dim <= 64 ? 512 : a.dim <= 128 ? 256 : 128;  // ids that four waves ask for at once
  const bool held = a.pg.bytes <= 64u << 20;                       // keys' codes; as much again for the values'
  if (a.n_seq * a.q_heads >= 2048 && (a.k < pass || held)) return f16 ? ids_type<F16, 1>(a, st) : ids_type<Bf16, 1>(a, st);
  return f16 ? ids_type<F16, 4>(a, st) : ids_type<Bf16, 4>(a, st);
}

hipError_t launch_append_packed(const AppendArgs &a, hipStream_t st) {
  const uint32_t threads = a.s.max_q * a.kv_heads * ((a.dim + 31) / 32 * 4);
  const dim3 grid((threads + 255) / 256, a.s.n_seq);
  if (a.f16) k_append_packed<F16><<<grid, 256, 0, st>>>(a);
  else k_append_packed<Bf16><<<grid, 256, 0, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_read(const ReadArgs &a, hipStream_t st) {
  const uint32_t grid = (uint32_t)(((uint64_t)a.n * a.kv_heads * (a.dim / 8) + 255) / 256);
  if (a.f16) k_read<F16><<<grid, 256, 0, st>>>(a);
  else k_read<Bf16><<<grid, 256, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace gr
