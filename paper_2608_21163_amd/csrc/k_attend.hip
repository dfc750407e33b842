// k_attend.hip -- attention over 16-bit pages: which kernels run, and the kernels
// themselves where no first tokens are kept visible.
#include "attend.h"

namespace gr {
namespace {

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
  const KeyLine<Sinks> line(a, ch, r0 / a.group, r1 / a.group);
  const uint32_t n = max(1u, (line.hi - line.lo + a.split - 1) / a.split);
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
  const KeyLine<Sinks> line(a, ch, r0 / a.group, r1 / a.group);
  const uint32_t n = min(max(1u, (line.hi - line.lo + a.split - 1) / a.split), kShortSplits);
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

// Where part s of a sequence's row lies (share_of): the first unit may have begun
// with an earlier sequence, the others begin with this one.
__device__ __forceinline__ size_t unit_part(const AttendArgs &a, const Share &sh, uint32_t u0, uint32_t s, uint32_t kvh, uint32_t r, uint32_t tile_rows) {
  return (((size_t)(u0 + s) * 2 + (s == 0 && u0 * sh.per != sh.before ? 1 : 0)) * a.kv_heads + kvh) * tile_rows + r;
}

// The same for shares of all sequences' keys (share_of): a sequence whose keys
// lie in one unit's share has its results already.
template <class E, int LQ>
__global__ __launch_bounds__(256) void k_attend_join_units(AttendArgs a, uint32_t tile_rows) {
  constexpr int G = 256 / LQ, CHUNK = 1024;
  __shared__ float2 ml[4];
  __shared__ float factor[CHUNK];
  __shared__ v4f acc[256];
  const uint32_t b = blockIdx.y, kvh = blockIdx.x % a.kv_heads, r = blockIdx.x / a.kv_heads;
  const Chunk ch = chunk_of(a.s, b, a.err);
  if (r >= ch.ql * a.group) return;
  const Share sh = share_of(a, false, [&](uint32_t) { return b; });
  const uint32_t u0 = sh.before / sh.per, u1 = (sh.before + steps_of(a, b) - 1) / sh.per, n = u1 - u0 + 1;
  if (n == 1) return;
  const uint32_t token = ch.r0 + r / a.group, head = kvh * a.group + r % a.group;
  const size_t row = (size_t)token * a.q_heads + head;
  auto place = [&](uint32_t s) { return unit_part(a, sh, u0, s, kvh, r, tile_rows); };
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  float m = neg_inf(), l = 0.f;
  for (uint32_t s = t; s < n; s += 256) {
    const float2 x = a.part_ml[place(s)];
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
      const float x = a.part_ml[place(s0 + s)].x;
      factor[s] = x == neg_inf() ? 1.f : ex2(x - m);
    }
    __syncthreads();
    if (c * 4 < (int)a.dim) {
#pragma unroll 4
      for (uint32_t s = g; s < m1; s += G) o += *(const v4f *)(a.part + place(s0 + s) * a.dim + c * 4) * factor[s];
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

// For few parts a sequence: LQ lanes a row, eight parts at a time.
template <class E, int LQ>
__global__ __launch_bounds__(256) void k_attend_join_units_short(AttendArgs a, uint32_t tile_rows) {
  const uint32_t b = blockIdx.y;
  const Chunk ch = chunk_of(a.s, b, a.err);
  const uint32_t x = blockIdx.x * (256 / LQ) + threadIdx.x / LQ, c = threadIdx.x % LQ;
  const uint32_t kvh = x % a.kv_heads, r = x / a.kv_heads;
  const Share sh = share_of(a, false, [&](uint32_t) { return b; });
  const uint32_t u0 = sh.before / sh.per, u1 = (sh.before + steps_of(a, b) - 1) / sh.per, n = u1 - u0 + 1;
  if (n == 1 || r >= ch.ql * a.group || c * 4 >= a.dim) return;
  const uint32_t token = ch.r0 + r / a.group, head = kvh * a.group + r % a.group;
  const size_t row = (size_t)token * a.q_heads + head;
  float m = neg_inf(), l = 0.f;
  v4f o{0, 0, 0, 0};
  for (uint32_t s0 = 0; s0 < n; s0 += kShortSplits) {
    float2 ml[kShortSplits];
    v4f part[kShortSplits];
    float top = m;
#pragma unroll
    for (uint32_t s = 0; s < kShortSplits; s++) {
      ml[s] = make_float2(neg_inf(), 0.f);
      part[s] = v4f{0, 0, 0, 0};
      if (s0 + s < n) {
        const size_t at = unit_part(a, sh, u0, s0 + s, kvh, r, tile_rows);
        ml[s] = a.part_ml[at];
        part[s] = *(const v4f *)(a.part + at * a.dim + c * 4);
      }
    }
#pragma unroll
    for (uint32_t s = 0; s < kShortSplits; s++) top = fmaxf(top, ml[s].x);
    const float f0 = m == neg_inf() ? 1.f : ex2(m - top);
    l *= f0;
    o *= f0;
#pragma unroll
    for (uint32_t s = 0; s < kShortSplits; s++) {
      const float f = ml[s].x == neg_inf() ? 1.f : ex2(ml[s].x - top);
      l += ml[s].y * f;
      o += part[s] * f;
    }
    m = top;
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
// half of the cache.  PAST: scores that the caches do not hold are read past them, and the weights
// written so (two packed sequences of 131,072, 33 MB of scores, heads outside slots: the call
// 88 us -> 80; 8 MB of them 32.6, past the caches 33.2).
template <bool PAST>
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
    // (scores of places that no tile covers were not written)
    const KeyLine<Sinks> line(a, ch, 0, (rows - 1) / a.group);
    const uint32_t front = line.gap ? a.sink_keys : 0, lo = front + line.gap, hi = line.hi + line.gap;
    const float *sc = a.scores + ((size_t)b * a.kv_heads + kvh) * a.score_rows * a.score_keys;
#pragma unroll 4
    for (uint32_t r = 0; r < rows; r++)
#pragma unroll
      for (int j = 0; j < 4; j++) {
        const uint32_t key = key0 + j * 256;
        if ((key >= lo || key < front) && key < hi) {
          const float *at = sc + (size_t)r * a.score_keys + key;
          const float x = PAST ? __builtin_nontemporal_load(at) : *at;
          sum[j] += x == neg_inf() ? 0.f : ex2(x - z[r]);  // hidden: nothing, though the row's sum be NaN
        }
      }
  }
  float *wout = a.wout.p + (int64_t)b * a.wout.seq + (int64_t)kvh * a.wout.head;
#pragma unroll
  for (int j = 0; j < 4; j++)
    if (key0 + j * 256 < ch.kl) {
      if (PAST) __builtin_nontemporal_store(old[j] + sum[j], wout + key0 + j * 256);
      else wout[key0 + j * 256] = old[j] + sum[j];
    }
}

__global__ __launch_bounds__(256) void k_weights_add(AttendArgs a) {
  const uint32_t b = blockIdx.y, kvh = blockIdx.x % a.kv_heads, key0 = blockIdx.x / a.kv_heads * kAgainKeys, key = key0 + threadIdx.x;
  const Chunk ch = chunk_of(a.s, b, a.err);
  if (key >= ch.kl) return;
  const AgainRows range = again_rows<Sinks>(a, ch, key0);
  const float old = a.win.p[(int64_t)b * a.win.seq + (int64_t)kvh * a.win.head + key];
  float sum = 0.f;
  if (range.n) {
    const float *at = a.row_sums + ((size_t)b * a.kv_heads + kvh) * a.sum_keys + again_tile<Sinks>(a, ch, key0) * kAgainKeys + threadIdx.x;
    const size_t part = (size_t)a.s.n_seq * a.kv_heads * a.sum_keys;
#pragma unroll 4
    for (uint32_t i = 0; i < range.n; i++) sum += at[i * part];
  }
  a.wout.p[(int64_t)b * a.wout.seq + (int64_t)kvh * a.wout.head + key] = old + sum;
}

}  // namespace

hipError_t launch_attend(uint32_t tile_rows, bool f16, const AttendArgs &a, hipStream_t st) {
  if (a.sc.k) return launch_attend_packed(tile_rows, f16, a, st);
  if (a.sinks) return launch_attend_sinks(tile_rows, f16, a, st);
  return f16 ? attend_type<F16, Whole>(tile_rows, a, st) : attend_type<Bf16, Whole>(tile_rows, a, st);
}

template <class E>
static hipError_t join_type(const AttendArgs &a, uint32_t tile_rows, hipStream_t st) {
  const uint32_t rows = a.s.max_q * a.q_heads;
  if (a.units && a.units <= 4 * a.s.n_seq) {  // some sequences may have more than eight parts, few have
    if (a.dim <= 64) k_attend_join_units_short<E, 16><<<dim3((rows + 15) / 16, a.s.n_seq), 256, 0, st>>>(a, tile_rows);
    else if (a.dim <= 128) k_attend_join_units_short<E, 32><<<dim3((rows + 7) / 8, a.s.n_seq), 256, 0, st>>>(a, tile_rows);
    else k_attend_join_units_short<E, 64><<<dim3((rows + 3) / 4, a.s.n_seq), 256, 0, st>>>(a, tile_rows);
    return hipGetLastError();
  }
  if (a.units) {
    const dim3 grid(rows, a.s.n_seq);
    if (a.dim <= 64) k_attend_join_units<E, 16><<<grid, 256, 0, st>>>(a, tile_rows);
    else if (a.dim <= 128) k_attend_join_units<E, 32><<<grid, 256, 0, st>>>(a, tile_rows);
    else k_attend_join_units<E, 64><<<grid, 256, 0, st>>>(a, tile_rows);
    return hipGetLastError();
  }
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
    const dim3 grid((a.s.max_k + 1023) / 1024, a.kv_heads, a.s.n_seq);
    if ((uint64_t)a.s.n_seq * a.kv_heads * a.score_rows * a.score_keys >= 1 << 23) k_weights_stored<true><<<grid, 256, 0, st>>>(a);
    else k_weights_stored<false><<<grid, 256, 0, st>>>(a);
    return hipGetLastError();
  }
  const hipError_t e = a.sc.k ? launch_weights_packed(f16, a, st) : a.sinks ? launch_weights_sinks(f16, a, st)
                       : f16 ? weights_type<F16, Whole>(a, st) : weights_type<Bf16, Whole>(a, st);
  if (e != hipSuccess || !a.row_sums) return e;
  k_weights_add<<<dim3((a.s.max_k + kAgainKeys - 1) / kAgainKeys * a.kv_heads, a.s.n_seq), 256, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace gr
