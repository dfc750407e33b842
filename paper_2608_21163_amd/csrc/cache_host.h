// cache_host.h -- what the host side of the key/value-cache operators shares
// (cache.hip, pages.hip): handles, checks of arguments, workspaces.
#pragma once
#include "cache.h"

#include <math.h>
#include <stdarg.h>
#include <stdio.h>
#include <string.h>

#include <algorithm>
#include <new>

#include "../../include/grand.h"

using namespace gr;

struct grand_cache {
  grand_cache_params p;
  hipStream_t stream = nullptr;
  bool poisoned = false;
  uint32_t shift = 0;       // log2 of the page size
  uint8_t *ws = nullptr;    // workspace
  size_t ws_bytes = 0;
  bool ws_captured = false; // a graph may use it: kept until the handle goes
  struct Kept { uint8_t *p; Kept *next; } *kept = nullptr;
  CacheErr *err = nullptr;  // device
  // allocations that buffers of the present call were found in: small
  // tensors share theirs, and asking for one takes 0.6 us
  struct { uintptr_t base, end; } seen[4];
  int n_seen = 0;
  char msg[256] = "";
};

namespace {

constexpr float kLog2e = 1.44269504088896341f;
constexpr uint64_t kMostGroups = 1u << 24;  // workgroups of 256 in a grid's x: fewer than 2^32 threads

grand_status fail(grand_cache *h, grand_status code, const char *fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(h->msg, sizeof h->msg, fmt, ap);
  va_end(ap);
  return code;
}

grand_status fail_dev(grand_cache *h, hipError_t e, const char *what) {
  (void)hipGetLastError();  // the error stays with this handle
  // refusals during a stream capture (the codes are consecutive): nothing was enqueued
  if (e >= hipErrorStreamCaptureUnsupported && e <= hipErrorStreamCaptureWrongThread)
    return fail(h, GRAND_E_STATE, "a stream capture does not allow %s: %s", what, hipGetErrorString(e));
  h->poisoned = true;
  return fail(h, GRAND_E_DEVICE, "HIP error in %s: %s", what, hipGetErrorString(e));
}

#define HCHK(h, x)                                      \
  do {                                                  \
    hipError_t e_ = (x);                                \
    if (e_ != hipSuccess) return fail_dev((h), e_, #x); \
  } while (0)
#define TRY(x)                            \
  do {                                    \
    const grand_status s_ = (x);          \
    if (s_ != GRAND_OK) return s_;        \
  } while (0)

grand_status check_usable(grand_cache *h) {
  if (!h) return GRAND_E_ARG;
  if (h->poisoned) return GRAND_E_STATE;
  h->msg[0] = 0;
  h->n_seen = 0;
  return GRAND_OK;
}

// Calls that wait for the handle's stream would break its capture.
grand_status check_no_capture(grand_cache *h, const char *call) {
  hipStreamCaptureStatus cs = hipStreamCaptureStatusNone;
  HCHK(h, hipStreamIsCapturing(h->stream, &cs));
  return cs == hipStreamCaptureStatusNone ? GRAND_OK : fail(h, GRAND_E_STATE, "%s waits for the stream, which a capture does not allow", call);
}

// A buffer must lie in this GPU's memory, and its allocation must hold it.
grand_status check_mem(grand_cache *h, const char *name, const void *p, uint64_t bytes, size_t align) {
  if (!p) return fail(h, GRAND_E_ARG, "%s is null", name);
  if ((uintptr_t)p % align) return fail(h, GRAND_E_ARG, "%s is not aligned to %zu bytes", name, align);
  for (int i = 0; i < h->n_seen; i++)
    if ((uintptr_t)p >= h->seen[i].base && (uintptr_t)p < h->seen[i].end)
      return bytes <= h->seen[i].end - (uintptr_t)p ? GRAND_OK : fail(h, GRAND_E_ARG, "%s is shorter than the call needs", name);
  hipPointerAttribute_t a{};
  if (hipPointerGetAttributes(&a, p) != hipSuccess || a.type != hipMemoryTypeDevice || a.device != h->p.device) {
    (void)hipGetLastError();
    return fail(h, GRAND_E_ARG, "%s is not memory of GPU %d", name, h->p.device);
  }
  hipDeviceptr_t base = nullptr;
  size_t size = 0;
  if (hipMemGetAddressRange(&base, &size, const_cast<void *>(p)) != hipSuccess) {
    (void)hipGetLastError();
    return fail(h, GRAND_E_ARG, "%s has no device allocation", name);
  }
  if (h->n_seen < 4) h->seen[h->n_seen++] = {(uintptr_t)base, (uintptr_t)base + size};
  const uint64_t room = (uint64_t)((uintptr_t)base + size - (uintptr_t)p);
  if (bytes > room) return fail(h, GRAND_E_ARG, "%s is shorter than the call needs", name);
  return GRAND_OK;
}

// The stride of an axis of one element says nothing (views may have any).
int64_t step(uint64_t n, int64_t stride) { return n > 1 ? stride : 0; }

// Elements up to which rows n0 x n1 x n2 at these strides reach; false when
// a stride is negative or the extent does not fit 62 bits.
bool extent(uint64_t n0, int64_t s0, uint64_t n1, int64_t s1, uint64_t n2, int64_t s2, uint64_t row, uint64_t *out) {
  if (s0 < 0 || s1 < 0 || s2 < 0) return false;
  const __uint128_t e = (__uint128_t)(n0 - 1) * s0 + (__uint128_t)(n1 - 1) * s1 + (__uint128_t)(n2 - 1) * s2 + row;
  if (e >> 62) return false;
  *out = (uint64_t)e;
  return true;
}

// Rows of len bytes at p + i0 * s0 + i1 * s1, and what two of them share.
struct Region {
  uintptr_t p;
  uint64_t n0, n1;
  int64_t s0, s1;
  uint64_t len;
};
Region region(const RowsView &r, uint64_t tokens, uint64_t heads, uint32_t dim) {
  return {(uintptr_t)r.p, tokens, heads, r.token, r.head, dim * 2ull};
}
Region region(const WeightsView &w, uint64_t n_seq, uint64_t heads, uint64_t cap) {
  return {(uintptr_t)w.p, n_seq, heads, w.seq * 4, w.head * 4, cap * 4};
}
Region region(const void *p, uint64_t bytes) { return {(uintptr_t)p, 1, 1, 0, 0, bytes}; }

bool same_rows(const Region &a, const Region &b) {
  return a.p == b.p && (a.n0 == 1 || a.s0 == b.s0) && (a.n1 == 1 || a.s1 == b.s1);
}
int64_t floor_div(int64_t x, int64_t y) { return x / y - (x % y < 0); }  // y > 0
// Rows of like strides may lie between each other's; rows of other strides
// share memory if one's lies inside the other's extent at all.
bool overlap(Region a, Region b) {
  if (!a.len || !b.len) return false;
  if (a.p + (a.n0 - 1) * a.s0 + (a.n1 - 1) * a.s1 + a.len <= b.p || b.p + (b.n0 - 1) * b.s0 + (b.n1 - 1) * b.s1 + b.len <= a.p) return false;
  // the stride of an axis of one row says nothing
  if (a.n0 == 1) a.s0 = b.s0;
  if (b.n0 == 1) b.s0 = a.s0;
  if (a.n1 == 1) a.s1 = b.s1;
  if (b.n1 == 1) b.s1 = a.s1;
  if (a.s0 != b.s0 || a.s1 != b.s1) return true;
  for (int64_t i1 = 1 - (int64_t)a.n1; i1 < (int64_t)b.n1; i1++) {
    // rows of a at 0 and of b at d + i0 * s0: some i0 of theirs with -len(b) < that < len(a)
    const int64_t d = (int64_t)(b.p - a.p) + i1 * a.s1, la = (int64_t)a.len, lb = (int64_t)b.len;
    if (a.s0 == 0 ? d < la && -d < lb
                  : std::max(floor_div(-lb - d, a.s0) + 1, 1 - (int64_t)a.n0) <= std::min(-floor_div(d - la, a.s0) - 1, (int64_t)b.n0 - 1))
      return true;
  }
  return false;
}

grand_status check_rows(grand_cache *h, const char *name, const grand_rows *r, uint64_t tokens, uint32_t heads, bool written,
                        RowsView *out) {
  if (!r) return fail(h, GRAND_E_ARG, "%s is null", name);
  uint64_t e = 0;
  const int64_t token = step(tokens, r->token_stride), head = step(heads, r->head_stride);
  if (token % 8 || head % 8 || !extent(tokens, token, heads, head, 1, 0, h->p.head_dim, &e))
    return fail(h, GRAND_E_ARG, "strides of %s must be multiples of 8 elements, not negative", name);
  // rows that are written must not overlap: one head's rows lie inside the
  // other stride
  if (written) {
    const uint64_t d = h->p.head_dim, ts = (uint64_t)token, hs = (uint64_t)head;
    const bool ok = (heads == 1 || hs >= d) && (tokens == 1 || ts >= d) &&
                    (tokens == 1 || heads == 1 || ts >= (heads - 1) * hs + d || hs >= (tokens - 1) * ts + d);
    if (!ok) return fail(h, GRAND_E_ARG, "rows of %s overlap", name);
  }
  TRY(check_mem(h, name, r->p, e * 2, 16));
  out->p = static_cast<uint8_t *>(r->p);
  out->token = token * 2;
  out->head = head * 2;
  return GRAND_OK;
}

grand_status check_pages(grand_cache *h, const grand_pages *g, PagesView *out) {
  if (!g) return fail(h, GRAND_E_ARG, "pages is null");
  uint64_t e = 0;
  if (g->n_pages == 0) return fail(h, GRAND_E_ARG, "the pool has no pages");
  if ((uint64_t)g->n_pages << h->shift > 0xFFFFFFFFull) return fail(h, GRAND_E_CAPACITY, "a pool holds fewer than 2^32 slots");
  const int64_t page = step(g->n_pages, g->page_stride), slot = step(h->p.page_size, g->slot_stride), head = step(h->p.kv_heads, g->head_stride);
  if (page % 8 || slot % 8 || head % 8 ||
      !extent(g->n_pages, page, h->p.page_size, slot, h->p.kv_heads, head, h->p.head_dim, &e))
    return fail(h, GRAND_E_ARG, "strides of pages must be multiples of 8 elements, not negative");
  // offsets inside a page are computed in 32 bits
  uint64_t in_page = 0;
  if (!extent(1, 0, h->p.page_size, slot, h->p.kv_heads, head, h->p.head_dim, &in_page) || in_page >= 1ull << 31 ||
      page >= 1ll << 31 || slot >= 1ll << 31 || head >= 1ll << 31)
    return fail(h, GRAND_E_CAPACITY, "a page and its strides must stay below 2^31 elements");
  TRY(check_mem(h, "pages.k", g->k, e * 2, 16));
  TRY(check_mem(h, "pages.v", g->v, e * 2, 16));
  out->k = static_cast<const uint8_t *>(g->k);
  out->v = static_cast<const uint8_t *>(g->v);
  out->page = (uint32_t)page * 2;
  out->slot = (uint32_t)slot * 2;
  out->head = (uint32_t)head * 2;
  out->bytes = e * 2;
  out->n_pages = g->n_pages;
  out->shift = h->shift;
  return GRAND_OK;
}

// The rows of a pool that is written, by page, slot and head: rows of `row`
// bytes, axes in the order of their strides.
struct PoolRows {
  uintptr_t p;
  uint64_t row;
  struct { uint64_t n, s; } axes[3];
};
PoolRows pool_rows(const grand_cache_params &p, const void *at, uint64_t row, uint32_t n_pages, uint32_t page, uint32_t slot, uint32_t head) {
  PoolRows r{(uintptr_t)at, row, {{n_pages, page}, {p.page_size, slot}, {p.kv_heads, head}}};
  std::sort(r.axes, r.axes + 3, [](const auto &a, const auto &b) { return a.s < b.s; });
  return r;
}
// No two of its rows share memory: every axis steps over all that the shorter
// steps reach.
bool rows_apart(const PoolRows &r) {
  uint64_t reach = r.row;
  for (const auto &x : r.axes) {
    if (x.n == 1) continue;
    if (x.s < reach) return false;
    reach += (x.n - 1) * x.s;
  }
  return true;
}
// Whether rows of two such pools may share memory, a's first at 0 and b's at d, along the
// `axes` shortest axes.  Along an axis of the same steps in both only those
// rows can meet whose steps are as far apart as d is, or one more: what the shorter axes reach
// lies within a step.  From the first unlike axis on (codes and scales of a page, side by side)
// the extents are compared.
bool rows_meet(const PoolRows &a, const PoolRows &b, int axes, int64_t d) {
  int64_t ra = (int64_t)a.row, rb = (int64_t)b.row;
  for (int i = 0; i < axes; i++) {
    ra += (int64_t)((a.axes[i].n - 1) * a.axes[i].s);
    rb += (int64_t)((b.axes[i].n - 1) * b.axes[i].s);
  }
  if (d >= ra || -d >= rb) return false;
  if (axes == 0) return true;
  const auto &x = a.axes[axes - 1], &y = b.axes[axes - 1];
  if (x.n != y.n) return true;
  if (x.n == 1) return rows_meet(a, b, axes - 1, d);
  if (x.s != y.s) return true;
  const int64_t n = (int64_t)x.n, s = (int64_t)x.s, t = floor_div(-d, s);
  return (t > -n && t < n && rows_meet(a, b, axes - 1, d + t * s)) || (t + 1 > -n && t + 1 < n && rows_meet(a, b, axes - 1, d + (t + 1) * s));
}
// (of pools whose own rows are apart)
bool pools_apart(const PoolRows &a, const PoolRows &b) { return !rows_meet(a, b, 3, (int64_t)(b.p - a.p)); }

// Pages that are written: no row shares memory with another; keys and values may be one pool.
grand_status check_pages_apart(grand_cache *h, const PagesView &g) {
  const PoolRows k = pool_rows(h->p, g.k, h->p.head_dim * 2, g.n_pages, g.page, g.slot, g.head);
  const PoolRows v = pool_rows(h->p, g.v, h->p.head_dim * 2, g.n_pages, g.page, g.slot, g.head);
  if (!rows_apart(k)) return fail(h, GRAND_E_ARG, "slots of pages overlap");
  return g.k == g.v || pools_apart(k, v) ? GRAND_OK : fail(h, GRAND_E_ARG, "keys and values overlap");
}

// Packed pages: rows of whole blocks, their scales beside them.
struct PackedBytes { uint64_t codes, scales; };  // up to the last row's last
grand_status check_packed(grand_cache *h, const grand_packed *g, PagesView *out, ScalesView *sc, PackedBytes *bytes) {
  if (!g) return fail(h, GRAND_E_ARG, "pages is null");
  if (g->n_pages == 0) return fail(h, GRAND_E_ARG, "the pool has no pages");
  if ((uint64_t)g->n_pages << h->shift > 0xFFFFFFFFull) return fail(h, GRAND_E_CAPACITY, "a pool holds fewer than 2^32 slots");
  const grand_cache_params &p = h->p;
  const uint32_t blocks = (p.head_dim + 31) / 32;
  const int64_t page = step(g->n_pages, g->page_stride), slot = step(p.page_size, g->slot_stride), head = step(p.kv_heads, g->head_stride);
  const int64_t spage = step(g->n_pages, g->scale_page_stride), sslot = step(p.page_size, g->scale_slot_stride),
                shead = step(p.kv_heads, g->scale_head_stride);
  uint64_t in_page = 0, in_scales = 0;
  if (page % 16 || slot % 16 || head % 16 || !extent(g->n_pages, page, p.page_size, slot, p.kv_heads, head, blocks * 16, &bytes->codes))
    return fail(h, GRAND_E_ARG, "strides of packed pages must be multiples of 16 bytes, not negative");
  if (!extent(g->n_pages, spage, p.page_size, sslot, p.kv_heads, shead, blocks, &bytes->scales))
    return fail(h, GRAND_E_ARG, "strides of scales must not be negative");
  // offsets inside a page are computed in 32 bits
  if (!extent(1, 0, p.page_size, slot, p.kv_heads, head, blocks * 16, &in_page) ||
      !extent(1, 0, p.page_size, sslot, p.kv_heads, shead, blocks, &in_scales) || in_page >= 1ull << 32 || in_scales >= 1ull << 32 ||
      page >= 1ll << 32 || slot >= 1ll << 32 || head >= 1ll << 32 || spage >= 1ll << 32 || sslot >= 1ll << 32 || shead >= 1ll << 32)
    return fail(h, GRAND_E_CAPACITY, "a page and its strides must stay below 2^32 bytes");
  TRY(check_mem(h, "pages.k", g->k, bytes->codes, 16));
  TRY(check_mem(h, "pages.v", g->v, bytes->codes, 16));
  TRY(check_mem(h, "pages.k_scales", g->k_scales, bytes->scales, 1));
  TRY(check_mem(h, "pages.v_scales", g->v_scales, bytes->scales, 1));
  *out = {g->k, g->v, (uint32_t)page, (uint32_t)slot, (uint32_t)head, g->n_pages, h->shift, bytes->codes};
  *sc = {g->k_scales, g->v_scales, (uint32_t)spage, (uint32_t)sslot, (uint32_t)shead};
  return GRAND_OK;
}

// Packed pages that are written: no row shares memory with another.
grand_status check_packed_apart(grand_cache *h, const PagesView &g, const ScalesView &sc) {
  const uint32_t blocks = (h->p.head_dim + 31) / 32;
  const PoolRows r[] = {pool_rows(h->p, g.k, blocks * 16, g.n_pages, g.page, g.slot, g.head),
                        pool_rows(h->p, g.v, blocks * 16, g.n_pages, g.page, g.slot, g.head),
                        pool_rows(h->p, sc.k, blocks, g.n_pages, sc.page, sc.slot, sc.head),
                        pool_rows(h->p, sc.v, blocks, g.n_pages, sc.page, sc.slot, sc.head)};
  const bool one = g.k == g.v && sc.k == sc.v;  // keys that are values: the caller sees to it that both are written alike
  for (int i = 0; i < 4; i++) {
    if (!rows_apart(r[i])) return fail(h, GRAND_E_ARG, "slots of pages overlap");
    for (int j = 0; j < i; j++)
      if (!(one && i - j != 2 && i / 2 == j / 2) && !pools_apart(r[i], r[j])) return fail(h, GRAND_E_ARG, "codes and scales of keys and values overlap");
  }
  return GRAND_OK;
}

grand_status check_apart(grand_cache *h, const Region &out, const PagesView &pg, const ScalesView &sc, uint64_t scale_bytes) {
  return overlap(out, region(pg.k, pg.bytes)) || overlap(out, region(pg.v, pg.bytes)) || overlap(out, region(sc.k, scale_bytes)) ||
                 overlap(out, region(sc.v, scale_bytes))
             ? fail(h, GRAND_E_ARG, "out overlaps pages") : GRAND_OK;
}

grand_status check_seqs(grand_cache *h, const grand_seqs *s, bool chunks, SeqsView *out) {
  if (!s) return fail(h, GRAND_E_ARG, "seqs is null");
  if (s->n_seq > 65535) return fail(h, GRAND_E_CAPACITY, "at most 65535 sequences a call");
  const int64_t stride = s->n_seq > 1 ? s->table_stride : s->max_pages;
  if (stride < (int64_t)s->max_pages) return fail(h, GRAND_E_ARG, "table_stride is below max_pages");
  if (s->max_k > (uint64_t)s->max_pages << h->shift) return fail(h, GRAND_E_ARG, "max_k tokens do not fit max_pages pages");
  if (s->max_k >= 1u << 31) return fail(h, GRAND_E_CAPACITY, "max_k must be below 2^31");
  if (chunks) {
    if (!s->q_start && (s->n_tokens != s->n_seq || s->max_q != 1))
      return fail(h, GRAND_E_ARG, "without q_start every sequence has one new token (n_tokens = n_seq, max_q = 1)");
    // positions are ints: to a tile of 64 keys past the last, and a window before a chunk longer than its cache
    if ((uint64_t)s->max_k + std::min(s->max_q, s->n_tokens) > (1u << 31) - 64)
      return fail(h, GRAND_E_CAPACITY, "max_k and max_q must be at most 2^31 - 64 together");
    if (s->q_start) TRY(check_mem(h, "q_start", s->q_start, ((uint64_t)s->n_seq + 1) * 4, 4));
  }
  uint64_t e = 0;
  if (!extent(s->n_seq, stride, 1, 0, 1, 0, s->max_pages, &e)) return fail(h, GRAND_E_ARG, "table_stride is too large");
  if (s->max_pages) TRY(check_mem(h, "table", s->table, e * 4, 4));
  TRY(check_mem(h, "lens", s->lens, (uint64_t)s->n_seq * 4, 4));
  out->table = s->table;
  out->table_stride = stride;
  out->q_start = s->q_start;
  out->lens = s->lens;
  out->n_seq = s->n_seq;
  out->n_tokens = s->n_tokens;
  out->max_pages = s->max_pages;
  out->max_q = std::min(s->max_q, s->n_tokens);
  out->max_k = s->max_k;
  return GRAND_OK;
}

grand_status check_weights(grand_cache *h, const char *name, const grand_weights *w, uint32_t n_seq, uint32_t heads, uint32_t cap,
                           bool written, WeightsView *out) {
  if (!w) return fail(h, GRAND_E_ARG, "%s is null", name);
  uint64_t e = 0;
  const int64_t seq = step(n_seq, w->seq_stride), head = step(heads, w->head_stride);
  if (!extent(n_seq, seq, heads, head, 1, 0, cap, &e)) return fail(h, GRAND_E_ARG, "strides of %s are negative", name);
  if (written) {
    const uint64_t ss = (uint64_t)seq, hs = (uint64_t)head, c = cap;
    const bool ok = (heads == 1 || hs >= c) && (n_seq == 1 || ss >= c) &&
                    (n_seq == 1 || heads == 1 || ss >= (heads - 1) * hs + c || hs >= (n_seq - 1) * ss + c);
    if (!ok) return fail(h, GRAND_E_ARG, "rows of %s overlap", name);
  }
  TRY(check_mem(h, name, w->p, e * 4, 4));
  out->p = w->p;
  out->seq = seq;
  out->head = head;
  return GRAND_OK;
}

// A workspace of parts of these sizes, each 256-byte aligned.
struct Parts {
  size_t at[8] = {}, total = 0;
  int n = 0;
  int add(uint64_t bytes) {
    at[n] = total;
    total += (bytes + 255) / 256 * 256;
    return n++;
  }
};
grand_status ensure_ws(grand_cache *h, size_t bytes) {
  if (!bytes) return GRAND_OK;
  hipStreamCaptureStatus cs = hipStreamCaptureStatusNone;
  HCHK(h, hipStreamIsCapturing(h->stream, &cs));
  const bool capturing = cs != hipStreamCaptureStatusNone;
  if (bytes <= h->ws_bytes) {
    h->ws_captured |= capturing;
    return GRAND_OK;
  }
  if (capturing)
    return fail(h, GRAND_E_CAPACITY, "the workspace must grow to %zu bytes: run the call once before the capture", bytes);
  HCHK(h, hipStreamSynchronize(h->stream));
  if (h->ws_captured) {
    grand_cache::Kept *k = new (std::nothrow) grand_cache::Kept{h->ws, h->kept};
    if (!k) return fail(h, GRAND_E_OOM, "no host memory");
    h->kept = k;
  } else if (h->ws) {
    (void)hipFree(h->ws);
  }
  h->ws = nullptr;
  h->ws_bytes = 0;
  h->ws_captured = false;
  const size_t want = bytes + bytes / 4;
  if (hipMalloc((void **)&h->ws, want) != hipSuccess) {
    (void)hipGetLastError();
    h->ws = nullptr;
    return fail(h, GRAND_E_OOM, "no memory for a workspace of %zu bytes", want);
  }
  h->ws_bytes = want;
  return GRAND_OK;
}

}  // namespace
