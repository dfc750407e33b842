// cache.hip -- the host side of the key/value-cache operators: checks of
// arguments, plans, workspaces and launches.  No call here waits for the GPU
// unless a workspace grows.
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

// No two slots, heads or pages of pools that are written share memory: every
// axis steps over all that the shorter steps reach.
bool slots_apart(const grand_cache_params &p, const PagesView &g) {
  const uint64_t n = p.page_size;
  struct { uint64_t n, s; } axes[] = {{g.n_pages, g.page}, {n, g.slot}, {p.kv_heads, g.head}};
  std::sort(axes, axes + 3, [](const auto &a, const auto &b) { return a.s < b.s; });
  uint64_t reach = p.head_dim * 2;
  for (const auto &x : axes) {
    if (x.n == 1) continue;
    if (x.s < reach) return false;
    reach += (x.n - 1) * x.s;
  }
  return true;
}

grand_status check_apart(grand_cache *h, const Region &out, const PagesView &pg) {
  return overlap(out, region(pg.k, pg.bytes)) || overlap(out, region(pg.v, pg.bytes)) ? fail(h, GRAND_E_ARG, "out overlaps pages") : GRAND_OK;
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

extern "C" {

void grand_default_cache_params(grand_cache_params *p) {
  if (!p) return;
  memset(p, 0, sizeof *p);
  p->struct_size = sizeof(grand_cache_params);
  p->dtype = GRAND_BF16;
  p->q_heads = 32;
  p->kv_heads = 8;
  p->head_dim = 128;
  p->page_size = 16;
}

grand_status grand_cache_create(const grand_cache_params *p, grand_cache **out) {
  if (!out) return GRAND_E_ARG;
  *out = nullptr;
  const char *why = nullptr;
  if (!p || p->struct_size != sizeof(grand_cache_params)) why = "struct_size does not match";
  else if (p->dtype != GRAND_BF16 && p->dtype != GRAND_F16) why = "dtype must be GRAND_BF16 or GRAND_F16";
  else if (!p->kv_heads || !p->q_heads || p->q_heads % p->kv_heads) why = "q_heads must be a multiple of kv_heads";
  else if (p->q_heads > 1024) why = "at most 1024 query heads";
  else if (!p->head_dim || p->head_dim % 8 || p->head_dim > 256) why = "head_dim must be a multiple of 8 up to 256";
  else if (!p->page_size || p->page_size > 1024 || (p->page_size & (p->page_size - 1))) why = "page_size must be a power of two up to 1024";
  if (why) {
    fprintf(stderr, "grand_cache_create: %s\n", why);
    return GRAND_E_ARG;
  }
  grand_cache *h = new (std::nothrow) grand_cache();
  if (!h) return GRAND_E_OOM;
  h->p = *p;
  h->stream = (hipStream_t)p->stream;
  while ((1u << h->shift) < p->page_size) h->shift++;
  if (hipSetDevice(p->device) != hipSuccess) {
    (void)hipGetLastError();
    delete h;
    return GRAND_E_DEVICE;
  }
  if (hipMalloc((void **)&h->err, sizeof(CacheErr)) != hipSuccess) {
    (void)hipGetLastError();
    delete h;
    return GRAND_E_OOM;
  }
  if (hipMemset(h->err, 0, sizeof(CacheErr)) != hipSuccess || hipDeviceSynchronize() != hipSuccess) {
    (void)hipGetLastError();
    (void)hipFree(h->err);
    delete h;
    return GRAND_E_DEVICE;
  }
  *out = h;
  return GRAND_OK;
}

grand_status grand_cache_destroy(grand_cache *h) {
  if (!h) return GRAND_OK;
  (void)hipSetDevice(h->p.device);
  if (!h->poisoned) (void)hipStreamSynchronize(h->stream);
  if (h->ws) (void)hipFree(h->ws);
  while (grand_cache::Kept *k = h->kept) {
    h->kept = k->next;
    (void)hipFree(k->p);
    delete k;
  }
  if (h->err) (void)hipFree(h->err);
  delete h;
  return GRAND_OK;
}

grand_status grand_cache_set_stream(grand_cache *h, void *stream) {
  TRY(check_usable(h));
  if ((hipStream_t)stream == h->stream) return GRAND_OK;
  HCHK(h, hipSetDevice(h->p.device));  // the default stream is the current GPU's
  TRY(check_no_capture(h, "grand_cache_set_stream"));
  HCHK(h, hipStreamSynchronize(h->stream));
  h->stream = (hipStream_t)stream;
  return GRAND_OK;
}

grand_status grand_cache_check(grand_cache *h) {
  TRY(check_usable(h));
  HCHK(h, hipSetDevice(h->p.device));
  TRY(check_no_capture(h, "grand_cache_check"));
  CacheErr e{};
  HCHK(h, hipMemcpyAsync(&e, h->err, sizeof e, hipMemcpyDeviceToHost, h->stream));
  HCHK(h, hipStreamSynchronize(h->stream));
  if (e.code == kCacheOk) return GRAND_OK;
  HCHK(h, hipMemsetAsync(h->err, 0, sizeof e, h->stream));
  HCHK(h, hipStreamSynchronize(h->stream));
  switch (e.code) {
    case kCachePage: return fail(h, GRAND_E_ID, "a page id of sequence %u is outside the pool", e.where);
    case kCacheId: return fail(h, GRAND_E_ID, "a slot id of sequence %u is outside the pool", e.where);
    case kCacheLen: return fail(h, GRAND_E_ARG, "the length of sequence %u is above max_k or below its chunk's", e.where);
    default: return fail(h, GRAND_E_ARG, "the chunk of sequence %u is not within n_tokens rows and max_q", e.where);
  }
}

const char *grand_cache_last_error(const grand_cache *h) { return h ? h->msg : "null handle"; }

grand_status grand_cache_append(grand_cache *h, const grand_seqs *s, const grand_rows *k, const grand_rows *v,
                                const grand_pages *pages) {
  TRY(check_usable(h));
  if (s && (s->n_seq == 0 || s->n_tokens == 0 || s->max_q == 0)) return GRAND_OK;
  HCHK(h, hipSetDevice(h->p.device));
  AppendArgs a{};
  TRY(check_seqs(h, s, true, &a.s));
  TRY(check_pages(h, pages, &a.pg));
  if (!slots_apart(h->p, a.pg)) return fail(h, GRAND_E_ARG, "slots of pages overlap");
  TRY(check_rows(h, "k", k, s->n_tokens, h->p.kv_heads, false, &a.k));
  TRY(check_rows(h, "v", v, s->n_tokens, h->p.kv_heads, false, &a.v));
  if (pages->k == pages->v && !same_rows(region(a.k, s->n_tokens, h->p.kv_heads, h->p.head_dim), region(a.v, s->n_tokens, h->p.kv_heads, h->p.head_dim)))
    return fail(h, GRAND_E_ARG, "pages.k is pages.v, but k is not v");
  if ((uint64_t)a.s.max_q * h->p.kv_heads * (h->p.head_dim / 8) >= 1ull << 31)
    return fail(h, GRAND_E_CAPACITY, "max_q is too large");
  a.kv_heads = h->p.kv_heads;
  a.dim = h->p.head_dim;
  a.err = h->err;
  HCHK(h, launch_append(a, h->stream));
  return GRAND_OK;
}

grand_status grand_cache_attend(grand_cache *h, const grand_seqs *s, const grand_rows *q, const grand_pages *pages, float scale,
                                int causal, uint32_t window, const grand_rows *out, float *lse, const grand_weights *weights_in,
                                const grand_weights *weights_out) {
  TRY(check_usable(h));
  if (s && (s->n_seq == 0 || ((s->n_tokens == 0 || s->max_q == 0) && !weights_out))) return GRAND_OK;
  HCHK(h, hipSetDevice(h->p.device));
  const grand_cache_params &p = h->p;
  AttendArgs a{};
  TRY(check_seqs(h, s, true, &a.s));
  if (!(scale > 0.f) || !isfinite(scale * kLog2e)) return fail(h, GRAND_E_ARG, "scale must be positive and finite");
  if (!weights_in != !weights_out) return fail(h, GRAND_E_ARG, "weights_in and weights_out come together");
  TRY(check_pages(h, pages, &a.pg));
  if (s->n_tokens) {
    TRY(check_rows(h, "q", q, s->n_tokens, p.q_heads, false, &a.q));
    TRY(check_rows(h, "out", out, s->n_tokens, p.q_heads, true, &a.out));
    if (lse) TRY(check_mem(h, "lse", lse, (uint64_t)s->n_tokens * p.q_heads * 4, 4));
  }
  if (s->n_tokens) {
    const Region rq = region(a.q, s->n_tokens, p.q_heads, p.head_dim), ro = region(a.out, s->n_tokens, p.q_heads, p.head_dim);
    // the weights are computed from q once out is written
    if (overlap(rq, ro) && (weights_out || !same_rows(rq, ro)))
      return fail(h, GRAND_E_ARG, same_rows(rq, ro) ? "out is q, which the weights still need" : "out overlaps q");
    TRY(check_apart(h, ro, a.pg));
  }
  if (weights_out && s->max_k) {
    TRY(check_weights(h, "weights_in", weights_in, s->n_seq, p.kv_heads, s->max_k, false, &a.win));
    TRY(check_weights(h, "weights_out", weights_out, s->n_seq, p.kv_heads, s->max_k, true, &a.wout));
    const Region ri = region(a.win, s->n_seq, p.kv_heads, s->max_k), ro = region(a.wout, s->n_seq, p.kv_heads, s->max_k);
    if (!same_rows(ri, ro) && overlap(ri, ro)) return fail(h, GRAND_E_ARG, "weights_out overlaps weights_in");
  }
  a.lse = lse;
  a.q_heads = p.q_heads;
  a.kv_heads = p.kv_heads;
  a.group = p.q_heads / p.kv_heads;
  a.dim = p.head_dim;
  a.c = scale * kLog2e;
  a.causal = causal != 0;
  a.window = window < s->max_k ? window : 0;  // a window as long as the cache hides nothing
  a.err = h->err;

  const uint64_t rows = (uint64_t)a.s.max_q * a.group;
  if (rows >= 1u << 30) return fail(h, GRAND_E_CAPACITY, "max_q is too large");
  const bool few = rows <= kFewRows;
  const uint32_t tile_rows = rows <= 16 ? 16 : few ? 32 : kManyRows;
  a.row_tiles = (uint32_t)((rows + tile_rows - 1) / tile_rows);
  // Keys a row tile sees at most, and the splits of them.  A split costs a
  // workgroup's start and end (about 6 us, behind the others' loads) and a
  // row of sums to join; too few leave the last workgroups alone.  64 single
  // tokens over 1 to 8,192 cached ones, 8 heads: 1,024 workgroups 216 us,
  // 4,096 209 us, 8,192 212 us; two over 131,072: 180, 184, 184 us.  Chunks
  // of one or two sequences fill the chip once (one of 512 over 8,192: 512
  // workgroups 91 us, 1,024 117; two 164, 171; two of up to 1,024 over up to
  // 20,000, by their lengths: 480, 555; 491, 560; 587, 552; 633, 563; 441, 398),
  // of more twice, for where their lengths differ (four of up to 512 over up to
  // 8,192: 182, 151; 204, 164; 190, 191; four of 512 over 8,192 298, 314).  Few
  // rows: up to 512 keys are one launch (a token over 300: 12.1 us, in two splits
  // 14.6); splits have 256 keys while that leaves CUs idle (a token over
  // 1,000 waited for: 29.5 us, with 512 31.5), else 512 (16,000: 37.3, 36.8).
  // (a tile's rows see up to its last token, or up to the chunk's if not causal)
  const uint64_t tokens = causal ? std::min<uint64_t>(a.s.max_q, tile_rows / a.group + 2) : a.s.max_q;
  const uint64_t span = std::min<uint64_t>(s->max_k, a.window ? (uint64_t)a.window + tokens + 31 : s->max_k);
  const uint64_t base = std::max<uint64_t>(1, (uint64_t)p.kv_heads * a.row_tiles * s->n_seq);
  const uint64_t want = ((few ? 4096 : s->n_seq <= 2 ? 512 : 1024) + base - 1) / base;
  const uint64_t least = !few || (span > 512 && base * ((span + 255) / 256) <= 256) ? 256 : 512;
  uint64_t split = std::max<uint64_t>(least, (span + want - 1) / want);
  split = (split + kKeysStep - 1) / kKeysStep * kKeysStep;
  // (31: a window's first key is rounded down to a tile; without one the last
  // split has no keys where the split length divides max_k)
  a.n_splits = (uint32_t)std::max<uint64_t>(1, (span + 31 + split - 1) / split);
  if (span <= split) a.n_splits = 1, split = span + 31;
  a.split = (uint32_t)split;
  const uint64_t groups = few ? (base * a.n_splits + 8 * p.kv_heads) : (uint64_t)p.kv_heads * a.row_tiles * a.n_splits;
  if (groups >= kMostGroups) return fail(h, GRAND_E_CAPACITY, "too many sequences, heads and new tokens for one call");
  if (weights_out && ((uint64_t)s->max_k / kAgainKeys + 1) * p.kv_heads * 32 >= kMostGroups) return fail(h, GRAND_E_CAPACITY, "max_k is too large");

  Parts w;
  const uint64_t all_rows = (uint64_t)s->n_tokens * p.q_heads;
  const int w_part = a.n_splits > 1 ? w.add(all_rows * a.n_splits * p.head_dim * 4) : -1;
  const int w_ml = a.n_splits > 1 ? w.add(all_rows * a.n_splits * 8) : -1;
  int w_lse = -1, w_scores = -1, w_sums = -1;
  a.row_splits = 1;
  if (weights_out) {
    w_lse = w.add(all_rows * 4);
    // scores of a few rows are kept (4 bytes a row and key, against half of
    // the cache to compute them again)
    const uint64_t keys = ((uint64_t)s->max_k + 31) / 32 * 32;
    const uint64_t bytes = (uint64_t)s->n_seq * p.kv_heads * rows * keys * 4;
    if (few && bytes <= 1ull << 30) {
      w_scores = w.add(bytes);
      a.score_rows = (uint32_t)rows;
    } else {
      // workgroups of 256 keys that have rows, and splits of the rows (256 at
      // least) where they are too few: six chunks of up to 614 tokens, 8 query
      // heads of 256 elements to one key/value head, over up to 1,904 cached
      // ones take 386 us with 48 workgroups, 172 with splits
      const uint64_t seen = a.window ? std::min<uint64_t>(s->max_k, (uint64_t)a.window + a.s.max_q) : s->max_k;
      const uint64_t tiles = (seen / kAgainKeys + 1) * p.kv_heads * s->n_seq;
      const uint64_t most = std::min<uint64_t>((rows + 255) / 256, std::max<uint64_t>(1, (256ull << 20) / ((uint64_t)s->n_seq * p.kv_heads * keys * 4 + 1)));
      a.row_splits = (uint32_t)std::max<uint64_t>(1, std::min<uint64_t>((1024 + tiles - 1) / tiles, std::min<uint64_t>(most, 32)));
      if (a.row_splits > 1) w_sums = w.add((uint64_t)a.row_splits * s->n_seq * p.kv_heads * keys * 4);
    }
    a.score_keys = (uint32_t)keys;
  }
  TRY(ensure_ws(h, w.total));
  if (w_part >= 0) a.part = (float *)(h->ws + w.at[w_part]);
  if (w_ml >= 0) a.part_ml = (float2 *)(h->ws + w.at[w_ml]);
  if (w_lse >= 0) a.lse2 = (float *)(h->ws + w.at[w_lse]);
  if (w_sums >= 0) a.row_sums = (float *)(h->ws + w.at[w_sums]);
  if (w_scores >= 0) a.scores = (float *)(h->ws + w.at[w_scores]);
  const bool f16 = p.dtype == GRAND_F16;
  if (s->n_tokens && s->max_q) {
    HCHK(h, launch_attend(tile_rows, f16, a, h->stream));
    if (a.n_splits > 1) HCHK(h, launch_attend_join(f16, a, tile_rows, h->stream));
  }
  if (weights_out && s->max_k) HCHK(h, launch_attend_weights(f16, a, h->stream));
  return GRAND_OK;
}

grand_status grand_cache_attend_ids(grand_cache *h, uint32_t n_seq, const grand_rows *q, const grand_pages *pages, const uint32_t *ids,
                                    uint32_t k, int64_t ids_seq_stride, int64_t ids_head_stride, float scale, const grand_rows *prior,
                                    const float *prior_lse, const grand_rows *out, float *lse) {
  TRY(check_usable(h));
  if (n_seq == 0) return GRAND_OK;
  HCHK(h, hipSetDevice(h->p.device));
  const grand_cache_params &p = h->p;
  IdsArgs a{};
  if (!(scale > 0.f) || !isfinite(scale * kLog2e)) return fail(h, GRAND_E_ARG, "scale must be positive and finite");
  if (!prior != !prior_lse) return fail(h, GRAND_E_ARG, "prior and prior_lse come together");
  if ((uint64_t)n_seq * p.q_heads >= kMostGroups) return fail(h, GRAND_E_CAPACITY, "too many sequences and heads for one call");
  if (k >= 1u << 30) return fail(h, GRAND_E_CAPACITY, "lists are too long");
  TRY(check_pages(h, pages, &a.pg));
  TRY(check_rows(h, "q", q, n_seq, p.q_heads, false, &a.q));
  TRY(check_rows(h, "out", out, n_seq, p.q_heads, true, &a.out));
  if (prior) {
    TRY(check_rows(h, "prior", prior, n_seq, p.q_heads, false, &a.prior));
    TRY(check_mem(h, "prior_lse", prior_lse, (uint64_t)n_seq * p.q_heads * 4, 4));
  }
  const Region rq = region(a.q, n_seq, p.q_heads, p.head_dim), ro = region(a.out, n_seq, p.q_heads, p.head_dim);
  if (!same_rows(rq, ro) && overlap(rq, ro)) return fail(h, GRAND_E_ARG, "out overlaps q");
  TRY(check_apart(h, ro, a.pg));
  if (prior) {
    const Region rp = region(a.prior, n_seq, p.q_heads, p.head_dim);
    if (!same_rows(rp, ro) && overlap(rp, ro)) return fail(h, GRAND_E_ARG, "out overlaps prior");
    const uint64_t bytes = (uint64_t)n_seq * p.q_heads * 4;
    if (lse && lse != prior_lse && overlap(region(lse, bytes), region(prior_lse, bytes))) return fail(h, GRAND_E_ARG, "lse overlaps prior_lse");
  }
  uint64_t e = 0;
  a.ids_seq = step(n_seq, ids_seq_stride);
  a.ids_head = step(p.q_heads, ids_head_stride);
  if (!extent(n_seq, a.ids_seq, p.q_heads, a.ids_head, 1, 0, k, &e)) return fail(h, GRAND_E_ARG, "strides of ids are negative");
  if (k) TRY(check_mem(h, "ids", ids, e * 4, 4));
  if (lse) TRY(check_mem(h, "lse", lse, (uint64_t)n_seq * p.q_heads * 4, 4));
  a.prior_lse = prior_lse;
  a.lse = lse;
  a.ids = ids;
  a.n_seq = n_seq;
  a.k = k;
  a.q_heads = p.q_heads;
  a.group = p.q_heads / p.kv_heads;
  a.dim = p.head_dim;
  a.c = scale * kLog2e;
  a.err = h->err;
  HCHK(h, launch_attend_ids(p.dtype == GRAND_F16, a, h->stream));
  return GRAND_OK;
}

grand_status grand_cache_evict(grand_cache *h, const grand_seqs *s, uint32_t heads, uint32_t cap, const grand_weights *weights,
                               const uint32_t *budget, uint32_t sinks, uint32_t recent, uint32_t *out_table,
                               const grand_weights *out_weights, uint32_t *out_lens, uint32_t *freed, uint32_t *n_freed) {
  TRY(check_usable(h));
  if (s && s->n_seq == 0) return GRAND_OK;
  HCHK(h, hipSetDevice(h->p.device));
  EvictArgs a{};
  TRY(check_seqs(h, s, false, &a.s));
  if (heads == 0 || heads > 65535) return fail(h, GRAND_E_ARG, "heads must be 1..65535");
  if (s->max_k > cap) return fail(h, GRAND_E_ARG, "max_k is above cap");
  if (cap >= 1u << 31) return fail(h, GRAND_E_CAPACITY, "cap must be below 2^31");
  if (cap) {
    TRY(check_weights(h, "weights", weights, s->n_seq, heads, cap, false, &a.win));
    TRY(check_weights(h, "out_weights", out_weights, s->n_seq, heads, cap, true, &a.wout));
  }
  TRY(check_mem(h, "budget", budget, (uint64_t)s->n_seq * 4, 4));
  const uint64_t cells = (uint64_t)s->n_seq * s->max_pages;
  if (s->max_pages) {
    TRY(check_mem(h, "out_table", out_table, cells * 4, 4));
    TRY(check_mem(h, "freed", freed, cells * 4, 4));
  }
  TRY(check_mem(h, "out_lens", out_lens, (uint64_t)s->n_seq * 4, 4));
  TRY(check_mem(h, "n_freed", n_freed, (uint64_t)s->n_seq * 4, 4));
  const Region results[] = {region(out_table, cells * 4), region(a.wout, s->n_seq, heads, cap), region(out_lens, s->n_seq * 4ull),
                            region(freed, cells * 4), region(n_freed, s->n_seq * 4ull)};
  const Region inputs[] = {{(uintptr_t)s->table, s->n_seq, 1, a.s.table_stride * 4, 0, s->max_pages * 4ull}, region(s->lens, s->n_seq * 4ull),
                           region(a.win, s->n_seq, heads, cap), region(budget, s->n_seq * 4ull)};
  for (const Region &r : results) {
    for (const Region &x : inputs)
      if (overlap(r, x)) return fail(h, GRAND_E_ARG, "a result overlaps an argument");
    for (const Region *x = results; x != &r; x++)
      if (overlap(r, *x)) return fail(h, GRAND_E_ARG, "results overlap");
  }
  Parts w;
  const int w_keys = w.add(cells * 4);
  int w_hist = -1, w_blk = -1, w_state = -1;
  if (s->max_pages > kEvictSmall) {
    w_hist = w.add((uint64_t)s->n_seq * 3 * 2048 * 4);
    w_blk = w.add((uint64_t)s->n_seq * ((s->max_pages + kEvictTile - 1) / kEvictTile) * 8);
    w_state = w.add((uint64_t)s->n_seq * 8);
  }
  TRY(ensure_ws(h, w.total));
  a.keys = (uint32_t *)(h->ws + w.at[w_keys]);
  if (w_hist >= 0) {
    a.hist = (uint32_t *)(h->ws + w.at[w_hist]);
    a.blk = (uint32_t *)(h->ws + w.at[w_blk]);
    a.state = (uint32_t *)(h->ws + w.at[w_state]);
  }
  a.quads = h->p.page_size >= 4 && (uintptr_t)a.win.p % 16 == 0 && a.win.seq % 4 == 0 && a.win.head % 4 == 0;
  a.heads = heads;
  a.page = h->p.page_size;
  a.shift = h->shift;
  a.sinks = sinks;
  a.recent = recent;
  a.budget = budget;
  a.out_table = out_table;
  a.out_table_stride = s->max_pages;
  a.out_lens = out_lens;
  a.freed = freed;
  a.freed_stride = s->max_pages;
  a.n_freed = n_freed;
  a.cap = cap;
  a.err = h->err;
  HCHK(h, launch_evict(a, h->stream));
  return GRAND_OK;
}

}  // extern "C"
