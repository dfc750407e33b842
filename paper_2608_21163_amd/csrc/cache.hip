// cache.hip -- the host side of the key/value-cache operators: checks of
// arguments, plans and launches.  No call here waits for the GPU unless a
// workspace grows.
#include "cache_host.h"

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
    case kCacheParent: return fail(h, GRAND_E_ARG, "the parent of sequence %u is no row of the table", e.where);
    case kCacheFull: return fail(h, GRAND_E_CAPACITY, "the pool has no pages left for sequence %u", e.where);
    case kCacheRefs: return fail(h, GRAND_E_ARG, "more names of page %u than its count says", e.where);
    case kCacheList: return fail(h, GRAND_E_ID, "entry %u of a list is outside the pool", e.where);
    default: return fail(h, GRAND_E_ARG, "the chunk of sequence %u is not within n_tokens rows and max_q", e.where);
  }
}

const char *grand_cache_last_error(const grand_cache *h) { return h ? h->msg : "null handle"; }

static grand_status append(grand_cache *h, const grand_seqs *s, const grand_rows *k, const grand_rows *v, const grand_pages *pages,
                           const grand_packed *packed, bool is_packed) {
  TRY(check_usable(h));
  if (s && (s->n_seq == 0 || s->n_tokens == 0 || s->max_q == 0)) return GRAND_OK;
  HCHK(h, hipSetDevice(h->p.device));
  AppendArgs a{};
  TRY(check_seqs(h, s, true, &a.s));
  if (is_packed) {
    PackedBytes bytes;
    TRY(check_packed(h, packed, &a.pg, &a.sc, &bytes));
    TRY(check_packed_apart(h, a.pg, a.sc));
  } else {
    TRY(check_pages(h, pages, &a.pg));
    TRY(check_pages_apart(h, a.pg));
  }
  TRY(check_rows(h, "k", k, s->n_tokens, h->p.kv_heads, false, &a.k));
  TRY(check_rows(h, "v", v, s->n_tokens, h->p.kv_heads, false, &a.v));
  if (a.pg.k == a.pg.v && !same_rows(region(a.k, s->n_tokens, h->p.kv_heads, h->p.head_dim), region(a.v, s->n_tokens, h->p.kv_heads, h->p.head_dim)))
    return fail(h, GRAND_E_ARG, "pages.k is pages.v, but k is not v");
  const uint64_t pieces = is_packed ? (h->p.head_dim + 31) / 32 * 4 : h->p.head_dim / 8;
  if ((uint64_t)a.s.max_q * h->p.kv_heads * pieces >= 1ull << 31)
    return fail(h, GRAND_E_CAPACITY, "max_q is too large");
  a.kv_heads = h->p.kv_heads;
  a.dim = h->p.head_dim;
  a.f16 = h->p.dtype == GRAND_F16;
  a.err = h->err;
  HCHK(h, launch_append(a, h->stream));
  return GRAND_OK;
}

grand_status grand_cache_append(grand_cache *h, const grand_seqs *s, const grand_rows *k, const grand_rows *v, const grand_pages *pages) {
  return append(h, s, k, v, pages, nullptr, false);
}

grand_status grand_cache_append_packed(grand_cache *h, const grand_seqs *s, const grand_rows *k, const grand_rows *v,
                                       const grand_packed *pages) {
  return append(h, s, k, v, nullptr, pages, true);
}

static grand_status attend(grand_cache *h, const grand_seqs *s, const grand_rows *q, const grand_pages *pages, const grand_packed *packed,
                           bool is_packed, float scale, int causal, uint32_t window, uint32_t sinks, const grand_rows *out, float *lse,
                           const grand_weights *weights_in, const grand_weights *weights_out) {
  TRY(check_usable(h));
  if (s && (s->n_seq == 0 || ((s->n_tokens == 0 || s->max_q == 0) && !weights_out))) return GRAND_OK;
  HCHK(h, hipSetDevice(h->p.device));
  const grand_cache_params &p = h->p;
  AttendArgs a{};
  TRY(check_seqs(h, s, true, &a.s));
  if (!(scale > 0.f) || !isfinite(scale * kLog2e)) return fail(h, GRAND_E_ARG, "scale must be positive and finite");
  if (!weights_in != !weights_out) return fail(h, GRAND_E_ARG, "weights_in and weights_out come together");
  PackedBytes bytes{};
  if (is_packed) TRY(check_packed(h, packed, &a.pg, &a.sc, &bytes));
  else TRY(check_pages(h, pages, &a.pg));
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
    TRY(check_apart(h, ro, a.pg, a.sc, bytes.scales));
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
  // a window as long as the cache, or that reaches the first tokens that stay, hides nothing
  a.window = (uint64_t)window + sinks < s->max_k ? window : 0;
  a.sinks = a.window ? sinks : 0;
  a.err = h->err;

  const uint64_t rows = (uint64_t)a.s.max_q * a.group;
  if (rows >= 1u << 30) return fail(h, GRAND_E_CAPACITY, "max_q is too large");
  const bool few = rows <= kFewRows;
  const uint32_t tile_rows = rows <= 16 ? 16 : few ? 32 : kManyRows;
  a.row_tiles = (uint32_t)((rows + tile_rows - 1) / tile_rows);
  const uint32_t tile_keys = few ? 32 : rows_tile(p.head_dim);
  a.sink_keys = (a.sinks + tile_keys - 1) / tile_keys * tile_keys;
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
  const uint64_t span = std::min<uint64_t>(s->max_k, a.window ? (uint64_t)a.window + tokens + 31 + a.sink_keys : s->max_k);
  const uint64_t base = std::max<uint64_t>(1, (uint64_t)p.kv_heads * a.row_tiles * s->n_seq);
  const uint64_t want = ((few ? 4096 : s->n_seq <= 2 ? 512 : 1024) + base - 1) / base;
  const uint64_t least = !few || (span > 512 && base * ((span + 255) / 256) <= 256) ? 256 : 512;
  uint64_t split = std::max<uint64_t>(least, (span + want - 1) / want);
  split = (split + kKeysStep - 1) / kKeysStep * kKeysStep;
  // (31: a window's first key is rounded down to a tile; without one the last
  // split has no keys where the split length divides max_k)
  a.n_splits = (uint32_t)std::max<uint64_t>(1, (span + 31 + split - 1) / split);
  // (beside first tokens every long sequence's window is as long: one workgroup each as soon
  // as that is one a CU.  Windows of 1,024, 8 heads, 16, 32, 48, 64 and 96 single tokens:
  // 18.6 us, 23.5, 38.2, 45.6, 66.7; split 17.0, 26.8, 39.9, 51.2, 73.9.  Long windows
  // gain little, 64 of 4,000 143 and 151 us, and where few sequences reach them they are split)
  if (span <= split || (a.sinks && !is_packed && few && base >= 256 && span <= 2048)) a.n_splits = 1, split = span + 31;
  a.split = (uint32_t)split;
  // Packed pages, few rows: equal shares of all sequences' keys that fill the chip
  // once, not splits of each (64 single tokens over up to 8,192: 70 us, splits of 1,024
  // keys 81).  Up to 512 keys are one launch without parts; every workgroup
  // adds up all lengths, 64 at a time.  Three workgroups a CU rather than two where registers
  // allow it (64 over up to 1,024: 23.5 us, 26.6; 256: 55, 60; 96 elements 69, 75), but two for long
  // shares of slots of all heads whose runs lie in a page (64 over 4,096 and 8,192: 65.4 us, 141,
  // three 73, 152; over up to 8,192 83.5, 86; up to 4,096 43.3, 41.5; but pages of eight and
  // rows of 96 elements over up to 8,192 126 and 107, three 103.5 and 89).
  if (is_packed && few && span > 512 && s->n_seq <= 1024 && s->n_seq * (span / kKeysStep + 2) < 1u << 31) {
    uint32_t groups_of_cu = packed_groups(packed_row(p.head_dim), tile_rows / 16);
    const bool beside = a.pg.slot == (p.head_dim + 31) / 32 * 16;  // a head's slots
    if (!beside && groups_of_cu == 3 && p.head_dim > 64 && packed_wide(a) && s->n_seq * span * p.kv_heads > 2048 * 512) groups_of_cu = 2;
    a.units = std::max(1u, 256 * groups_of_cu / p.kv_heads);
  }
  const uint64_t groups = few ? ((a.units ? (uint64_t)p.kv_heads * a.units : base * a.n_splits) + 8 * p.kv_heads) : (uint64_t)p.kv_heads * a.row_tiles * a.n_splits;
  if (groups >= kMostGroups) return fail(h, GRAND_E_CAPACITY, "too many sequences, heads and new tokens for one call");
  if (weights_out && ((uint64_t)s->max_k / kAgainKeys + 1) * p.kv_heads * 32 >= kMostGroups) return fail(h, GRAND_E_CAPACITY, "max_k is too large");

  Parts w;
  const uint64_t all_rows = (uint64_t)s->n_tokens * p.q_heads;
  const uint64_t parts = a.units ? 2ull * a.units * p.kv_heads * tile_rows : a.n_splits > 1 ? all_rows * a.n_splits : 0;
  const int w_part = parts ? w.add(parts * p.head_dim * 4) : -1, w_ml = parts ? w.add(parts * 8) : -1;
  int w_lse = -1, w_scores = -1, w_sums = -1;
  a.row_splits = 1;
  if (weights_out && s->max_k) {
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
      a.sum_keys = again_tiles(a) * kAgainKeys;
      const uint64_t tiles = (uint64_t)again_tiles(a) * p.kv_heads * s->n_seq, sums = (uint64_t)s->n_seq * p.kv_heads * a.sum_keys * 4;
      const uint64_t most = std::min<uint64_t>((rows + 255) / 256, std::max<uint64_t>(1, (256ull << 20) / sums));
      a.row_splits = (uint32_t)std::max<uint64_t>(1, std::min<uint64_t>((1024 + tiles - 1) / tiles, std::min<uint64_t>(most, 32)));
      if (a.row_splits > 1 || a.window) w_sums = w.add(a.row_splits * sums);
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
    if (parts) HCHK(h, launch_attend_join(f16, a, tile_rows, h->stream));
  }
  if (weights_out && s->max_k) HCHK(h, launch_attend_weights(f16, a, h->stream));
  return GRAND_OK;
}

grand_status grand_cache_attend(grand_cache *h, const grand_seqs *s, const grand_rows *q, const grand_pages *pages, float scale,
                                int causal, uint32_t window, const grand_rows *out, float *lse, const grand_weights *weights_in,
                                const grand_weights *weights_out) {
  return attend(h, s, q, pages, nullptr, false, scale, causal, window, 0, out, lse, weights_in, weights_out);
}

grand_status grand_cache_attend_sinks(grand_cache *h, const grand_seqs *s, const grand_rows *q, const grand_pages *pages, float scale,
                                      int causal, uint32_t window, uint32_t sinks, const grand_rows *out, float *lse,
                                      const grand_weights *weights_in, const grand_weights *weights_out) {
  return attend(h, s, q, pages, nullptr, false, scale, causal, window, sinks, out, lse, weights_in, weights_out);
}

grand_status grand_cache_attend_packed(grand_cache *h, const grand_seqs *s, const grand_rows *q, const grand_packed *pages, float scale,
                                       int causal, uint32_t window, uint32_t sinks, const grand_rows *out, float *lse,
                                       const grand_weights *weights_in, const grand_weights *weights_out) {
  return attend(h, s, q, nullptr, pages, true, scale, causal, window, sinks, out, lse, weights_in, weights_out);
}

static grand_status attend_ids(grand_cache *h, uint32_t n_seq, const grand_rows *q, const grand_pages *pages, const grand_packed *packed,
                               bool is_packed, const uint32_t *ids, uint32_t k, int64_t ids_seq_stride, int64_t ids_head_stride, float scale,
                               const grand_rows *prior, const float *prior_lse, const grand_rows *out, float *lse) {
  TRY(check_usable(h));
  if (n_seq == 0) return GRAND_OK;
  HCHK(h, hipSetDevice(h->p.device));
  const grand_cache_params &p = h->p;
  IdsArgs a{};
  if (!(scale > 0.f) || !isfinite(scale * kLog2e)) return fail(h, GRAND_E_ARG, "scale must be positive and finite");
  if (!prior != !prior_lse) return fail(h, GRAND_E_ARG, "prior and prior_lse come together");
  if ((uint64_t)n_seq * p.q_heads >= kMostGroups) return fail(h, GRAND_E_CAPACITY, "too many sequences and heads for one call");
  if (k >= 1u << 30) return fail(h, GRAND_E_CAPACITY, "lists are too long");
  PackedBytes bytes{};
  if (is_packed) TRY(check_packed(h, packed, &a.pg, &a.sc, &bytes));
  else TRY(check_pages(h, pages, &a.pg));
  TRY(check_rows(h, "q", q, n_seq, p.q_heads, false, &a.q));
  TRY(check_rows(h, "out", out, n_seq, p.q_heads, true, &a.out));
  if (prior) {
    TRY(check_rows(h, "prior", prior, n_seq, p.q_heads, false, &a.prior));
    TRY(check_mem(h, "prior_lse", prior_lse, (uint64_t)n_seq * p.q_heads * 4, 4));
  }
  const Region rq = region(a.q, n_seq, p.q_heads, p.head_dim), ro = region(a.out, n_seq, p.q_heads, p.head_dim);
  if (!same_rows(rq, ro) && overlap(rq, ro)) return fail(h, GRAND_E_ARG, "out overlaps q");
  TRY(check_apart(h, ro, a.pg, a.sc, bytes.scales));
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

grand_status grand_cache_attend_ids(grand_cache *h, uint32_t n_seq, const grand_rows *q, const grand_pages *pages, const uint32_t *ids,
                                    uint32_t k, int64_t ids_seq_stride, int64_t ids_head_stride, float scale, const grand_rows *prior,
                                    const float *prior_lse, const grand_rows *out, float *lse) {
  return attend_ids(h, n_seq, q, pages, nullptr, false, ids, k, ids_seq_stride, ids_head_stride, scale, prior, prior_lse, out, lse);
}

grand_status grand_cache_attend_ids_packed(grand_cache *h, uint32_t n_seq, const grand_rows *q, const grand_packed *pages,
                                           const uint32_t *ids, uint32_t k, int64_t ids_seq_stride, int64_t ids_head_stride, float scale,
                                           const grand_rows *prior, const float *prior_lse, const grand_rows *out, float *lse) {
  return attend_ids(h, n_seq, q, nullptr, pages, true, ids, k, ids_seq_stride, ids_head_stride, scale, prior, prior_lse, out, lse);
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
