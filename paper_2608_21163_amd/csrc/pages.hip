// pages.hip -- the host side of pages that sequences share, of copies of pages
// and of rows read from packed pages: checks of arguments, workspaces and
// launches.  No call here waits for the GPU unless a workspace grows.
#include "cache_host.h"

namespace {

// Results overlap no argument and not each other.
grand_status check_results(grand_cache *h, const Region *results, size_t n, const Region *args, size_t m) {
  for (size_t i = 0; i < n; i++) {
    for (size_t j = 0; j < m; j++)
      if (overlap(results[i], args[j])) return fail(h, GRAND_E_ARG, "a result overlaps an argument");
    for (size_t j = 0; j < i; j++)
      if (overlap(results[i], results[j])) return fail(h, GRAND_E_ARG, "results overlap");
  }
  return GRAND_OK;
}

Region table_region(const SeqsView &s) { return {(uintptr_t)s.table, s.n_seq ? s.n_seq : 1, 1, s.table_stride * 4, 0, s.n_seq ? s.max_pages * 4ull : 0}; }
Region words(const void *p, uint64_t n) { return region(p, n * 4); }

grand_status check_refs(grand_cache *h, uint32_t n_pages, const uint32_t *refs_in, uint32_t *refs_out, RefArgs *a) {
  if (n_pages == 0) return fail(h, GRAND_E_ARG, "the pool has no pages");
  if ((uint64_t)n_pages << h->shift > 0xFFFFFFFFull) return fail(h, GRAND_E_CAPACITY, "a pool holds fewer than 2^32 slots");
  TRY(check_mem(h, "refs_in", refs_in, n_pages * 4ull, 4));
  TRY(check_mem(h, "refs_out", refs_out, n_pages * 4ull, 4));
  if (refs_in != refs_out && overlap(words(refs_in, n_pages), words(refs_out, n_pages))) return fail(h, GRAND_E_ARG, "refs_out overlaps refs_in");
  a->n_pages = n_pages;
  a->refs_in = refs_in;
  a->refs_out = refs_out;
  a->shift = h->shift;
  a->err = h->err;
  return GRAND_OK;
}

// Like check_seqs, but there may be no sequences.
grand_status check_table(grand_cache *h, const grand_seqs *s, SeqsView *out) {
  if (!s) return fail(h, GRAND_E_ARG, "seqs is null");
  if (s->n_seq) return check_seqs(h, s, false, out);
  *out = {};
  out->max_pages = s->max_pages;
  return GRAND_OK;
}

uint32_t blocks_of(uint32_t n_pages) { return (uint32_t)(((uint64_t)n_pages + kRefPages - 1) / kRefPages); }

grand_status copy_pages(grand_cache *h, uint32_t n, const uint32_t *src, const uint32_t *dst, CopyArgs &a) {
  TRY(check_mem(h, "src", src, n * 4ull, 4));
  TRY(check_mem(h, "dst", dst, n * 4ull, 4));
  a.src = src;
  a.dst = dst;
  a.n = n;
  a.slots = h->p.page_size;
  a.heads = h->p.kv_heads;
  a.pieces = (uint32_t)((uint64_t)a.slots * a.heads * a.row / 16);
  // rows side by side: the shorter of the two strides is a row, the longer all that the other axis holds
  const uint32_t n0 = a.pg.slot < a.pg.head ? a.slots : a.heads, s0 = std::min(a.pg.slot, a.pg.head);
  const uint32_t s1 = std::max(a.pg.slot, a.pg.head);
  a.flat = a.slots == 1 || a.heads == 1 ? a.slots * a.heads == 1 || s1 == a.row : s0 == a.row && s1 == (uint64_t)n0 * a.row;
  const uint64_t wgs = (uint64_t)n * ((2ull * a.pieces + 1023) / 1024);
  if (wgs >= kMostGroups || (uint64_t)a.slots * a.heads * a.row >= 1ull << 32) return fail(h, GRAND_E_CAPACITY, "too many or too large pages for one call");
  a.err = h->err;
  HCHK(h, launch_copy(a, h->stream));
  return GRAND_OK;
}

}  // namespace

extern "C" {

grand_status grand_packed_read(grand_cache *h, uint32_t n, const uint32_t *slots, const grand_packed *pages, const grand_rows *k,
                               const grand_rows *v) {
  TRY(check_usable(h));
  if (n == 0 || (!k && !v)) return GRAND_OK;
  HCHK(h, hipSetDevice(h->p.device));
  ReadArgs a{};
  PackedBytes bytes;
  TRY(check_packed(h, pages, &a.pg, &a.sc, &bytes));
  TRY(check_mem(h, "slots", slots, n * 4ull, 4));
  if (k) TRY(check_rows(h, "k", k, n, h->p.kv_heads, true, &a.k));
  if (v) TRY(check_rows(h, "v", v, n, h->p.kv_heads, true, &a.v));
  const Region rows[] = {region(a.k, n, h->p.kv_heads, k ? h->p.head_dim : 0), region(a.v, n, h->p.kv_heads, v ? h->p.head_dim : 0)};
  const Region args[] = {words(slots, n), region(a.pg.k, bytes.codes), region(a.pg.v, bytes.codes), region(a.sc.k, bytes.scales),
                         region(a.sc.v, bytes.scales)};
  TRY(check_results(h, rows, 2, args, 5));
  if (((uint64_t)n * h->p.kv_heads * (h->p.head_dim / 8) + 255) / 256 >= kMostGroups) return fail(h, GRAND_E_CAPACITY, "too many slots for one call");
  a.slots = slots;
  a.n = n;
  a.kv_heads = h->p.kv_heads;
  a.dim = h->p.head_dim;
  a.f16 = h->p.dtype == GRAND_F16;
  a.err = h->err;
  HCHK(h, launch_read(a, h->stream));
  return GRAND_OK;
}

grand_status grand_pages_fork(grand_cache *h, const grand_seqs *s, uint32_t n_out, const uint32_t *parents, int drop, uint32_t n_pages,
                              const uint32_t *refs_in, uint32_t *refs_out, uint32_t *out_table, uint32_t *out_lens) {
  TRY(check_usable(h));
  HCHK(h, hipSetDevice(h->p.device));
  RefArgs a{};
  TRY(check_table(h, s, &a.s));
  TRY(check_refs(h, n_pages, refs_in, refs_out, &a));
  const uint64_t cells = (uint64_t)n_out * a.s.max_pages;
  if (n_out) {
    TRY(check_mem(h, "parents", parents, n_out * 4ull, 4));
    if (cells) TRY(check_mem(h, "out_table", out_table, cells * 4, 4));
    TRY(check_mem(h, "out_lens", out_lens, n_out * 4ull, 4));
  }
  if (((uint64_t)n_out + a.s.n_seq) * (a.s.max_pages / 256 + 1) >= kMostGroups) return fail(h, GRAND_E_CAPACITY, "too many sequences and pages for one call");
  const Region results[] = {words(refs_out, n_pages), words(out_table, cells), words(out_lens, n_out)};
  const Region args[] = {table_region(a.s), words(s->lens, a.s.n_seq), words(parents, n_out), words(refs_in == refs_out ? nullptr : refs_in, refs_in == refs_out ? 0 : n_pages)};
  TRY(check_results(h, results, 3, args, 4));
  a.parents = parents;
  a.n_out = n_out;
  a.drop = drop != 0;
  a.out_table = out_table;
  a.out_lens = out_lens;
  a.out_stride = a.s.max_pages;
  HCHK(h, launch_fork(a, h->stream));
  return GRAND_OK;
}

grand_status grand_pages_grow(grand_cache *h, const grand_seqs *s, const uint32_t *n_new, uint32_t n_pages, const uint32_t *refs_in,
                              uint32_t *refs_out, uint32_t *table, uint32_t *lens, uint32_t *src, uint32_t *dst) {
  TRY(check_usable(h));
  HCHK(h, hipSetDevice(h->p.device));
  RefArgs a{};
  TRY(check_table(h, s, &a.s));
  TRY(check_refs(h, n_pages, refs_in, refs_out, &a));
  const uint32_t n_seq = a.s.n_seq;
  if (n_seq) {
    if (table != s->table || lens != s->lens) return fail(h, GRAND_E_ARG, "table and lens must be those of seqs");
    TRY(check_mem(h, "n_new", n_new, n_seq * 4ull, 4));
    TRY(check_mem(h, "src", src, n_seq * 4ull, 4));
    TRY(check_mem(h, "dst", dst, n_seq * 4ull, 4));
    const bool same = refs_in == refs_out;
    const Region results[] = {words(refs_out, n_pages), table_region(a.s), words(lens, n_seq), words(src, n_seq), words(dst, n_seq)};
    const Region args[] = {words(n_new, n_seq), words(same ? nullptr : refs_in, same ? 0 : n_pages)};
    TRY(check_results(h, results, 5, args, 2));
  }
  Parts w;
  const uint32_t blocks = blocks_of(n_pages);
  const int w_bits = w.add(blocks * (kRefPages / 8ull)), w_blk = w.add(blocks * 4ull), w_need = w.add(n_seq * 4ull), w_at = w.add(n_seq * 4ull);
  const int w_start = w.add(n_seq > kFewSeqs ? (n_seq + 1) * 4ull : 0);
  TRY(ensure_ws(h, w.total));
  a.bits = (uint64_t *)(h->ws + w.at[w_bits]);
  a.blk = (uint32_t *)(h->ws + w.at[w_blk]);
  a.need = (uint32_t *)(h->ws + w.at[w_need]);
  a.at = (uint32_t *)(h->ws + w.at[w_at]);
  a.start = (uint32_t *)(h->ws + w.at[w_start]);
  a.n_new = n_new;
  a.out_table = table;
  a.lens = lens;
  a.src = src;
  a.dst = dst;
  HCHK(h, launch_grow(a, h->stream));
  return GRAND_OK;
}

grand_status grand_pages_release(grand_cache *h, uint32_t n_rows, uint32_t width, const uint32_t *ids, int64_t row_stride,
                                 const uint32_t *counts, int tokens, uint32_t n_pages, const uint32_t *refs_in, uint32_t *refs_out,
                                 uint32_t *freed, uint32_t *n_freed) {
  TRY(check_usable(h));
  HCHK(h, hipSetDevice(h->p.device));
  RefArgs a{};
  TRY(check_refs(h, n_pages, refs_in, refs_out, &a));
  const uint64_t cells = (uint64_t)n_rows * width;
  const int64_t stride = step(n_rows, row_stride);
  uint64_t e = 0;
  if (cells) {
    if (!extent(n_rows, stride, 1, 0, 1, 0, width, &e)) return fail(h, GRAND_E_ARG, "row_stride is negative or too large");
    TRY(check_mem(h, "ids", ids, e * 4, 4));
    if (counts) TRY(check_mem(h, "counts", counts, n_rows * 4ull, 4));
  }
  if (tokens && !counts) return fail(h, GRAND_E_ARG, "tokens needs counts");
  a.cap = (uint32_t)std::min<uint64_t>(n_pages, cells);
  if (a.cap) TRY(check_mem(h, "freed", freed, a.cap * 4ull, 4));
  TRY(check_mem(h, "n_freed", n_freed, 4, 4));
  if ((uint64_t)n_rows * (width / 256 + 1) >= kMostGroups) return fail(h, GRAND_E_CAPACITY, "too many rows for one call");
  const bool same = refs_in == refs_out;
  const Region results[] = {words(refs_out, n_pages), words(freed, a.cap), words(n_freed, 1)};
  const Region args[] = {words(ids, e), words(counts, counts && cells ? n_rows : 0), words(same ? nullptr : refs_in, same ? 0 : n_pages)};
  TRY(check_results(h, results, 3, args, 3));
  Parts w;
  const uint32_t blocks = blocks_of(n_pages);
  const int w_bits = w.add(blocks * (kRefPages / 8ull)), w_blk = w.add(blocks * 4ull), w_below = w.add(blocks * (kRefPages / 8ull));
  TRY(ensure_ws(h, w.total));
  a.bits = (uint64_t *)(h->ws + w.at[w_bits]);
  a.blk = (uint32_t *)(h->ws + w.at[w_blk]);
  a.below = (uint64_t *)(h->ws + w.at[w_below]);
  a.ids = ids;
  a.counts = counts;
  a.row_stride = stride;
  a.n_rows = n_rows;
  a.width = width;
  a.tokens = tokens != 0;
  a.freed = freed;
  a.n_freed = n_freed;
  HCHK(h, launch_release(a, h->stream));
  return GRAND_OK;
}

grand_status grand_pages_compact(grand_cache *h, const grand_seqs *s, uint32_t n_pages, const uint32_t *refs_in, uint32_t *refs_out,
                                 uint32_t *out_table, uint32_t *src, uint32_t *dst, uint32_t *n_moves) {
  TRY(check_usable(h));
  HCHK(h, hipSetDevice(h->p.device));
  RefArgs a{};
  TRY(check_table(h, s, &a.s));
  TRY(check_refs(h, n_pages, refs_in, refs_out, &a));
  const uint64_t cells = (uint64_t)a.s.n_seq * a.s.max_pages;
  const bool same = refs_in == refs_out, in_place = cells && out_table == s->table;
  if (cells && !in_place) TRY(check_mem(h, "out_table", out_table, cells * 4, 4));
  TRY(check_mem(h, "src", src, n_pages * 4ull, 4));
  TRY(check_mem(h, "dst", dst, n_pages * 4ull, 4));
  TRY(check_mem(h, "n_moves", n_moves, 4, 4));
  if (((uint64_t)a.s.max_pages / 256 + 1) * a.s.n_seq + n_pages / 256 + 1 >= kMostGroups) return fail(h, GRAND_E_CAPACITY, "too many sequences and pages for one call");
  const Region table = table_region(a.s);
  const Region results[] = {words(refs_out, n_pages), in_place ? table : words(out_table, cells), words(src, n_pages), words(dst, n_pages), words(n_moves, 1)};
  const Region args[] = {in_place ? words(nullptr, 0) : table, words(s->lens, a.s.n_seq), words(same ? nullptr : refs_in, same ? 0 : n_pages)};
  TRY(check_results(h, results, 5, args, 3));
  Parts w;
  const uint32_t blocks = blocks_of(n_pages);
  const int w_bits = w.add(blocks * (kRefPages / 8ull)), w_blk = w.add(blocks * 4ull), w_rank = w.add(n_pages * 4ull), w_total = w.add(4);
  TRY(ensure_ws(h, w.total));
  a.bits = (uint64_t *)(h->ws + w.at[w_bits]);
  a.blk = (uint32_t *)(h->ws + w.at[w_blk]);
  a.rank = (uint32_t *)(h->ws + w.at[w_rank]);
  a.total = (uint32_t *)(h->ws + w.at[w_total]);
  a.out_table = out_table;
  a.out_stride = in_place ? a.s.table_stride : a.s.max_pages;
  a.src = src;
  a.dst = dst;
  a.n_freed = n_moves;
  HCHK(h, launch_compact(a, h->stream));
  return GRAND_OK;
}

grand_status grand_pages_copy(grand_cache *h, uint32_t n, const uint32_t *src, const uint32_t *dst, const grand_pages *pages) {
  TRY(check_usable(h));
  if (n == 0) return GRAND_OK;
  HCHK(h, hipSetDevice(h->p.device));
  CopyArgs a{};
  TRY(check_pages(h, pages, &a.pg));
  TRY(check_pages_apart(h, a.pg));
  a.row = h->p.head_dim * 2;
  return copy_pages(h, n, src, dst, a);
}

grand_status grand_packed_copy(grand_cache *h, uint32_t n, const uint32_t *src, const uint32_t *dst, const grand_packed *pages) {
  TRY(check_usable(h));
  if (n == 0) return GRAND_OK;
  HCHK(h, hipSetDevice(h->p.device));
  CopyArgs a{};
  PackedBytes bytes;
  TRY(check_packed(h, pages, &a.pg, &a.sc, &bytes));
  TRY(check_packed_apart(h, a.pg, a.sc));
  const uint32_t blocks = (h->p.head_dim + 31) / 32;
  a.row = blocks * 16;
  a.scale_row = blocks;
  return copy_pages(h, n, src, dst, a);
}

}  // extern "C"
