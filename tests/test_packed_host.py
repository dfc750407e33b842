"""The host side of packed pages, of first tokens and of shared pages without a
GPU (as test_cache_host.py): what is refused, and what is not."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

from conftest import ROOT
from paper_2608_21163_amd import grand
from paper_2608_21163_amd.build import CSRC, HIPCC
from test_cache_host import Host, P, moved


@pytest.fixture(scope="module")
def built(tmp_path_factory):
    d = tmp_path_factory.mktemp("host")
    objects = []
    for src in (os.path.join(CSRC, "cache.hip"), os.path.join(CSRC, "pages.hip"), os.path.join(ROOT, "tests", "fake_hip.cpp"),
                os.path.join(ROOT, "tests", "fake_pages.cpp")):
        objects.append(str(d / os.path.basename(src)) + ".o")
        subprocess.check_call([HIPCC, "-x", "hip", "--offload-arch=gfx950", "--offload-host-only", "-O1", "-std=c++17", "-fPIC",
                               "-I", CSRC, "-I", os.path.join(ROOT, "include"), "-c", src, "-o", objects[-1]])
    out = str(d / "libhost.so")
    subprocess.check_call(["g++", "-shared", "-Wl,-Bsymbolic", "-o", out, *objects])
    lib = ctypes.CDLL(out)
    for name in grand.EXPORTED:
        if name.startswith(("grand_cache_", "grand_pages_", "grand_packed_")) and name != "grand_cache_last_error":
            getattr(lib, name).argtypes = getattr(grand.load_library(), name).argtypes
    lib.grand_cache_last_error.argtypes, lib.grand_cache_last_error.restype = [P], ctypes.c_char_p
    lib.fake_memory.argtypes, lib.fake_memory.restype = [ctypes.c_size_t, ctypes.c_int], ctypes.c_size_t
    lib.fake_log.restype = ctypes.c_char_p
    lib.fake_capture.argtypes = [ctypes.c_int, P]
    return lib


OK, ARG, CAPACITY = grand.OK, grand.E_ARG, grand.E_CAPACITY


class More(Host):
    """Pools held in 4 bits: 8 pages of 16 slots, 2 heads of 64 elements (32
    bytes of codes, 2 scales a row)."""

    def packed(self, n=8, **kw):
        blocks = -(-self.p.head_dim // 32)
        row, slots, heads = 16 * blocks, self.p.page_size, self.p.kv_heads
        size = n * slots * heads
        g = dict(k=self.memory(size * row), v=self.memory(size * row), k_scales=self.memory(size * blocks), v_scales=self.memory(size * blocks),
                 n_pages=n, page_stride=slots * heads * row, slot_stride=heads * row, head_stride=row, scale_page_stride=slots * heads * blocks,
                 scale_slot_stride=heads * blocks, scale_head_stride=blocks)
        g.update(kw)
        return grand.PackedPages(*[g[f] for f, _ in grand.PackedPages._fields_])

    def attend_packed(self, s, q, pages, out, window=0, sinks=0, wi=None, wo=None):
        r = [None if x is None else ctypes.byref(x) for x in (s, q, pages, out, wi, wo)]
        return self.lib.grand_cache_attend_packed(self.h, r[0], r[1], r[2], 0.125, 1, window, sinks, r[3], None, r[4], r[5])

    def append_packed(self, s, k, v, pages):
        return self.lib.grand_cache_append_packed(self.h, *[ctypes.byref(x) for x in (s, k, v, pages)])


def changed(x, **kw):
    return type(x)(*[kw.get(f, getattr(x, f)) for f, _ in x._fields_])


def test_struct_layout(tmp_path):
    fields = [f for f, _ in grand.PackedPages._fields_]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(["#include <stddef.h>", "#include <stdio.h>", f'#include "{ROOT}/include/grand.h"', "int main(void) {",
                              'printf("%zu\\n", sizeof(grand_packed));', *[f'printf("%zu\\n", offsetof(grand_packed, {f}));' for f in fields],
                              "return 0; }"]))
    subprocess.check_call(["gcc", "-std=c11", str(src), "-o", str(exe)])
    want = [ctypes.sizeof(grand.PackedPages)] + [getattr(grand.PackedPages, f).offset for f in fields]
    assert [int(x) for x in subprocess.check_output([str(exe)]).split()] == want


def test_null_handles():
    lib = grand.load_library()
    assert lib.grand_cache_append_packed(None, None, None, None, None) == ARG
    assert lib.grand_cache_attend_sinks(None, None, None, None, 1.0, 1, 0, 0, None, None, None, None) == ARG
    assert lib.grand_cache_attend_packed(None, None, None, None, 1.0, 1, 0, 0, None, None, None, None) == ARG
    assert lib.grand_cache_attend_ids_packed(None, 1, None, None, None, 1, 0, 0, 1.0, None, None, None, None) == ARG
    assert lib.grand_packed_read(None, 1, None, None, None, None) == ARG
    assert lib.grand_packed_copy(None, 1, None, None, None) == lib.grand_pages_copy(None, 1, None, None, None) == ARG
    assert lib.grand_pages_fork(None, None, 1, None, 0, 1, None, None, None, None) == ARG
    assert lib.grand_pages_grow(None, None, None, 1, None, None, None, None, None, None) == ARG
    assert lib.grand_pages_release(None, 1, 1, None, 1, None, 0, 1, None, None, None, None) == ARG
    assert lib.grand_pages_compact(None, None, 1, None, None, None, None, None, None) == ARG


def test_packed_pages(built):
    """Extents, alignment and strides of codes and scales."""
    c = More(built)
    s, q, out, g = c.seqs(), c.rows(), c.rows(), c.packed()
    assert c.attend_packed(s, q, g, out) == OK, c.error()
    for kw, want in ((dict(k=None), ARG), (dict(k_scales=None), ARG), (dict(k=g.k + 8), ARG), (dict(v=g.v + 16), OK), (dict(v=g.v + 512), ARG),
                     (dict(v_scales=g.v_scales + 1), OK), (dict(v_scales=g.v_scales + 400), ARG), (dict(slot_stride=72), ARG),
                     (dict(page_stride=-1024), ARG), (dict(scale_slot_stride=-4), ARG), (dict(scale_slot_stride=3), OK), (dict(n_pages=0), ARG),
                     (dict(n_pages=9), ARG), (dict(n_pages=1 << 28), CAPACITY), (dict(page_stride=1 << 33), CAPACITY),
                     (dict(slot_stride=1 << 30), CAPACITY), (dict(scale_page_stride=1 << 32), CAPACITY)):
        assert c.attend_packed(s, q, changed(g, **kw), out) == want, (kw, c.error())
    assert c.attend_packed(s, q, None, out) == ARG
    one = More(built, page_size=1, kv_heads=1, q_heads=1)          # strides along axes of one say nothing
    g = one.packed(1, page_stride=3, slot_stride=-1, head_stride=1 << 40, scale_page_stride=-3, scale_slot_stride=-1, scale_head_stride=-1)
    assert one.attend_packed(one.seqs(1, max_k=1), one.rows(1), g, one.rows(1)) == OK, one.error()
    odd = More(built, head_dim=72)                                  # three blocks, the last of 8 elements
    assert odd.attend_packed(odd.seqs(), odd.rows(), odd.packed(), odd.rows()) == OK, odd.error()


def test_packed_results_apart(built):
    c = More(built)
    s, q, g = c.seqs(), c.rows(), c.packed(32)
    d = 64
    for at in (g.k, g.v, g.v + 64, g.k_scales, g.v_scales):
        assert c.attend_packed(s, q, g, grand.Rows(at, 4 * d, d)) == ARG and "pages" in c.error()
    assert c.attend_packed(s, q, g, q) == OK and c.attend_packed(s, q, g, moved(q, 8)) == ARG
    ids = c.memory(2 * 4 * 3 * 4)

    def listed(out, pages=g):
        r = [ctypes.byref(x) for x in (q, pages, out)]
        return built.grand_cache_attend_ids_packed(c.h, 2, r[0], r[1], ids, 3, 12, 3, 0.5, None, None, r[2], None)
    assert listed(c.rows()) == listed(q) == OK
    assert listed(grand.Rows(g.v, 4 * d, d)) == listed(grand.Rows(g.k_scales, 4 * d, d)) == ARG
    assert listed(c.rows(), changed(g, k=g.k + 4)) == ARG
    k, v, slots = c.rows(2, 2), c.rows(2, 2), c.memory(8)

    def read(k, v, slots=slots):
        r = [None if x is None else ctypes.byref(x) for x in (g, k, v)]
        return built.grand_packed_read(c.h, 2, slots, *r)
    assert read(k, v) == read(k, None) == read(None, v) == read(None, None) == OK
    assert read(k, k) == read(grand.Rows(g.k, 128, 64), v) == read(k, grand.Rows(g.v_scales, 128, 64)) == read(k, v, None) == ARG
    assert read(k, changed(v, token_stride=64)) == ARG              # rows that overlap
    assert read(grand.Rows(slots & ~15, 128, 64), v) == ARG


def test_packed_rows_apart(built):
    """Pools that are written: no row of codes or scales inside another; one
    buffer may hold all four."""
    c = More(built)
    s, k, v, g = c.seqs(), c.rows(heads=2), c.rows(heads=2), c.packed()
    assert c.append_packed(s, k, v, g) == OK
    for kw in (dict(slot_stride=0), dict(page_stride=0), dict(head_stride=16), dict(slot_stride=32), dict(scale_slot_stride=0),
               dict(scale_head_stride=1), dict(scale_page_stride=60), dict(v=g.k + 32), dict(v_scales=g.k_scales), dict(k_scales=g.v + 64),
               dict(v=g.k)):
        shared = changed(g, **kw)
        if "v" in kw and kw["v"] == g.k:
            assert c.append_packed(s, k, v, shared) == ARG
            assert c.append_packed(s, k, k, shared) == ARG          # the scales still differ
            assert c.append_packed(s, k, k, changed(shared, v_scales=g.k_scales)) == OK
            assert c.append_packed(s, k, v, changed(shared, v_scales=g.k_scales)) == ARG
            continue
        assert c.attend_packed(c.seqs(), c.rows(), shared, c.rows()) == OK, kw
        assert c.append_packed(s, k, v, shared) == ARG and "overlap" in c.error(), kw
    # rows of 48 bytes: codes, then scales of keys, then those of values; values' codes behind all keys
    at = c.memory(2 * 8 * 16 * 2 * 48)
    strides = dict(page_stride=16 * 2 * 48, slot_stride=2 * 48, head_stride=48, scale_page_stride=16 * 2 * 48, scale_slot_stride=2 * 48,
                   scale_head_stride=48)
    one = c.packed(k=at, v=at + 8 * 16 * 2 * 48, k_scales=at + 32, v_scales=at + 8 * 16 * 2 * 48 + 32, **strides)
    assert c.append_packed(s, k, v, one) == OK, c.error()
    assert c.append_packed(s, k, v, changed(one, v_scales=at + 34)) == OK
    assert c.append_packed(s, k, v, changed(one, v_scales=at + 33)) == ARG
    assert c.append_packed(s, k, v, changed(one, k_scales=at + 31)) == ARG
    assert c.append_packed(s, k, v, changed(one, k_scales=at + 47)) == ARG
    # pages whose keys and values alternate
    both = dict(page_stride=2 * 1024, slot_stride=64, head_stride=32)
    at = c.memory(2 * 8 * 1024)
    assert c.append_packed(s, k, v, c.packed(k=at, v=at + 1024, **both)) == OK, c.error()
    assert c.append_packed(s, k, v, c.packed(k=at, v=at + 1008, **both)) == ARG
    src, dst = c.memory(12), c.memory(12)
    assert built.grand_packed_copy(c.h, 3, src, dst, ctypes.byref(g)) == OK
    assert built.grand_packed_copy(c.h, 3, src, dst, ctypes.byref(changed(g, v=g.k + 32))) == ARG
    assert built.grand_packed_copy(c.h, 3, src, None, ctypes.byref(g)) == ARG


def test_first_tokens(built):
    c = More(built)
    s, q, out, pages, g = c.seqs(max_k=300), c.rows(), c.rows(), c.pages(32), c.packed(32)
    for window, sinks in ((0, 4), (10, 4), (10, 1 << 31), (0xFFFFFFFF, 0xFFFFFFFF), (299, 1), (1, 0)):
        r = [ctypes.byref(x) for x in (s, q, pages, out)]
        assert built.grand_cache_attend_sinks(c.h, *r[:3], 0.125, 1, window, sinks, r[3], None, None, None) == OK, c.error()
        assert c.attend_packed(s, q, g, out, window, sinks) == OK
    big = More(built, page_size=1024)
    s = big.seqs(1, max_q=1, max_k=(1 << 31) - 65)
    assert big.attend_packed(s, big.rows(1), big.packed(2), big.rows(1), (1 << 31) - 100_000, 99_000) == OK, big.error()


def pages_args(c, n_seq=3, n_pages=40):
    """Arguments of the shared-page calls: rows of 5 pages."""
    m = lambda n: c.memory(4 * n)
    s = grand.Seqs(n_seq, 0, 0, 80, m(5 * n_seq), 5, 5, None, m(n_seq))
    return s, dict(refs=m(n_pages), out=m(n_pages), table=m(40), lens=m(8), a=m(n_pages), b=m(n_pages), one=m(1), given=m(8))


def test_forks(built):
    c = More(built)
    s, m = pages_args(c)

    def fork(s=s, n=8, parents=m["given"], pages=40, refs=m["refs"], out=m["out"], table=m["table"], lens=m["lens"]):
        return built.grand_pages_fork(c.h, ctypes.byref(s) if s else None, n, parents, 1, pages, refs, out, table, lens)
    assert fork() == fork(out=m["refs"]) == fork(n=0, parents=None, table=None, lens=None) == OK, c.error()
    none = grand.Seqs(0, 0, 0, 0, None, 0, 0, None, None)
    assert fork(none) == OK, c.error()
    for kw in (dict(s=None), dict(pages=0), dict(refs=None), dict(out=None), dict(parents=None), dict(table=None), dict(lens=None), dict(n=1000),
               dict(pages=400), dict(out=m["refs"] + 4), dict(table=s.table), dict(lens=s.lens), dict(lens=m["given"]), dict(table=m["out"]),
               dict(table=m["refs"]), dict(lens=m["table"] + 8)):
        assert fork(**kw) == ARG, (kw, c.error())
    assert fork(pages=1 << 29) == CAPACITY


def test_growth(built):
    c = More(built)
    s, m = pages_args(c)

    def grow(s=s, new=m["given"], pages=40, refs=m["refs"], out=m["out"], table=None, lens=None, src=m["a"], dst=m["b"]):
        return built.grand_pages_grow(c.h, ctypes.byref(s) if s else None, new, pages, refs, out, table or s.table, lens or s.lens, src, dst)
    assert grow() == grow(out=m["refs"]) == OK, c.error()
    assert grow(grand.Seqs(0, 0, 0, 0, None, 0, 0, None, None), None, src=None, dst=None) == OK
    for kw in (dict(new=None), dict(src=None), dict(table=m["table"]), dict(lens=m["lens"]), dict(new=s.lens), dict(src=s.table), dict(dst=m["a"]),
               dict(out=s.table), dict(src=m["refs"]), dict(src=m["given"]), dict(pages=0), dict(out=m["refs"] + 8)):
        assert grow(**kw) == ARG, (kw, c.error())
    shared = changed(s, table_stride=4)
    assert grow(shared) == ARG
    # the workspace may not grow during a capture, and may be used in one
    built.fake_capture(1, None)
    c2 = More(built)
    s2, m = pages_args(c2)
    built.fake_capture(1, None)
    call = lambda: built.grand_pages_grow(c2.h, ctypes.byref(s2), m["given"], 40, m["refs"], m["out"], s2.table, s2.lens, m["a"], m["b"])
    assert call() == CAPACITY and "capture" in c2.error()
    built.fake_capture(0, None)
    assert call() == OK
    built.fake_capture(1, None)
    assert call() == OK
    built.fake_capture(0, None)


def test_releases(built):
    c = More(built)
    _, m = pages_args(c)
    ids = c.memory(4 * 3 * 10)

    def release(rows=3, width=5, ids=ids, stride=10, counts=m["given"], tokens=0, pages=40, refs=m["refs"], out=m["out"], freed=m["a"], n=m["one"]):
        return built.grand_pages_release(c.h, rows, width, ids, stride, counts, tokens, pages, refs, out, freed, n)
    assert release() == release(out=m["refs"]) == release(counts=None) == release(tokens=1) == release(stride=0) == OK, c.error()
    assert release(rows=0, ids=None, counts=None, freed=None) == OK, c.error()
    for kw in (dict(ids=None), dict(stride=-1), dict(stride=200), dict(counts=None, tokens=1), dict(freed=None), dict(n=None), dict(freed=ids),
               dict(n=m["given"]), dict(freed=m["out"]), dict(n=m["a"]), dict(freed=m["refs"]), dict(out=ids), dict(pages=0)):
        assert release(**kw) == ARG, (kw, c.error())


def test_compactions(built):
    c = More(built)
    s, m = pages_args(c)

    def compact(s=s, pages=40, refs=m["refs"], out=m["out"], table=m["table"], src=m["a"], dst=m["b"], n=m["one"]):
        return built.grand_pages_compact(c.h, ctypes.byref(s) if s else None, pages, refs, out, table, src, dst, n)
    assert compact() == compact(out=m["refs"]) == compact(table=s.table) == OK, c.error()
    assert compact(grand.Seqs(0, 0, 0, 0, None, 0, 0, None, None), table=None) == OK, c.error()
    for kw in (dict(s=None), dict(table=None), dict(src=None), dict(n=None), dict(table=s.table + 4), dict(src=s.table), dict(dst=m["a"]), dict(n=m["b"]),
               dict(src=s.lens), dict(dst=m["refs"]), dict(out=s.table), dict(pages=0), dict(pages=400)):
        assert compact(**kw) == ARG, (kw, c.error())


def test_copies(built):
    """Pages whose rows lie side by side are copied as one piece, in either order of their axes."""
    c = More(built)
    g, src, dst = c.pages(), c.memory(40), c.memory(40)

    def copy(g, n=10, src=src, dst=dst):
        return built.grand_pages_copy(c.h, n, src, dst, ctypes.byref(g))
    assert copy(g) == OK and built.fake_copy_flat() == 1
    assert copy(changed(g, slot_stride=64, head_stride=16 * 64)) == OK and built.fake_copy_flat() == 1
    wide = grand.Pages(c.memory(8 * 16 * 3 * 64 * 2), c.memory(8 * 16 * 3 * 64 * 2), 8, 16 * 3 * 64, 3 * 64, 64)
    assert copy(wide) == OK and built.fake_copy_flat() == 0
    assert copy(g, 0, None, None) == OK
    assert copy(g, src=None) == copy(g, n=1000) == copy(changed(g, slot_stride=64)) == ARG
    assert copy(g, n=0x7FFFFFFF) == ARG
    for kw in (dict(page_size=1), dict(kv_heads=1, q_heads=1), dict(page_size=1, kv_heads=1, q_heads=1)):
        one = More(built, **kw)
        assert built.grand_pages_copy(one.h, 4, one.memory(16), one.memory(16), ctypes.byref(one.pages())) == OK
        assert built.fake_copy_flat() == 1, kw


def test_weights_of_chunks_without_cached_tokens(built):
    """max_k 0 beside a chunk of more rows than one tile's: its rows see nothing, and
    there are no weights to lay out."""
    c = More(built, q_heads=8)
    s, q, out, none = c.seqs(1, max_q=64, max_k=0), c.rows(64), c.rows(64), grand.Weights(None, 0, 0)
    for window, sinks in ((0, 0), (10, 0), (10, 4)):
        c.log()
        assert c.attend(s, q, c.pages(), out, wi=none, wo=none, window=window) == OK, c.error()
        r = [ctypes.byref(x) for x in (s, q, c.pages(), out, none, none)]
        assert built.grand_cache_attend_sinks(c.h, *r[:3], 0.125, 1, window, sinks, r[3], None, *r[4:]) == OK, c.error()
        assert c.attend_packed(s, q, c.packed(), out, window, sinks, none, none) == OK, c.error()
        launches = [x.split()[0] for x in c.log() if x.split()[0] in ("attend", "join", "weights")]
        assert launches == ["attend"] * 3


def test_scales_that_drift_into_codes(built):
    """Slots of codes leave room for scales beside them, but pages of scales are longer or shorter
    than the codes': from some page on they lie on codes of other slots."""
    for heads, slot in ((1, 32), (2, 64)):
        c = More(built, q_heads=heads, kv_heads=heads, head_dim=32)
        s, k, v, page = c.seqs(), c.rows(heads=heads), c.rows(heads=heads), 16 * slot
        at, src, dst = [c.memory(16 * page) for _ in range(4)], c.memory(12), c.memory(12)
        strides = dict(page_stride=page, slot_stride=slot, head_stride=32, scale_slot_stride=slot, scale_head_stride=32)
        for scales, want in ((page, OK), (page + 8, ARG), (page - 8, ARG)):
            for g in (c.packed(k=at[0], k_scales=at[0] + 16, v=at[1], v_scales=at[2], **strides),
                      c.packed(k=at[0], k_scales=at[1], v=at[2], v_scales=at[2] + 16, **strides)):
                g.scale_page_stride = scales
                assert c.append_packed(s, k, v, g) == want, (heads, scales, c.error())
                assert built.grand_packed_copy(c.h, 3, src, dst, ctypes.byref(g)) == want, (heads, scales)


def test_one_buffer_holds_codes_and_scales(built):
    """Codes and scales take turns, page by page, head by head or slot by slot, keys and
    values in one buffer or two: attention reads them and appends and copies write them."""
    c = More(built)                                    # rows of 32 and 2 bytes
    s, k, v, src, dst = c.seqs(), c.rows(heads=2), c.rows(heads=2), c.memory(12), c.memory(12)
    q, out = c.rows(), c.rows()
    page, head, slot = 16 * 2 * 34, 16 * 34 + 16, 2 * 32 + 16
    layouts = [
        # a page's codes, then its scales
        (dict(page_stride=page, slot_stride=64, head_stride=32, scale_page_stride=page, scale_slot_stride=4, scale_head_stride=2), 1024, page),
        # the same with heads outermost on one side
        (dict(page_stride=page, slot_stride=32, head_stride=512, scale_page_stride=page, scale_slot_stride=4, scale_head_stride=2), 1024, page),
        # a head's codes, then its scales
        (dict(page_stride=2 * head, head_stride=head, slot_stride=32, scale_page_stride=2 * head, scale_head_stride=head, scale_slot_stride=2),
         512, 2 * head),
        # a slot's codes, then its scales
        (dict(page_stride=16 * slot, slot_stride=slot, head_stride=32, scale_page_stride=16 * slot, scale_slot_stride=slot, scale_head_stride=2),
         64, 16 * slot),
    ]
    for strides, behind, size in layouts:
        # keys' pages, then values' pages; and the pages of both in turn
        apart = [c.memory(8 * size) for _ in range(2)]
        pools = [dict(k=apart[0], k_scales=apart[0] + behind, v=apart[1], v_scales=apart[1] + behind, **strides)]
        both = c.memory(16 * size)
        turns = dict(strides, page_stride=2 * size, scale_page_stride=2 * size)
        pools.append(dict(k=both, k_scales=both + behind, v=both + size, v_scales=both + size + behind, **turns))
        # (values a page further on: between pages of keys, not behind them)
        longer = c.memory(20 * size)
        pools.append(dict(k=longer, k_scales=longer + behind, v=longer + 3 * size, v_scales=longer + 3 * size + behind, **turns))
        for kw in pools:
            g = c.packed(**kw)
            assert c.attend_packed(s, q, g, out) == OK, c.error()
            assert c.append_packed(s, k, v, g) == OK, (strides, c.error())
            assert built.grand_packed_copy(c.h, 3, src, dst, ctypes.byref(g)) == OK
            for worse in (dict(k_scales=g.k_scales - 1), dict(v_scales=g.v_scales - 1), dict(k_scales=g.v_scales), dict(v=g.k + 16)):
                assert c.append_packed(s, k, v, changed(g, **worse)) == ARG, (strides, worse)
                assert built.grand_packed_copy(c.h, 3, src, dst, ctypes.byref(changed(g, **worse))) == ARG


def rows_bytes(at, row, n, strides):
    """Every byte of a pool's rows; None where two rows share one."""
    starts = at + sum(np.arange(m).reshape([-1 if i == j else 1 for j in range(3)]) * s for i, (m, s) in enumerate(zip(n, strides)))
    x = (starts.reshape(-1, 1) + np.arange(row)).ravel()
    return x if len(np.unique(x)) == len(x) else None


def test_pools_share_memory_or_not(built):
    """Random strides and places: no pools are written that share a byte, and none are
    refused whose codes and scales have the same steps along every axis."""
    c = More(built, q_heads=2, kv_heads=2, head_dim=64, page_size=4)
    s, k, v, r = c.seqs(max_k=12), c.rows(heads=2), c.rows(heads=2), np.random.default_rng(0)
    n, found = (3, 4, 2), {OK: 0, ARG: 0}
    far = c.memory(1 << 16)
    for _ in range(4000):
        def steps(row, unit):
            order, at, reach = r.permutation(3), [0, 0, 0], row
            for i in order:
                at[i] = -(-(reach + int(r.choice([0, 0, 0, 1, 2, 16, 32, 64, 200]))) // unit) * unit
                reach += (n[i] - 1) * at[i]
            return at
        codes = steps(32, 16)
        scales = codes if r.random() < 0.6 else steps(2, 1)
        if r.random() < 0.3:
            scales = [codes[0] if r.random() < 0.8 else x for x in scales]
        at = c.memory(1 << 15)
        place = 4096 + int(r.choice([r.integers(-2000, 2000), r.integers(-200, 200), 32, codes[0] - 4, codes[1] - 4, codes[2] - 4]))
        g = c.packed(3, k=at + 4096, k_scales=at + place, v=far, v_scales=far + (1 << 15), page_stride=codes[0], slot_stride=codes[1],
                     head_stride=codes[2], scale_page_stride=scales[0], scale_slot_stride=scales[1], scale_head_stride=scales[2])
        a, b = rows_bytes(at + 4096, 32, n, codes), rows_bytes(at + place, 2, n, scales)
        got = c.append_packed(s, k, v, g)
        assert got in (OK, ARG)
        found[got] += 1
        apart = a is not None and b is not None and not len(np.intersect1d(a, b))
        if got == OK:
            assert apart, (codes, scales, place)
        elif scales == codes:
            assert not apart, (codes, place)
    assert min(found.values()) > 400, found


def test_keys_and_values_that_partly_overlap(built):
    """16-bit pages that are written: keys and values are one pool, or share nothing."""
    c = More(built)
    s, k, v, g, src, dst = c.seqs(), c.rows(heads=2), c.rows(heads=2), c.pages(), c.memory(40), c.memory(40)
    size = 16 * 2 * 64 * 2                              # bytes of a page

    def write(g, k=k, v=v):
        r = [ctypes.byref(x) for x in (s, k, v, g)]
        return built.grand_cache_append(c.h, *r), built.grand_pages_copy(c.h, 10, src, dst, r[3])
    assert write(g) == (OK, OK)
    two = c.memory(2 * 8 * size)
    for at, want in ((0, OK), (64, ARG), (128, ARG), (size, ARG), (8 * size - 128, ARG), (8 * size, OK)):
        shared = grand.Pages(two, two + at, 8, g.page_stride, g.slot_stride, g.head_stride)
        assert c.attend(c.seqs(), c.rows(), shared, c.rows()) == OK, c.error()
        assert write(shared, k, v if at else k) == (want, want), (at, c.error())
        if want != OK:
            assert "overlap" in c.error()
    # keys and values of a page, of a slot, of a head in turn
    for strides, at in (((2 * 2048, 128, 64), 2 * 2048), ((2 * 2048, 2 * 128, 64), 2 * 128), ((2 * 2048, 2 * 128, 2 * 64), 2 * 64)):
        assert write(grand.Pages(two, two + at, 8, *strides)) == (OK, OK), c.error()
        assert write(grand.Pages(two, two + at - 16, 8, *strides)) == (ARG, ARG)


def test_workspace_of_windowed_weights(built):
    """Sums of rows are kept for the keys that a window reaches, not for all that are cached."""
    built.fake_largest.restype = ctypes.c_size_t
    n, chunk, length = 64, 64, 131_072
    for window, sinks in ((1024, 0), (1024, 300)):
        for packed in (False, True):
            c = More(built, q_heads=32, kv_heads=8)
            s, q, out = c.seqs(n, max_q=chunk, max_k=length), c.rows(n * chunk), c.rows(n * chunk)
            w, pages = c.weights(n, length), c.packed() if packed else c.pages()
            r = [ctypes.byref(x) for x in (s, q, pages, out, w, w)]
            call = built.grand_cache_attend_packed if packed else built.grand_cache_attend_sinks
            assert call(c.h, *r[:3], 0.125, 1, window, sinks, r[3], None, *r[4:]) == OK, c.error()
            # log-sum-exps of all rows; 256 keys of eight tiles at most for each head, a quarter more when it grows
            assert built.fake_largest() <= 1.25 * (n * chunk * 32 * 4 + n * 8 * 8 * 256 * 4 + 1024), built.fake_largest()


def test_shares_of_packed_tokens(built):
    """Equal shares of all keys fill the chip with three workgroups a CU, with two only where long
    shares of slots of all heads are read in runs of a page."""
    for kw, want in ((dict(), 2), (dict(page_size=8), 3), (dict(head_dim=96), 3), (dict(head_dim=104), 2), (dict(head_dim=64), 3),
                     (dict(head_dim=256), 2), (dict(page_size=64), 2)):
        c = More(built, **dict(dict(q_heads=32, kv_heads=8, head_dim=128), **kw))
        s, q, out, g = c.seqs(64, max_k=8192), c.rows(64), c.rows(64), c.packed()
        assert c.attend_packed(s, q, g, out) == OK and built.fake_units() * 8 == want * 256, kw
        row, most = 16 * -(-c.p.head_dim // 32), 2 if c.p.head_dim > 128 else 3
        beside = changed(g, slot_stride=row, head_stride=c.p.page_size * row)       # a head's slots side by side
        assert c.attend_packed(s, q, beside, out) == OK and built.fake_units() * 8 == most * 256, kw
        assert c.attend_packed(c.seqs(64, max_k=2048), q, g, out) == OK and built.fake_units() * 8 == most * 256, kw
    odd = More(built, q_heads=32, kv_heads=8, head_dim=128)
    g = odd.packed()
    assert odd.attend_packed(odd.seqs(64, max_k=8192), odd.rows(64), changed(g, k_scales=g.k_scales + 1), odd.rows(64)) == OK
    assert built.fake_units() * 8 == 3 * 256                                       # scales that are no aligned words
