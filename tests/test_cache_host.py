"""The host side of the cache operators without a GPU: built alone, with
stand-ins for the HIP calls and the launches (fake_hip.cpp)."""
import ctypes
import os
import subprocess

import pytest

from conftest import ROOT
from paper_2608_21163_amd import grand
from paper_2608_21163_amd.build import CSRC, HIPCC

P = ctypes.c_void_p


@pytest.fixture(scope="module")
def built(tmp_path_factory):
    d = tmp_path_factory.mktemp("host")
    objects = []
    for src in (os.path.join(CSRC, "cache.hip"), os.path.join(ROOT, "tests", "fake_hip.cpp")):
        objects.append(str(d / os.path.basename(src)) + ".o")
        subprocess.check_call([HIPCC, "-x", "hip", "--offload-arch=gfx950", "--offload-host-only", "-O1", "-std=c++17", "-fPIC",
                               "-I", CSRC, "-I", os.path.join(ROOT, "include"), "-c", src, "-o", objects[-1]])
    out = str(d / "libhost.so")
    # (its own definitions first, also where the process has the HIP runtime)
    subprocess.check_call(["g++", "-shared", "-Wl,-Bsymbolic", "-o", out, *objects])
    lib = ctypes.CDLL(out)
    for name in grand.EXPORTED:
        if name.startswith("grand_cache_") and name != "grand_cache_last_error":
            getattr(lib, name).argtypes = getattr(grand.load_library(), name).argtypes
    lib.grand_cache_last_error.argtypes, lib.grand_cache_last_error.restype = [P], ctypes.c_char_p
    lib.fake_memory.argtypes, lib.fake_memory.restype = [ctypes.c_size_t, ctypes.c_int], ctypes.c_size_t
    lib.fake_log.restype = ctypes.c_char_p
    lib.fake_capture.argtypes = [ctypes.c_int, P]
    return lib


class Host:
    """A handle on the stand-ins, and arguments for its calls: two sequences of
    one new token and 40 cached ones, 4 query heads, 2 key/value heads of 64."""

    def __init__(self, lib, device=0, stream=None, **kw):
        lib.fake_reset()
        self.lib, self.device, self.h = lib, device, P()
        p = grand.CacheParams(ctypes.sizeof(grand.CacheParams), grand.BF16, 4, 2, 64, 16, device, stream)
        for k, v in kw.items():
            setattr(p, k, v)
        assert lib.grand_cache_create(ctypes.byref(p), ctypes.byref(self.h)) == grand.OK
        self.p = p
        self.log()

    def log(self):
        return self.lib.fake_log().decode().splitlines()

    def error(self):
        return self.lib.grand_cache_last_error(self.h).decode()

    def memory(self, size):
        return self.lib.fake_memory(size + 256, self.device)   # (more than it is, as allocators give)

    def seqs(self, n=2, max_q=1, max_k=40, q_start=False):
        pages = -(-max_k // self.p.page_size)
        return grand.Seqs(n, n * max_q, max_q, max_k, self.memory(n * pages * 4) if pages else None, pages, pages,
                          self.memory(n * 4 + 4) if q_start or max_q > 1 else None, self.memory(n * 4))

    def pages(self, n=8):
        row = self.p.kv_heads * self.p.head_dim
        size = n * self.p.page_size * row
        return grand.Pages(self.memory(size * 2), self.memory(size * 2), n, self.p.page_size * row, row, self.p.head_dim)

    def rows(self, tokens=2, heads=None):
        heads = self.p.q_heads if heads is None else heads
        return grand.Rows(self.memory(tokens * heads * self.p.head_dim * 2), heads * self.p.head_dim, self.p.head_dim)

    def weights(self, n=2, cap=40, heads=None):
        heads = self.p.kv_heads if heads is None else heads
        return grand.Weights(self.memory(n * heads * cap * 4), heads * cap, cap)

    def attend(self, s, q, pages, out, lse=None, wi=None, wo=None, causal=1, window=0):
        r = [None if x is None else ctypes.byref(x) for x in (s, q, pages, out, wi, wo)]
        return self.lib.grand_cache_attend(self.h, r[0], r[1], r[2], 0.125, causal, window, r[3], lse, r[4], r[5])


def test_a_stream_is_waited_for_on_its_own_gpu(built):
    """The default stream is every GPU's own: the wait before a change of
    streams is for the handle's GPU, whichever is current."""
    c = Host(built, device=3)
    built.fake_device(0)
    assert built.grand_cache_set_stream(c.h, 77) == grand.OK
    assert c.log() == ["hipSetDevice on 3", "hipStreamIsCapturing on 3", "hipStreamSynchronize of stream 0 on 3"]
    built.fake_device(0)
    assert built.grand_cache_set_stream(c.h, 77) == grand.OK and c.log() == []   # no change, no wait
    s, q, pages, out = c.seqs(), c.rows(), c.pages(), c.rows()
    assert c.attend(s, q, pages, out) == grand.OK
    assert all(x.endswith(" on 3") for x in c.log())


IMPLICIT, LAUNCH_FAILURE = 906, 719   # hipErrorStreamCaptureImplicit, hipErrorLaunchFailure


def test_calls_that_a_capture_does_not_allow(built):
    """The check and a change of streams wait, which would break a capture of the
    handle's stream: they are refused before that, and the handle goes on."""
    c = Host(built, stream=5)
    built.fake_capture(1, 5)
    for call in (lambda: built.grand_cache_check(c.h), lambda: built.grand_cache_set_stream(c.h, 6)):
        assert call() == grand.E_STATE and "capture" in c.error()
        assert not any("Synchronize" in x or "Memcpy" in x for x in c.log())
    assert built.grand_cache_set_stream(c.h, 5) == grand.OK
    assert c.attend(c.seqs(), c.rows(), c.pages(), c.rows()) == grand.OK
    built.fake_capture(0, None)
    assert built.grand_cache_check(c.h) == grand.OK
    assert built.grand_cache_set_stream(c.h, 6) == grand.OK
    assert c.attend(c.seqs(), c.rows(), c.pages(), c.rows()) == grand.OK


def test_a_capture_elsewhere_does_not_end_the_handle(built):
    """A handle on the default stream while another stream is captured: HIP
    refuses what is done there, and the handle is as it was afterwards."""
    c = Host(built)
    args = c.seqs(max_k=4000), c.rows(), c.pages(600), c.rows()
    for call in (b"hipStreamIsCapturing", b"attend", b"join"):
        built.fake_fail(call, IMPLICIT)
        assert c.attend(*args) == grand.E_STATE and "capture" in c.error()
        built.fake_fail(call, 0)
        assert c.attend(*args) == grand.OK
    for call in (b"hipStreamIsCapturing", b"hipMemcpyAsync", b"hipStreamSynchronize"):
        built.fake_fail(call, IMPLICIT)
        assert built.grand_cache_check(c.h) == grand.E_STATE
        built.fake_fail(call, 0)
        assert built.grand_cache_check(c.h) == grand.OK
    built.fake_fail(b"attend", LAUNCH_FAILURE)     # any other failure does end it
    assert c.attend(*args) == grand.E_DEVICE
    built.fake_fail(b"attend", 0)
    assert c.attend(*args) == grand.E_STATE


def moved(r, elements, **strides):
    """The same rows, pages or weights further on, with other strides."""
    out = type(r)()
    ctypes.pointer(out)[0] = r
    size = 4 if isinstance(r, grand.Weights) else 2
    out.p += elements * size
    for k, v in strides.items():
        setattr(out, k, v)
    return out


def test_results_beside_and_over_the_queries(built):
    """out may be q itself, or lie between its rows; every other way of sharing
    memory races with the rows still to be read."""
    c = Host(built)
    n, d = 6, 64
    s, pages = c.seqs(2, max_q=3), c.pages()
    wide = grand.Rows(c.memory(2 * n * 12 * d * 2), 12 * d, d)     # the first six of twelve tokens of 12 heads
    wi = c.weights()
    ok, bad = grand.OK, grand.E_ARG
    for q, out, want, weighted in (
            (wide, wide, ok, bad),                                                  # in place
            (wide, moved(wide, 4 * d), ok, ok),                                     # the next heads of the same rows
            (moved(wide, 8 * d), wide, ok, ok),
            (wide, moved(wide, 3 * d), bad, bad),                                   # one head in common
            (wide, moved(wide, 8), bad, bad),                                       # a few elements in common
            (wide, moved(wide, 12 * d), bad, bad),                                  # a token on
            (wide, moved(wide, 12 * d + 4 * d), ok, ok),                            # a token on, the next heads
            (wide, moved(wide, 0, token_stride=4 * d), bad, bad),                   # the same start, other strides
            (wide, moved(wide, 0, token_stride=d, head_stride=6 * d), bad, bad),
            (wide, moved(wide, 6 * 12 * d // 2, token_stride=4 * d), bad, bad)):    # packed, in the second half
        assert c.attend(s, q, pages, out) == want, (out.p - q.p, c.error())
        assert c.attend(s, q, pages, out, wi=wi, wo=wi) == weighted, (out.p - q.p, c.error())
    one = c.seqs(1)
    q = grand.Rows(c.memory(12 * d * 2), 12 * d, d)
    assert c.attend(one, q, pages, moved(q, 0, token_stride=8 * d)) == ok       # one token: its stride says nothing
    assert c.attend(one, q, pages, moved(q, 4 * d, token_stride=8 * d)) == ok
    assert c.attend(one, q, pages, moved(q, 2 * d, token_stride=8 * d)) == bad
    q, row = c.rows(n), c.p.kv_heads * d
    assert c.attend(s, q, pages, grand.Rows(pages.k + 4 * row * 2, 4 * d, d)) == bad and "pages" in c.error()
    assert c.attend(s, q, pages, grand.Rows(pages.v, 4 * d, d)) == bad


def test_weights_in_place_or_apart(built):
    c = Host(built)
    s, q, pages, out = c.seqs(), c.rows(), c.pages(), c.rows()
    w = grand.Weights(c.memory(4 * 6 * 100 * 4), 600, 100)     # rows of 40 of 100 entries, two of six heads
    ok, bad = grand.OK, grand.E_ARG
    for wo, want in ((w, ok), (moved(w, 200), ok), (moved(w, 40), ok), (moved(w, 39), bad), (moved(w, 100), bad), (moved(w, 600), bad),
                     (moved(w, 0, head_stride=200), bad), (moved(w, 600, seq_stride=100, head_stride=200), bad), (moved(w, 1200), ok)):
        assert c.attend(s, q, pages, out, wi=w, wo=wo) == want, ((wo.p - w.p) // 4, c.error())


def test_listed_attention_in_place_or_apart(built):
    c = Host(built)
    n, d = 5, 64
    pages, ids = c.pages(), c.memory(n * 4 * 7 * 4)
    q, prior = c.rows(n), grand.Rows(c.memory(n * 12 * d * 2), 12 * d, d)
    lse, prior_lse = c.memory(n * 4 * 4), c.memory(2 * n * 4 * 4)

    def call(out, q=q, lse=lse):
        return built.grand_cache_attend_ids(c.h, n, ctypes.byref(q), ctypes.byref(pages), ids, 7, 28, 7, 0.125, ctypes.byref(prior), prior_lse,
                                            ctypes.byref(out), lse)
    assert call(prior) == call(c.rows(n)) == call(q) == call(moved(prior, 4 * d)) == grand.OK
    assert call(prior, lse=prior_lse) == call(prior, lse=prior_lse + n * 16) == grand.OK
    assert call(moved(prior, 2 * d)) == call(moved(prior, 0, token_stride=8 * d)) == call(moved(q, 8, token_stride=4 * d)) == grand.E_ARG
    assert call(prior, lse=prior_lse + 16) == grand.E_ARG and "lse" in c.error()
    assert call(grand.Rows(pages.v, 4 * d, d)) == grand.E_ARG


def test_evictions_write_over_nothing_they_read(built):
    c = Host(built)
    s = c.seqs(2, max_k=64)
    buffers = dict(budget=c.memory(8), out_table=c.memory(32), out_lens=c.memory(8), freed=c.memory(32), n_freed=c.memory(8))
    w, wo = c.weights(2, 64), c.weights(2, 64)

    def call(wo=wo, **kw):
        b = dict(buffers, **kw)
        return built.grand_cache_evict(c.h, ctypes.byref(s), 2, 64, ctypes.byref(w), b["budget"], 1, 1, b["out_table"], ctypes.byref(wo),
                                       b["out_lens"], b["freed"], b["n_freed"])
    assert call() == grand.OK
    for kw in (dict(out_table=s.table), dict(out_table=s.table + 28), dict(freed=s.table), dict(out_lens=s.lens), dict(n_freed=s.lens + 4),
               dict(out_lens=buffers["budget"]), dict(freed=buffers["out_table"] + 16), dict(n_freed=buffers["out_lens"]), dict(wo=w),
               dict(wo=moved(w, 32)), dict(out_table=wo.p), dict(freed=w.p)):
        assert call(**kw) == grand.E_ARG and "overlap" in c.error(), kw
    wide = grand.Weights(c.memory(2 * 6 * 64 * 4), 6 * 64, 64)
    w = wide
    assert call(wo=moved(wide, 2 * 64)) == grand.OK and call(wo=moved(wide, 64)) == grand.E_ARG


def test_new_tokens_go_into_slots_of_their_own(built):
    """Pages whose slots share memory may be read, but not appended to; keys
    and values go to one pool only if they are the same rows."""
    c = Host(built)
    s, k, v, pages, q, out = c.seqs(), c.rows(heads=2), c.rows(heads=2), c.pages(), c.rows(), c.rows()

    def append(pages, k=k, v=v):
        r = [ctypes.byref(x) for x in (s, k, v, pages)]
        return built.grand_cache_append(c.h, *r)
    assert append(pages) == grand.OK
    for kw in (dict(slot_stride=0), dict(page_stride=0), dict(head_stride=0), dict(slot_stride=64), dict(head_stride=56), dict(page_stride=2000)):
        shared = grand.Pages(*[kw.get(f, getattr(pages, f)) for f, _ in grand.Pages._fields_])
        assert c.attend(s, q, shared, out) == grand.OK
        assert append(shared) == grand.E_ARG and "overlap" in c.error(), kw
    heads_outside = grand.Pages(pages.k, pages.v, 8, 16 * 2 * 64, 64, 16 * 64)
    assert append(heads_outside) == grand.OK
    one = grand.Pages(pages.k, pages.k, 8, pages.page_stride, pages.slot_stride, pages.head_stride)
    assert append(one) == grand.E_ARG and append(one, k, k) == grand.OK
    assert c.attend(s, q, one, out) == grand.OK


def test_positions_fit_31_bits(built):
    """Kernels compute positions in signed 32 bits: up to a tile of 64 keys past
    the last cached token, and a window before a chunk that is longer than
    its cache."""
    c = Host(built, page_size=1024)
    q, pages, out = c.rows(4096), c.pages(2), c.rows(4096)
    for max_k, max_q, want in (((1 << 31) - 65, 1, grand.OK), ((1 << 31) - 64, 1, grand.E_CAPACITY), ((1 << 31) - 1, 1, grand.E_CAPACITY),
                               ((1 << 31) - 4160, 4096, grand.OK), ((1 << 31) - 4159, 4096, grand.E_CAPACITY)):
        s = c.seqs(1, max_q=max_q, max_k=max_k)
        assert c.attend(s, q, pages, out, window=(1 << 31) - 5000) == want, (max_k, max_q)
    s = c.seqs(1, max_q=1, max_k=(1 << 31) - 65)
    s.max_q = 0xFFFFFFFF                      # a loose bound: there is one new token
    s.q_start = c.memory(8)
    assert c.attend(s, q, pages, out) == grand.OK


def test_weights_of_no_cached_tokens(built):
    """max_k 0: weights have no entries and, as empty tensors, no memory."""
    c = Host(built)
    none = grand.Weights(None, 0, 0)
    assert c.attend(c.seqs(2, max_k=0), c.rows(), c.pages(), c.rows(), wi=none, wo=none) == grand.OK
    assert c.attend(c.seqs(2, max_k=1), c.rows(), c.pages(), c.rows(), wi=none, wo=none) == grand.E_ARG


def test_steps_along_axes_of_one_say_nothing(built):
    """A view's stride along an axis of length one may be anything."""
    c = Host(built, q_heads=1, kv_heads=1, page_size=1)
    s = c.seqs(1, max_k=6)
    q, out, pages = c.rows(1), c.rows(1), c.pages(1)
    w = c.weights(1, 6)
    s.table_stride = 1
    for x in (q, out):
        x.token_stride, x.head_stride = 1, -3
    pages.page_stride, pages.slot_stride, pages.head_stride = 3, -1, 1 << 40
    w.seq_stride = w.head_stride = -1
    assert c.attend(s, q, pages, out, wi=w, wo=w) == grand.OK, c.error()
    r = [ctypes.byref(x) for x in (s, q, out, pages)]
    assert built.grand_cache_append(c.h, *r) == grand.OK, c.error()
    ids = c.memory(24)
    assert built.grand_cache_attend_ids(c.h, 1, ctypes.byref(q), ctypes.byref(pages), ids, 6, -5, -7, 0.5, None, None, ctypes.byref(out), None) == grand.OK
    assert built.grand_cache_evict(c.h, ctypes.byref(s), 1, 6, ctypes.byref(w), c.memory(4), 0, 0, c.memory(24), ctypes.byref(c.weights(1, 6)),
                                   c.memory(4), c.memory(24), c.memory(4)) == grand.OK, c.error()
    two = c.seqs(2, max_k=6)                     # of more they are judged as before
    two.table_stride = 1
    assert c.attend(two, c.rows(2), c.pages(2), c.rows(2)) == grand.E_ARG
    assert c.attend(c.seqs(2), moved(c.rows(3), 0, token_stride=60), c.pages(2), c.rows(2)) == grand.E_ARG
    assert c.attend(c.seqs(2), c.rows(2), c.pages(2), moved(c.rows(2), 0, token_stride=-64)) == grand.E_ARG
