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
        return self.lib.fake_memory(size, self.device)

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
