"""The structs of the cache operators match the header, and arguments that
need no GPU to be judged are refused."""
import ctypes
import subprocess

import pytest

from conftest import ROOT
from paper_2608_21163_amd import grand

STRUCTS = {"grand_cache_params": grand.CacheParams, "grand_pages": grand.Pages, "grand_rows": grand.Rows,
           "grand_weights": grand.Weights, "grand_seqs": grand.Seqs}


def test_struct_layouts(tmp_path):
    lines = ["#include <stddef.h>", "#include <stdio.h>", f'#include "{ROOT}/include/grand.h"', "int main(void) {"]
    want = []
    for name, cls in STRUCTS.items():
        lines.append(f'printf("%zu\\n", sizeof({name}));')
        want.append(ctypes.sizeof(cls))
        for f, _ in cls._fields_:
            lines.append(f'printf("%zu\\n", offsetof({name}, {f}));')
            want.append(getattr(cls, f).offset)
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines + ["return 0; }"]))
    subprocess.check_call(["gcc", "-std=c11", str(src), "-o", str(exe)])
    assert [int(x) for x in subprocess.check_output([str(exe)]).split()] == want


def test_default_params():
    p = grand.CacheParams()
    grand.load_library().grand_default_cache_params(ctypes.byref(p))
    assert p.struct_size == ctypes.sizeof(grand.CacheParams) and p.dtype == grand.BF16
    assert (p.q_heads, p.kv_heads, p.head_dim, p.page_size) == (32, 8, 128, 16)


@pytest.mark.parametrize("field,value", [("struct_size", 8), ("dtype", grand.F32), ("q_heads", 12), ("q_heads", 0), ("kv_heads", 0),
                                         ("head_dim", 100), ("head_dim", 512), ("head_dim", 0), ("page_size", 0), ("page_size", 24),
                                         ("page_size", 2048), ("q_heads", 4096)])
def test_create_rejects_bad_parameters_before_touching_the_gpu(field, value):
    lib = grand.load_library()
    p = grand.CacheParams()
    lib.grand_default_cache_params(ctypes.byref(p))
    setattr(p, field, value)
    h = ctypes.c_void_p()
    assert lib.grand_cache_create(ctypes.byref(p), ctypes.byref(h)) == grand.E_ARG and not h.value


def test_null_handles():
    lib = grand.load_library()
    assert lib.grand_cache_destroy(None) == grand.OK
    assert lib.grand_cache_check(None) == grand.E_ARG
    assert lib.grand_cache_set_stream(None, None) == grand.E_ARG
    assert lib.grand_cache_append(None, None, None, None, None) == grand.E_ARG
    assert lib.grand_cache_attend(None, None, None, None, 1.0, 1, 0, None, None, None, None) == grand.E_ARG
    assert lib.grand_cache_attend_ids(None, 1, None, None, None, 1, 0, 0, 1.0, None, None, None, None) == grand.E_ARG
    assert lib.grand_cache_evict(None, None, 1, 1, None, None, 0, 0, None, None, None, None, None) == grand.E_ARG
    assert b"null" in lib.grand_cache_last_error(None)
    assert lib.grand_cache_create(None, None) == grand.E_ARG
