"""The paged cache's calls as a program makes them from Python, without a GPU: what is accepted and refused before anything is launched."""
import ctypes as C

import pytest

from paper_2607_15105_b200 import binding, build


@pytest.fixture(scope="module")
def lib():
    build.build_library()
    return binding.lib()


def params(**kw):
    a = dict(n_seq=3, n_q_heads=4, n_kv_heads=2, head_dim=128, page_size=16, n_pages=40, max_pages=9, fmt=binding.HGA_CACHE_MXFP8,
             n_tokens=12, max_new=8, max_len=64)
    a.update(kw)
    return binding.make_cache_params(**a)


@pytest.fixture(scope="module")
def ptr():
    buf = (C.c_char * 4096)()
    ptr.keep = buf
    a = C.addressof(buf)
    return a + (-a) % 16


@pytest.mark.parametrize("fmt", (binding.HGA_CACHE_BF16, binding.HGA_CACHE_MXFP8))
def test_tensors_of_no_rows_may_have_no_address(lib, ptr, fmt):
    """an empty torch tensor's address is zero"""
    p = params(n_tokens=0, fmt=fmt)
    assert lib.hga_cache_write(C.byref(p), None, None, *[ptr] * 7, None, None) == 0
    assert lib.hga_cache_attn(C.byref(p), None, *[ptr] * 7, None, None, None, 0, None, None) == 0
    assert lib.hga_cache_read(C.byref(p), 7, 7, *[ptr] * 6, None, None, None, None) == 0
    # with rows, and what is no tensor of rows, as before
    q = params(fmt=fmt)
    assert lib.hga_cache_write(C.byref(q), None, None, *[ptr] * 7, None, None) == -1
    assert lib.hga_cache_attn(C.byref(q), None, *[ptr] * 8, None, None, 0, None, None) == -1
    assert lib.hga_cache_attn(C.byref(q), *[ptr] * 8, None, None, None, 0, None, None) == -1
    assert lib.hga_cache_read(C.byref(q), 7, 8, *[ptr] * 6, None, None, None, None) == -1
    assert lib.hga_cache_write(C.byref(p), None, None, None, *[ptr] * 6, None, None) == -1
    assert lib.hga_cache_attn(C.byref(p), None, ptr, None, *[ptr] * 5, None, None, None, 0, None, None) == -1
    assert lib.hga_cache_read(C.byref(p), 7, 7, None, *[ptr] * 5, None, None, None, None) == -1
