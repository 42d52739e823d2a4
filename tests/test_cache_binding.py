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


def test_tensors_that_are_not_dense_need_strides():
    import torch
    p = params(fmt=binding.HGA_CACHE_BF16)
    wide = torch.zeros(12, 4, 256)
    half, dense = wide[..., :128], torch.zeros(12, 4, 128)
    for name in ("q_stride", "o_stride", "kn_stride", "vn_stride", "k_stride", "v_stride", "out_stride", "table_stride", None):
        binding._check_cache_tensor("call", -1, p, name, dense)
        with pytest.raises(ValueError, match="strides"):
            binding._check_cache_tensor("call", -1, p, name, half)
        with pytest.raises(ValueError, match="current device"):
            binding._check_cache_tensor("call", 0, p, name, dense)
    p.q_stride[:] = half.stride()[:2]
    binding._check_cache_tensor("call", -1, p, "q_stride", half)
    p.table_stride = 16
    binding._check_cache_tensor("call", -1, p, "table_stride", torch.zeros(3, 16)[:, :9])
    with pytest.raises(ValueError, match="strides"):
        binding._check_cache_tensor("call", -1, p, "o_stride", half)


def test_strides_are_named_for_every_argument():
    """in the order of the calls' parameters"""
    import inspect
    for call, strides in ((binding.hga_cache_write, binding._WRITE_STRIDES), (binding.hga_cache_attn, binding._ATTN_STRIDES),
                          (binding.hga_cache_read, binding._READ_STRIDES)):
        names = [n for n in inspect.signature(call).parameters if n not in ("p", "stream", "tok_begin", "tok_end")]
        want = {"K_new": "kn_stride", "V_new": "vn_stride", "block_table": "table_stride", "K_cache": "k_stride", "V_cache": "v_stride",
                "K_out": "out_stride", "V_out": "out_stride", "Q": "q_stride", "O": "o_stride"}
        assert strides == tuple(want.get(n) for n in names)


def test_a_misaligned_status_word_is_refused(lib, ptr):
    """it is written by an atomic, which faults there (no launch here: refused ahead of it)"""
    p = params(n_tokens=0)
    for off in (1, 2, 3):
        assert lib.hga_cache_write(C.byref(p), *[ptr] * 9, ptr + off, None) == -3
        assert lib.hga_cache_attn(C.byref(p), *[ptr] * 10, None, 0, ptr + off, None) == -3
        assert lib.hga_cache_read(C.byref(p), 7, 7, *[ptr] * 8, ptr + off, None) == -3
    assert lib.hga_cache_write(C.byref(p), *[ptr] * 9, ptr + 4, None) == 0
