"""The paged cache without a GPU: refusals of the entry points, the layout of their parameters, and the tests' own statement
of the formats against torch's conversions."""
import ctypes as C

import numpy as np
import pytest
import torch

import cache_testlib as T
from paper_2607_15105_b200 import binding, build


@pytest.fixture(scope="module")
def lib():
    build.build_library()
    return binding.lib()


def params(**kw):
    a = dict(n_seq=3, n_q_heads=4, n_kv_heads=2, head_dim=128, page_size=16, n_pages=40, max_pages=9, fmt=binding.HGA_CACHE_MXFP8,
             n_tokens=12, max_new=8, max_len=100)
    a.update(kw)
    return binding.make_cache_params(**a)


@pytest.fixture(scope="module")
def ptr():
    buf = (C.c_char * 4096)()
    a = C.addressof(buf)
    ptr.keep = buf
    return a + (-a) % 16


def calls(lib, p, ptr, **kw):
    """status codes of the three calls; kw replaces a pointer by name (nothing is launched: every case here is refused)"""
    def a(name):
        return kw.get(name, ptr)
    w = lib.hga_cache_write(C.byref(p), a("K_new"), a("V_new"), a("cu_q"), a("seq_lens"), a("table"), a("K"), a("V"), a("K_scale"),
                            a("V_scale"), None, None)
    r = lib.hga_cache_read(C.byref(p), kw.get("begin", 0), kw.get("end", 10), a("seq_lens"), a("table"), a("K"), a("V"), a("K_scale"),
                           a("V_scale"), a("K_out"), a("V_out"), None, None)
    t = lib.hga_cache_attn(C.byref(p), a("Q"), a("cu_q"), a("seq_lens"), a("table"), a("K"), a("V"), a("K_scale"), a("V_scale"), a("O"),
                           a("LSE"), a("workspace"), kw.get("bytes", 1 << 40), None, None)
    return w, r, t


def test_parameter_block_layout():
    # 14 four-byte fields, then 4 x 2 + 3 x 3 + 1 strides of 8 bytes
    assert C.sizeof(binding.HgaCacheParams) == 56 + 8 * 18
    assert binding.HgaCacheParams.q_stride.offset == 56
    assert binding.HgaCacheParams.k_stride.offset == 56 + 64


@pytest.mark.parametrize("change,code", [
    (dict(n_seq=0), -2), (dict(n_seq=65536), -2), (dict(n_q_heads=0), -2), (dict(n_kv_heads=3), -2), (dict(head_dim=96), -4),
    (dict(n_q_heads=258, n_kv_heads=2), -4), (dict(fmt=3), -4), (dict(fmt=-1), -4), (dict(page_size=0), -2), (dict(page_size=12), -2),
    (dict(page_size=4104), -2), (dict(n_pages=0), -2), (dict(max_pages=0), -2), (dict(max_pages=1 << 30), -2), (dict(n_tokens=-1), -2),
    (dict(max_new=0), -2), (dict(max_len=-1), -2), (dict(n_tokens=1 << 30, n_q_heads=128, n_kv_heads=2), -2),
    (dict(table_stride=5), -2), (dict(q_stride=(4, 128)), -3), (dict(q_stride=(-512, 128)), -3), (dict(q_stride=(512, 64)), -2),
    (dict(o_stride=(0, 128)), -2), (dict(k_stride=(4096, 2048, 8)), -3), (dict(k_stride=(4096, 2048, 0)), -2),
    (dict(v_stride=(4096, 2048, 112)), -2), (dict(kn_stride=(256, 132)), -3), (dict(vn_stride=(256, 120)), -2)])
def test_parameters_are_refused(lib, ptr, change, code):
    p = params(**change)
    n = C.c_size_t()
    assert lib.hga_cache_workspace_bytes(C.byref(p), C.byref(n)) == code
    assert calls(lib, p, ptr) == (code,) * 3


def test_flags_and_reserved_are_refused(lib, ptr):
    for name in ("flags", "reserved"):
        p = params()
        setattr(p, name, 1)
        assert calls(lib, p, ptr) == (-4,) * 3


def test_null_and_misaligned_pointers(lib, ptr):
    p = params()
    n = C.c_size_t()
    assert lib.hga_cache_workspace_bytes(None, C.byref(n)) == -1
    assert lib.hga_cache_workspace_bytes(C.byref(p), None) == -1
    assert lib.hga_cache_write(None, *[ptr] * 9, None, None) == -1
    for name in ("seq_lens", "table", "K", "V", "K_scale", "V_scale"):
        assert calls(lib, p, ptr, **{name: None}) == (-1,) * 3, name
    assert calls(lib, p, ptr, cu_q=None, begin=-1) == (-1, -2, -1)
    assert calls(lib, p, ptr, K_new=None, V_new=None, K_out=None, V_out=None, Q=None) == (-1,) * 3
    assert calls(lib, p, ptr, K_new=ptr + 2, K_out=ptr + 2, O=None) == (-3, -3, -1)
    for name in ("K", "V", "K_scale", "V_scale"):
        assert calls(lib, p, ptr, **{name: ptr + 8}) == (-3,) * 3, name
    for name in ("seq_lens", "table"):
        assert calls(lib, p, ptr, **{name: ptr + 1}) == (-3,) * 3, name
    for name in ("Q", "O", "workspace"):
        assert lib.hga_cache_attn(C.byref(p), *[ptr + (8 if n == name else 0) for n in ("Q", "cu", "l", "t", "K", "V", "a", "b", "O", "LSE", "workspace")],
                                  1 << 40, None, None) == -3
    assert lib.hga_cache_attn(C.byref(p), *[ptr] * 9, ptr + 2, ptr, 1 << 40, None, None) == -3


def test_ranges_and_workspace(lib, ptr):
    # a problem that needs a workspace: one sequence whose keys are shared out
    p = params(n_seq=1, max_pages=4096, max_len=65536, n_tokens=2, max_new=2)
    need = binding.hga_cache_workspace_bytes(p)
    assert need > 0
    for bytes_, ws in ((need - 1, ptr), (need, None), (0, ptr)):
        assert lib.hga_cache_attn(C.byref(p), *[ptr] * 10, ws, bytes_, None, None) == -5
    # token ranges
    for begin, end in ((-1, 4), (5, 4)):
        assert lib.hga_cache_read(C.byref(p), begin, end, *[ptr] * 8, None, None) == -2
    # short sequences need none
    assert binding.hga_cache_workspace_bytes(params(max_len=64)) == 0


def test_nothing_to_do_is_no_error(lib, ptr):
    p = params(n_tokens=0, max_len=64)
    assert lib.hga_cache_write(C.byref(p), *[ptr] * 9, None, None) == 0
    assert lib.hga_cache_attn(C.byref(p), *[ptr] * 10, None, 0, None, None) == 0
    assert lib.hga_cache_read(C.byref(p), 5, 5, *[ptr] * 8, None, None) == 0


@pytest.mark.parametrize("fmt", (binding.HGA_CACHE_BF16, binding.HGA_CACHE_MXFP8, binding.HGA_CACHE_MXFP4))
@pytest.mark.parametrize("n_seq", (1, 2, 700))
@pytest.mark.parametrize("hq", (2, 130, 256))
def test_no_tokens_of_any_number_of_heads(lib, ptr, fmt, n_seq, hq):
    p = params(n_seq=n_seq, n_q_heads=hq, n_tokens=0, max_pages=4096, max_len=0, fmt=fmt)
    n = binding.hga_cache_workspace_bytes(p)
    assert n == 0
    assert lib.hga_cache_attn(C.byref(p), *[ptr] * 10, None, n, None, None) == 0


def test_positions_that_an_int_does_not_hold(lib, ptr):
    n = C.c_size_t()
    far = params(max_pages=(1 << 26) + 1, max_len=0)           # pages of 16
    assert lib.hga_cache_workspace_bytes(C.byref(far), C.byref(n)) == -2
    assert calls(lib, far, ptr) == (-2,) * 3
    assert binding.hga_cache_workspace_bytes(params(max_pages=(1 << 26) + 1, max_len=64)) == 0
    one = params(n_seq=1, n_q_heads=1, n_kv_heads=1)
    for end in (0x7fffffff, 0x7fffff01):
        assert lib.hga_cache_read(C.byref(one), 0, end, *[ptr] * 8, None, None) == -2


def test_formats_against_torch():
    codes = torch.arange(256, dtype=torch.uint8)
    want = codes.view(torch.float8_e4m3fn).double().numpy()
    scales = np.full((8,), 127, np.uint8)
    got = T.held(codes.numpy().reshape(8, 32), scales.reshape(8, 1), "mx8").reshape(-1)
    fine = ~np.isnan(want)
    assert (got[fine] == want[fine]).all() and fine.sum() == 254
    assert list(T.MAGNITUDES["mx4"]) == [0, .5, 1, 1.5, 2, 3, 4, 6]
    # rounding: against torch's conversion of numbers between -448 and 448 with the scale held at one
    x = torch.randn(64, 32, generator=torch.Generator().manual_seed(1)).bfloat16() * 3
    x[:, 0] = 448
    c, s = T.quantise(T.f64(x), "mx8")
    assert (s == 127).all() and (torch.from_numpy(c).view(torch.float8_e4m3fn).double() == x.to(torch.float8_e4m3fn).double()).all()


@pytest.mark.parametrize("fmt,top", [("mx8", 448.0), ("mx4", 6.0)])
def test_scale_is_the_smallest_that_fits(fmt, top):
    for amax, code in ((top, 127), (top * 1.0078125, 128), (top / 2, 126), (top * 0.9921875, 127), (0.0, 0), (2.0 ** -133, 0)):
        x = np.zeros((1, 32))
        x[0, 5] = -amax
        _, s = T.quantise(x, fmt)
        assert s[0, 0] == code, (amax, s)
    big = np.zeros((1, 32))
    big[0, 1] = (2 - 2.0 ** -7) * 2.0 ** 127              # the largest bf16 number
    c, s = T.quantise(big, fmt)
    v = T.held(c, s, fmt)
    assert v.max() < 2.0 ** 128 and torch.tensor(v).bfloat16().double().numpy().max() == v.max()
    big[0, 3] = np.inf
    assert T.quantise(big, fmt)[1][0, 0] == 255
