"""The chunk kernel's own powers of two (exp2_by_fma in hga_cache_attn_sm100.cu), step by step in fp32 with the coefficients that stand there,
against 64 bits."""
import os
import re

import numpy as np

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_15105_b200", "csrc")


def coefficients():
    with open(os.path.join(CSRC, "hga_cache_attn_sm100.cu")) as f:
        text = f.read()
    body = text[text.index("void exp2_by_fma("):]
    body = body[:body.index("\n}\n")]
    c = [np.float32(x) for x in re.findall(r"pack_f32x2\((0\.\d+)f, 0\.\d+f\)", body)]
    assert len(c) == 5 and "12582912.f" in body and "0fC2FE0000" in body      # (-127)
    return c


def exp2_by_fma(x):
    """x float32; an addition in float32, a fused multiply-add in float64 (products of two fp32 numbers are exact there) rounded once more"""
    f32, f64 = np.float32, np.float64
    x = np.maximum(x, f32(-127))
    t = (x + f32(12582912)).astype(f32)
    n = (t - f32(12582912)).astype(f32)
    f = (f64(x) - f64(n)).astype(f32)
    assert np.abs(f).max() <= 0.5
    c = coefficients()
    p = np.full_like(x, c[0])
    for k in c[1:]:
        p = (f64(p) * f64(f) + f64(k)).astype(f32)
    two_n = ((t.view(np.uint32) << np.uint32(23)) + np.uint32(0x3f800000)).view(f32)
    return (p * two_n).astype(f32)


def test_error_of_the_polynomial():
    x = np.concatenate([np.linspace(-126, 14.5, 2000001), np.linspace(-1, 1, 200001), -np.exp2(np.linspace(-40, 0, 4001))]).astype(np.float32)
    y, want = exp2_by_fma(x).astype(np.float64), np.exp2(x.astype(np.float64))
    worst = np.max(np.abs(y / want - 1))
    assert 2.0 ** -19 < worst < 2.0 ** -18                                   # (what hga.h states; 2.6e-6 = 2^-18.5)
    assert worst < 2.75e-6


def test_ends_of_the_range():
    y = exp2_by_fma(np.array([-np.inf, -1e30, -127, 0, 1, -1], np.float32))
    assert y[0] == y[1] == y[2] == 0                                         # 2^-127 is the bit pattern of zero
    assert np.allclose(y[3:], [1, 2, 0.5], rtol=2.75e-6, atol=0)
