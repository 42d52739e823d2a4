"""The paged cache's numbers at the edges of their types: NaN codes, blocks of zeros, scales out of fp16's range, what lies behind a
sequence, queries and values next to the ends of bf16's range.  Against 64 bits, or bit for bit against the same call with other
contents in what a row does not see."""
import numpy as np
import pytest
import torch

import cache_testlib as T
from paper_2607_15105_b200 import binding

pytestmark = pytest.mark.gpu


class Pool(T.Problem):
    """... with e4m3's two NaN codes read as what they are"""

    def values(self, name):
        v = super().values(name)
        if self.fmt == "mx8":
            v[(getattr(self, name).cpu().numpy() & 127) == 127] = np.nan
        return v


@pytest.mark.parametrize("fmt", ("mx8", "mx4"))
@pytest.mark.parametrize("d", (64, 128))
def test_any_byte_reads_back_as_the_type_says(fmt, d):
    """a pool that another program filled: all codes under all scales whose numbers bf16 holds, e4m3's NaN codes among them"""
    pr = Pool([(1, 97), (1, 64)], fmt, hq=2, hkv=2, d=d, page=16, seed=41)
    low, high = (3, 246) if fmt == "mx8" else (0, 252)
    for name in "KV":
        stored, scale = getattr(pr, name), getattr(pr, name + "_scale")
        stored.copy_(torch.randint(0, 256, stored.shape, generator=pr.g))
        s = torch.randint(low, high + 1, scale.shape, generator=pr.g)
        s[torch.rand(s.shape, generator=pr.g) < 0.05] = 255
        scale.copy_(s)
    out = [torch.full((2, 2, 97, d), 9.0, dtype=torch.bfloat16, device="cuda") for _ in "KV"]
    binding.hga_cache_read(pr.p, 0, 97, pr.d_lens, pr.d_table, *pr.cache(), *out, pr.status)
    for name, o in zip("KV", out):
        values = pr.values(name)
        for i, n in enumerate((97, 64)):
            want, got = pr.resident(values, i), T.f64(o[i])
            assert np.isnan(want).any()
            assert np.array_equal(got[:, :n], want, equal_nan=True)
            assert (got[:, n:] == 9).all()


