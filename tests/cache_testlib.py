"""Plain 64-bit statements of the paged key/value cache, for its tests: the formats element by element, where a token lies, and
attention row by row.  Nothing here uses the library's kernels."""
import numpy as np
import torch

from paper_2607_15105_b200 import binding

FORMATS = {"bf16": binding.HGA_CACHE_BF16, "mx8": binding.HGA_CACHE_MXFP8, "mx4": binding.HGA_CACHE_MXFP4}


def _e4m3(code):
    e, m = (code >> 3) & 15, code & 7
    return m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)


def _e2m1(code):
    e, m = (code >> 1) & 3, code & 1
    return m * 0.5 if e == 0 else (2 + m) * 2.0 ** (e - 2)


# magnitudes by code, ascending (e4m3's last code is NaN)
MAGNITUDES = {"mx8": np.array([_e4m3(c) for c in range(127)]), "mx4": np.array([_e2m1(c) for c in range(8)])}


def quantise(x, fmt):
    """x float64 [..., d] of bf16 numbers -> (element codes uint8 [..., d], scale codes uint8 [..., d / 32])"""
    mags = MAGNITUDES[fmt]
    b = x.reshape(*x.shape[:-1], -1, 32)
    amax = np.abs(b).max(-1)
    codes = np.zeros(b.shape, np.uint8)
    scales = np.zeros(amax.shape, np.uint8)
    for at in np.ndindex(amax.shape):
        if not np.isfinite(amax[at]):
            scales[at] = 255
            continue
        e = -127
        while amax[at] > mags[-1] * 2.0 ** e:
            e += 1
        v = np.abs(b[at]) / 2.0 ** e
        hi = np.clip(np.searchsorted(mags, v), 1, len(mags) - 1)          # mags[hi-1] < v <= mags[hi]
        lo = hi - 1
        down, up = v - mags[lo], mags[hi] - v
        c = np.where((down < up) | ((down == up) & (lo % 2 == 0)), lo, hi)
        while (mags[c] * 2.0 ** e >= 2.0 ** 128).any():                    # past bf16: toward zero
            c = np.where(mags[c] * 2.0 ** e >= 2.0 ** 128, c - 1, c)
        codes[at] = c + (128 if fmt == "mx8" else 8) * np.signbit(b[at])
        scales[at] = e + 127
    return codes.reshape(x.shape), scales


def held(codes, scales, fmt):
    """float64 [..., d]"""
    sign = 128 if fmt == "mx8" else 8
    v = MAGNITUDES[fmt][np.minimum(codes % sign, len(MAGNITUDES[fmt]) - 1)] * np.where(codes >= sign, -1.0, 1.0)
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return v * np.repeat(s, 32, -1)


def pack(codes, fmt):
    return codes if fmt == "mx8" else (codes[..., 0::2] | (codes[..., 1::2] << 4))


def unpack(stored, fmt):
    if fmt == "mx8":
        return stored
    out = np.empty(stored.shape[:-1] + (2 * stored.shape[-1],), np.uint8)
    out[..., 0::2], out[..., 1::2] = stored & 15, stored >> 4
    return out


def f64(t):
    return t.detach().to(torch.float64).cpu().numpy()


class Problem:
    """A pool with sequences in it.  seqs: (new tokens, resident tokens with them) of each."""

    def __init__(self, seqs, fmt="bf16", hq=4, hkv=2, d=64, page=16, seed=0, order="head", spare_rows=0, device="cuda",
                 max_new=None, max_len=None, spread=1.0, extra_pages=2):
        g = self.g = torch.Generator().manual_seed(seed)
        self.seqs, self.fmt, self.hq, self.hkv, self.d, self.page, self.device = seqs, fmt, hq, hkv, d, page, device
        used = [-(-t // page) for _, t in seqs]
        self.n_pages = sum(used) + extra_pages
        self.new = sum(n for n, _ in seqs)
        self.n_tokens = self.new + spare_rows
        perm = torch.randperm(self.n_pages, generator=g).int()
        self.table = torch.full((len(seqs), max(max(used), 1)), -7, dtype=torch.int32)
        at = 0
        for i, u in enumerate(used):
            self.table[i, :u] = perm[at:at + u]
            at += u
        self.cu = torch.tensor([0] + list(np.cumsum([n for n, _ in seqs])), dtype=torch.int32)
        self.lens = torch.tensor([t for _, t in seqs], dtype=torch.int32)
        row = {"bf16": d, "mx8": d, "mx4": d // 2}[fmt]
        shape = (self.n_pages, hkv, page) if order == "head" else (self.n_pages, page, hkv)

        def pool(values):
            """values bf16 [n_pages, hkv, page, d] -> (stored, scales) with the pool's axes in the order asked for"""
            if fmt == "bf16":
                stored, scales = values, None
            else:
                codes, sc = quantise(f64(values), fmt)
                stored, scales = torch.from_numpy(pack(codes, fmt)), torch.from_numpy(sc).to(device)
            if order != "head":
                stored = stored.transpose(1, 2).contiguous().transpose(1, 2)
            return stored.to(device) if order == "head" else stored.transpose(1, 2).contiguous().to(device).transpose(1, 2), scales

        self.K_values = (torch.randn(self.n_pages, hkv, page, d, generator=g) * spread).bfloat16()
        self.V_values = torch.randn(self.n_pages, hkv, page, d, generator=g).bfloat16()
        self.K, self.K_scale = pool(self.K_values)
        self.V, self.V_scale = pool(self.V_values)
        assert tuple(self.K.shape) == (self.n_pages, hkv, page, row) and shape
        self.p = binding.make_cache_params(
            n_seq=len(seqs), n_q_heads=hq, n_kv_heads=hkv, head_dim=d, page_size=page, n_pages=self.n_pages,
            max_pages=self.table.shape[1], fmt=FORMATS[fmt], n_tokens=self.n_tokens,
            max_new=max(max(n for n, _ in seqs), 1) if max_new is None else max_new,
            max_len=max(max(t for _, t in seqs), 1) if max_len is None else max_len,
            k_stride=self.K.stride()[:3], v_stride=self.V.stride()[:3])
        self.d_table, self.d_cu, self.d_lens = self.table.to(device), self.cu.to(device), self.lens.to(device)
        self.status = torch.zeros(1, dtype=torch.int32, device=device)

    def randn(self, *shape):
        return torch.randn(*shape, generator=self.g).bfloat16()

    def cache(self):
        return self.K, self.V, self.K_scale, self.V_scale

    def workspace(self):
        return torch.empty(binding.hga_cache_workspace_bytes(self.p), dtype=torch.uint8, device=self.device)

    def values(self, name):
        """what the pool holds now, float64 [n_pages, hkv, page, d]"""
        t = getattr(self, name)
        if self.fmt == "bf16":
            return f64(t)
        return held(unpack(t.cpu().numpy(), self.fmt), getattr(self, name + "_scale").cpu().numpy(), self.fmt)

    def resident(self, values, i, heads=slice(None)):
        """sequence i's tokens, float64 [hkv, len, d]; a page that is none of the pool's is zeros"""
        n = int(self.lens[i])
        pages = []
        for e in range(-(-n // self.page)):
            j = int(self.table[i, e]) if e < self.table.shape[1] else -1
            pages.append(values[j] if 0 <= j < self.n_pages else np.zeros(values.shape[1:]))
        if not pages:
            return np.zeros((self.hkv, 0, self.d))
        return np.concatenate(pages, 1)[:, :n]

    def new_slots(self):
        """(packed row, page, row of the page) of every new token that has a place"""
        out = []
        for i, (n, t) in enumerate(self.seqs):
            for j in range(n):
                pos = t - n + j
                if pos >= 0 and 0 <= int(self.table[i, pos // self.page]) < self.n_pages:
                    out.append((int(self.cu[i]) + j, int(self.table[i, pos // self.page]), pos % self.page))
        return out

    def attend(self, Q, scale=None):
        """(O, LSE, how far O may be off, how far LSE may be) in 64 bits, row by row; Q bf16 [n_tokens, hq, d]; rows of no sequence NaN.

        O: a probability is rounded to bf16, off by 2^-8 of itself at most, and O divided by the sum of the rounded ones: that moves O by at
        most 2^-8 sum w |v - O| <= 2^-8 (sum w |v| + |O|); O's own rounding adds 2^-8 |O|.  A logit is a sum of d exact products
        in fp32, each addition off by 2^-23 of sum |q k| at most (the tensor pipe cuts off instead of rounding), and so is a sum of up to
        n weighted values; exp2 and the powers that join partial sums are off by 2^-21 together.  A weight below 2^-126 of the row's reference (which is
        2^14 below its largest at most) is zero in fp32: with up to 2^20 keys and values below 2^6 that adds 2^-92 at most.  Quantised pages:
        weights are fp16, whose numbers below 2^-14 are 2^-24 apart, i.e. off by 2^-25; the row's largest is 2^6 or more in the same units, so
        a weight is off by 2^-31 of the largest at most, and O by that times sum |v|.  LSE: the logit's error, the sums'
        and the logarithm's, and its own rounding."""
        q = f64(Q)
        scale = scale or 1 / np.sqrt(self.d)
        O, LSE = np.full(q.shape, np.nan), np.full(q.shape[:2], np.nan)
        tol_O, tol_L = np.zeros(q.shape), np.zeros(q.shape[:2])
        Kv, Vv = self.values("K"), self.values("V")
        G = self.hq // self.hkv
        for i, (n, t) in enumerate(self.seqs):
            K, V = self.resident(Kv, i), self.resident(Vv, i)
            for j in range(n):
                row, end = int(self.cu[i]) + j, t - n + j + 1
                for h in range(self.hq):
                    if end <= 0:
                        O[row, h], LSE[row, h] = 0, -np.inf
                        continue
                    k, v = K[h // G, :end], V[h // G, :end]
                    x = k @ q[row, h] * scale
                    top = x.max()
                    w = np.exp(x - top)
                    LSE[row, h] = top + np.log(w.sum())
                    w /= w.sum()
                    O[row, h] = w @ v
                    size = np.abs(k) @ np.abs(q[row, h]) * scale
                    off = (self.d + 4) * 2.0 ** -23 * size.max() + 2.0 ** -21
                    a = w @ np.abs(v)
                    tol_O[row, h] = 2.0 ** -8 * (a + 2 * np.abs(O[row, h])) + 2 * (off + 2.0 ** -23 * min(end, 4096)) * (a + np.abs(O[row, h])) + 2.0 ** -92
                    if self.fmt != "bf16":
                        tol_O[row, h] += 2.0 ** -31 * w.max() * np.abs(v).sum(0)
                    tol_L[row, h] = 2 * off + 2.0 ** -23 * min(end, 4096) + 2.0 ** -22 * np.abs(LSE[row, h])
        return O, LSE, tol_O, tol_L

    def run_attn(self, Q, lse=True, workspace=None, stream=None, O=None):
        """the library's (O, LSE), rows that it leaves alone filled with 7"""
        O = torch.full_like(Q, 7) if O is None else O
        L = torch.full(Q.shape[:2], 7.0, device=Q.device) if lse else None
        binding.hga_cache_attn(self.p, Q, self.d_cu, self.d_lens, self.d_table, *self.cache(), O, L,
                               self.workspace() if workspace is None else workspace, self.status, stream)
        return O, L

    def check_attn(self, Q, O, LSE):
        want, lse, tol, tol_l = self.attend(Q)
        got = f64(O)
        real = ~np.isnan(lse)
        assert (got[~real] == 7).all(), "rows of no sequence were written"
        bad = np.abs(got - want)[real] > tol[real]
        assert not bad.any() and np.isfinite(got[real]).all(), (
            "%d of %d values of O off, worst %g of what is allowed" % (bad.sum(), bad.size, np.nanmax(np.abs(got - want)[real] / np.maximum(tol[real], 1e-30))))
        if LSE is not None:
            l = f64(LSE)
            assert (l[~real] == 7).all()
            empty = np.isneginf(lse)
            assert (np.isneginf(l) == empty).all()
            fine = real & ~empty
            off = np.abs(l[fine] - lse[fine])
            assert (off <= tol_l[fine]).all(), np.max(off / tol_l[fine])
