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


ROWS, CHUNKS = ([(6, 50), (4, 300)], 2), ([(100, 140), (64, 64)], 4)      # (sequences, query heads): the kernel for few rows, the one for chunks


def out_of_fp16(pr):
    """the first block of V of every sequence's first token far below fp16's range: the step, or the unit, is multiplied as bf16"""
    for i in range(len(pr.seqs)):
        page = int(pr.table[i, 0])
        pr.V_scale[page, :, 0, 0] -= 60


def check_rows(pr, Q, O, LSE, rows):
    """these rows against 64 bits: NaN where it is NaN there, within the tolerances of Problem.attend elsewhere"""
    want, lse, tol, tol_l = pr.attend(Q)
    got, l = T.f64(O)[rows], T.f64(LSE)[rows]
    nan = np.isnan(want[rows])
    assert np.array_equal(np.isnan(got), nan)
    assert (np.abs(got - want[rows])[~nan] <= tol[rows][~nan]).all()
    fine = ~np.isnan(lse[rows])
    assert np.array_equal(~np.isnan(l), fine)
    assert (np.abs(l - lse[rows])[fine] <= tol_l[rows][fine]).all()
    return nan


@pytest.mark.parametrize("seqs,hq", (ROWS, CHUNKS))
@pytest.mark.parametrize("as_bf16", (False, True))
@pytest.mark.parametrize("name", "KV")
def test_nan_codes_that_rows_see(seqs, hq, as_bf16, name):
    """in the history, which all rows see: of V they make their columns NaN, of K everything"""
    pr = Pool(seqs, "mx8", hq=hq, hkv=1, d=64, seed=42)
    if as_bf16:
        out_of_fp16(pr)
    for i, (n, t) in enumerate(seqs):
        if t > n:
            pos = (t - n) // 2
            page = int(pr.table[i, pos // pr.page])
            getattr(pr, name)[page, :, pos % pr.page, 3::7] = 0x7f
            getattr(pr, name)[page, :, pos % pr.page, 5::9] = 0xff
    Q = pr.randn(pr.n_tokens, hq, 64)
    O, LSE = pr.run_attn(Q.cuda())
    nan = check_rows(pr, Q, O, LSE, slice(0, seqs[0][0]))
    assert nan.any() and nan.all() == (name == "K")
    assert int(pr.status.item()) == 0


@pytest.mark.parametrize("seqs,hq", (ROWS, CHUNKS))
@pytest.mark.parametrize("as_bf16", (False, True))
def test_nan_codes_that_rows_do_not_see(seqs, hq, as_bf16):
    """in newer tokens, in the rest of the last page and in pages of nobody: rows ahead of them are what they would be"""
    pr = Pool(seqs, "mx8", hq=hq, hkv=1, d=64, seed=43)
    if as_bf16:
        out_of_fp16(pr)
    used = {(int(pr.table[i, x // pr.page]), x % pr.page) for i, (_, t) in enumerate(seqs) for x in range(t)}
    for page in range(pr.n_pages):
        for r in range(pr.page):
            if (page, r) not in used:
                pr.K[page, :, r] = pr.V[page, :, r] = 0x7f
    slots = {row: (page, r) for row, page, r in pr.new_slots()}
    for i, (n, t) in enumerate(seqs):
        page, r = slots[int(pr.cu[i]) + 2]
        pr.V[page, :, r, 3::7] = 0x7f
        pr.V[page, :, r, 5::9] = 0xff
        page, r = slots[int(pr.cu[i]) + n - 1]
        pr.K[page, :, r, 11] = 0xff
    Q = pr.randn(pr.n_tokens, hq, 64)
    O, LSE = pr.run_attn(Q.cuda())
    nan = check_rows(pr, Q, O, LSE, slice(None))
    for i, (n, t) in enumerate(seqs):
        a = int(pr.cu[i])
        assert not nan[a:a + 2].any()
        assert nan[a + 2:a + n - 1].any(-1).all() and not nan[a + 2:a + n - 1].all()
        assert nan[a + n - 1].all()
    assert int(pr.status.item()) == 0


@pytest.mark.parametrize("fmt", ("mx8", "mx4"))
@pytest.mark.parametrize("seqs,hq", (([(1, 27), (1, 95), (2, 31), (1, 300), (1, 5)], 4), ([(70, 91), (90, 125), (64, 64), (3, 30)], 4)))
def test_slots_behind_a_sequence_change_no_bit(fmt, seqs, hq):
    """whatever the page's owner before left there, scales that fp16 does not hold among it"""
    pr = T.Problem(seqs, fmt, hq=hq, hkv=1, d=64, seed=44)
    Q = pr.randn(pr.n_tokens, hq, 64).cuda()
    used = torch.zeros(pr.n_pages, pr.page, dtype=torch.bool)
    for i, (_, t) in enumerate(seqs):
        for x in range(t):
            used[int(pr.table[i, x // pr.page]), x % pr.page] = True
    free = (~used).cuda()[:, None, :, None]
    first = pr.run_attn(Q)
    for scale in (127, 0, 60, 200, 255):
        for t in (pr.K, pr.V):
            t.copy_(torch.where(free, torch.randint(0, 256, t.shape, generator=pr.g).to(torch.uint8).cuda(), t))
        for t in (pr.K_scale, pr.V_scale):
            t.copy_(torch.where(free, torch.full_like(t, scale), t))
        for a, b in zip(first, pr.run_attn(Q)):
            assert torch.equal(a.view(torch.int16), b.view(torch.int16)), scale


@pytest.mark.parametrize("fmt", ("mx8", "mx4"))
@pytest.mark.parametrize("new,lengths,hq", ((1, (2, 3, 5, 7, 8, 13, 17, 24, 33, 40, 50), 8), (13, (13, 14, 21, 40), 8)))
@pytest.mark.parametrize("what", ("lengths", "zeros", "no page"))
def test_weights_over_quantised_pages_are_fp16(fmt, new, lengths, hq, what):
    """where the scales of the values are in fp16's range: also in the last few keys of a sequence, beside blocks of zeros, and beside pages that are none.

    Values of one size and either sign: O is a difference of weights, so their rounding shows.  Off by 2^-11 of themselves and 2^-31 of the row's
    largest they move O, which is divided by the sum of the rounded ones, by 2^-11 (a + |O|) + 2^-30 n at most, a = sum w |v|; its own rounding adds 2^-8
    |O|; logits, exp2 (2^-18.5) and sums as in Problem.attend."""
    pr = T.Problem([(new, t) for t in lengths], fmt, hq=hq, hkv=1, d=64, page=8, seed=45)
    pr.V.copy_(torch.where(pr.V >= 128, 0xb8, 0x38) if fmt == "mx8" else (pr.V & 0x88) | 0x22)      # +-1
    pr.V_scale.fill_(127)
    if what == "zeros":
        zero = torch.rand(pr.V_scale.shape, generator=pr.g) < 0.3
        pr.V_scale[zero.cuda()] = 0
        pr.V.view(*pr.V_scale.shape, -1)[zero.cuda()] = 0
    if what == "no page":
        pr.table[:, 0] = -1
        pr.d_table = pr.table.cuda()
    Q = pr.randn(pr.n_tokens, hq, 64)
    O, LSE = pr.run_attn(Q.cuda())
    want, lse, _, _ = pr.attend(Q)
    Kv, Vv = pr.values("K"), pr.values("V")
    for i, t in enumerate(lengths):
        K, V = pr.resident(Kv, i)[0], pr.resident(Vv, i)[0]
        for j in range(new):
            row, end = i * new + j, t - new + j + 1
            q = T.f64(Q[row])
            a = np.exp(q @ K[:end].T / 8 - lse[row][:, None]) @ np.abs(V[:end])
            off = 68 * 2.0 ** -23 * (np.abs(q) @ np.abs(K[:end]).T / 8).max() + 2.0 ** -18.5 + 2.0 ** -23 * end
            tol = 2.0 ** -11 * (a + np.abs(want[row])) + 2.0 ** -30 * end + 2.0 ** -8 * np.abs(want[row]) + 2 * off * (a + np.abs(want[row]))
            assert (np.abs(T.f64(O[row]) - want[row]) <= tol).all()


@pytest.mark.parametrize("fmt", ("mx8", "mx4"))
@pytest.mark.parametrize("seqs,hq", (ROWS, CHUNKS))
@pytest.mark.parametrize("up", (110, 116, 118, 122))
@pytest.mark.parametrize("small_keys", (False, True))
def test_queries_next_to_the_end_of_bf16(fmt, seqs, hq, up, small_keys):
    """logits are of ordinary size by softmax_scale, or by it and keys that are small in turn (none below 2^-118)"""
    pr = T.Problem(seqs, fmt, hq=hq, hkv=1, d=64, seed=46)
    Q = (pr.randn(pr.n_tokens, hq, 64).float() * 2.0 ** up).bfloat16()
    assert torch.isfinite(Q).all()
    down = min(up, 100 if fmt == "mx8" else 114) if small_keys else 0
    pr.K_scale -= down
    scale = pr.p.softmax_scale = 2.0 ** (down - up - 3)
    O, LSE = pr.run_attn(Q.cuda())
    want, lse, tol, tol_l = pr.attend(Q, scale)
    assert (np.abs(T.f64(O) - want) <= tol).all() and (np.abs(T.f64(LSE) - lse) <= tol_l).all()
    assert tol.max() < 0.1 and int(pr.status.item()) == 0


@pytest.mark.parametrize("fmt", ("bf16", "mx8", "mx4"))
def test_summaries_straight_behind_a_read_back(fmt):
    """write, read back and summaries one straight behind the other, with other contents every time, against the same calls with a wait after each"""
    from paper_2607_15105_b200.workloads import HgaConfig
    hkv, d, total, n = 2, 128, 512, 24
    cfg = HgaConfig("cache", batch=2, n_q_heads=4, n_kv_heads=hkv, head_dim=d, total_len=total, seg_len=64, chunk=64, group=8, q_block=64,
                    topk_chunks=2, topk_groups=2, sink=64, local=64, topics=4, needles=0, backward=False, seed=1)
    pr = T.Problem([(total, total), (total, total)], fmt, hq=4, hkv=hkv, d=d, page=64, seed=51)
    new = pr.randn(n, 2 * total, hkv, d).cuda()
    bufs = [[binding.HgaLayerBuffers(cfg, backward=False) for _ in range(n)] for _ in range(2)]
    dense = torch.zeros(2, hkv, total, d, dtype=torch.bfloat16, device="cuda")

    def step(i, buf, wait):
        binding.hga_cache_write(pr.p, new[i], None, pr.d_cu, pr.d_lens, pr.d_table, pr.K, None, pr.K_scale, None, pr.status)
        wait()
        binding.hga_cache_read(pr.p, 0, total, pr.d_lens, pr.d_table, pr.K, None, pr.K_scale, None, dense, None, pr.status)
        wait()
        buf.build_summaries(dense, 0, total)
        wait()

    torch.cuda.synchronize()
    for i in range(n):
        step(i, bufs[0][i], lambda: None)
    torch.cuda.synchronize()
    for i in range(n):
        step(i, bufs[1][i], torch.cuda.synchronize)
    for a, b in zip(*bufs):
        assert torch.equal(a.chunk_sum.view(torch.int16), b.chunk_sum.view(torch.int16)) and a.chunk_sum.abs().max() > 0
        assert torch.equal(a.group_sum.view(torch.int16), b.group_sum.view(torch.int16))
    # the mean of what is held, rounded once
    k = T.f64(dense).reshape(2, hkv, total // 8, 8, d).mean(3)
    assert (np.abs(T.f64(bufs[1][n - 1].group_sum) - k) <= 2.0 ** -8 * np.abs(k)).all()
    assert int(pr.status.item()) == 0


def test_a_unit_that_takes_longer_than_a_bounded_wait():
    """1.7 10^8 keys in one unit: all but the last 4096 are the same page, with next to no weight, so only those count"""
    heads, page, d, new, pages = 148, 4096, 64, 64, 40960
    g = torch.Generator(device="cuda").manual_seed(52)
    K, V = (torch.randn(2, heads, page, d, generator=g, device="cuda").bfloat16() for _ in "KV")
    K[0], V[0] = -8, 0                                                       # logits near -64, against -5 to 5
    Q = (1 + 0.1 * torch.randn(new, heads, d, generator=g, device="cuda")).bfloat16()
    table = torch.zeros(1, pages, dtype=torch.int32, device="cuda")
    table[0, -1] = 1
    p = binding.make_cache_params(1, heads, heads, d, page, 2, pages, binding.HGA_CACHE_BF16, new, new)
    assert binding.hga_cache_workspace_bytes(p) == 0                         # (no unit is shared out)
    cu, lens = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, new], [pages * page]))
    O, LSE = torch.zeros_like(Q), torch.zeros(new, heads, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    start.record()
    binding.hga_cache_attn(p, Q, cu, lens, table, K, V, None, None, O, LSE, None, status)
    end.record()
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    assert start.elapsed_time(end) > 1000 * 2 ** 30 / 1.965e9                # longer than the waits' 2^30 cycles
    hidden = torch.arange(page, device="cuda")[None] > page - new + torch.arange(new, device="cuda")[:, None]
    for h in range(0, heads, 37):
        q, k, v = Q[:, h].double(), K[1, h].double(), V[1, h].double()
        x = (q @ k.T / 8).masked_fill(hidden, -np.inf)
        lse = torch.logsumexp(x, -1)
        w = torch.exp(x - lse[:, None])
        want, a = w @ v, w @ v.abs()
        off = 68 * 2.0 ** -23 * (q.abs() @ k.abs().T / 8).amax(-1) + 2.0 ** -18.5
        # (as Problem.attend; the pages before add exp(-59) 1.7 10^8 < 2^-57 to a weight of one)
        tol = 2.0 ** -8 * (a + 2 * want.abs()) + 2 * (off + 2.0 ** -23 * 4096)[:, None] * (a + want.abs())
        assert ((O[:, h].double() - want).abs() <= tol).all()
        assert ((LSE[:, h].double() - lse).abs() <= 2 * off + 2.0 ** -23 * 4096 + 2.0 ** -22 * lse.abs()).all()


@pytest.mark.parametrize("fmt", ("bf16", "mx8", "mx4"))
@pytest.mark.parametrize("seqs,hq", (([(1, 60), (2, 300), (1, 2000)], 4), ([(70, 250), (64, 64)], 4)))
def test_values_up_to_the_stated_size(fmt, seqs, hq):
    """keys times the largest value just below 2^108; and beyond it, in one sequence, which leaves the others as they are"""
    pr = T.Problem(seqs, fmt, hq=hq, hkv=1, d=64, seed=47)
    most = max(t for _, t in seqs)
    ordinary = pr.V.clone(), None if fmt == "bf16" else pr.V_scale.clone()
    Q = pr.randn(pr.n_tokens, hq, 64)
    plain = pr.run_attn(Q.cuda())
    up = int(np.floor(np.log2(2.0 ** 108 / most / np.abs(pr.values("V")).max())))
    if fmt == "bf16":
        pr.V.mul_(2.0 ** up)
    else:
        pr.V_scale += up
    assert 2.0 ** 107 / 2 < np.abs(pr.values("V")).max() * most < 2.0 ** 108
    O, LSE = pr.run_attn(Q.cuda())
    pr.check_attn(Q, O, LSE)
    pr.V.copy_(ordinary[0])
    if fmt != "bf16":
        pr.V_scale.copy_(ordinary[1])
    for page in pr.table[0][pr.table[0] >= 0].tolist():
        if fmt == "bf16":
            pr.V[page] *= 2.0 ** 124
        else:
            pr.V_scale[page] += 110
    O, LSE = pr.run_attn(Q.cuda())
    n = seqs[0][0]
    assert torch.equal(O[n:].view(torch.int16), plain[0][n:].view(torch.int16)) and torch.equal(LSE[n:], plain[1][n:])
    assert int(pr.status.item()) == 0


@pytest.mark.parametrize("fmt", ("mx8", "mx4"))
@pytest.mark.parametrize("seqs,hq", (ROWS, CHUNKS))
def test_keys_up_to_the_stated_size(fmt, seqs, hq):
    """just below 2^100, against queries that are small in turn, and against ordinary ones under a small softmax_scale"""
    pr = T.Problem(seqs, fmt, hq=hq, hkv=1, d=64, seed=53)
    up = int(np.floor(np.log2(2.0 ** 100 / np.abs(pr.values("K")).max())))
    pr.K_scale += up
    for down in (up, 0):
        Q = (pr.randn(pr.n_tokens, hq, 64).float() * 2.0 ** -down).bfloat16()
        scale = pr.p.softmax_scale = 2.0 ** (down - up - 3)
        O, LSE = pr.run_attn(Q.cuda())
        want, lse, tol, tol_l = pr.attend(Q, scale)
        assert (np.abs(T.f64(O) - want) <= tol).all() and (np.abs(T.f64(LSE) - lse) <= tol_l).all()
    assert int(pr.status.item()) == 0


@pytest.mark.parametrize("fmt,low,high", (("mx8", 109, 128), ("mx4", 111, 136)))
@pytest.mark.parametrize("new,lengths", ((1, (2, 3, 5, 8, 24, 40)), (13, (13, 14, 21, 40))))
def test_the_range_of_scales_with_fp16_weights(fmt, low, high, new, lengths):
    """2^-18 to 2^1 in e4m3 and 2^-16 to 2^9 in e2m1, of keys and values; tolerance as in the test of that rounding"""
    for code in (low, high):
        pr = T.Problem([(new, t) for t in lengths], fmt, hq=8, hkv=1, d=64, page=8, seed=54)
        pr.V.copy_(torch.where(pr.V >= 128, 0xb8, 0x38) if fmt == "mx8" else (pr.V & 0x88) | 0x22)      # +-1
        pr.V_scale.fill_(code)
        pr.K_scale.fill_(code)
        size = np.abs(pr.values("K")).max()
        Q = (pr.randn(pr.n_tokens, 8, 64).float() * (4 / size)).bfloat16()
        O, LSE = pr.run_attn(Q.cuda())
        want, lse, _, _ = pr.attend(Q)
        Kv, Vv = pr.values("K"), pr.values("V")
        for i, t in enumerate(lengths):
            K, V = pr.resident(Kv, i)[0], pr.resident(Vv, i)[0]
            for j in range(new):
                row, end = i * new + j, t - new + j + 1
                q = T.f64(Q[row])
                a = np.exp(q @ K[:end].T / 8 - lse[row][:, None]) @ np.abs(V[:end])
                off = 68 * 2.0 ** -23 * (np.abs(q) @ np.abs(K[:end]).T / 8).max() + 2.0 ** -18.5 + 2.0 ** -23 * end
                tol = 2.0 ** -11 * (a + np.abs(want[row])) + 2.0 ** -30 * end * 2.0 ** (code - 127) + 2.0 ** -8 * np.abs(want[row]) + 2 * off * (a + np.abs(want[row]))
                assert (np.abs(T.f64(O[row]) - want[row]) <= tol).all()


@pytest.mark.parametrize("fmt", ("bf16", "mx8", "mx4"))
@pytest.mark.parametrize("new,length,others,hq", (
    (1, 900, ((2, 800, 1, 300), (1, 70, 2, 7), (0, 0, 3, 1000)), 8), (1, 100, ((1, 80, 1, 90), (2, 2, 0, 50), (0, 5, 2, 100)), 8),
    (70, 400, ((30, 390, 40, 40), (70, 90, 0, 400), (1, 1, 69, 300)), 4)))
def test_neighbours_change_no_bit(fmt, new, length, others, hq):
    """one sequence beside others of other lengths and contents, in another place of the batch, with the same n_seq, n_tokens, max_new and max_len"""
    g = torch.Generator().manual_seed(48)
    q = torch.randn(new, hq, 64, generator=g).bfloat16()
    first = None
    for at in (0, 1, 2):
        for a, ta, b, tb in others:
            seqs = [(a, ta), (b, tb)]
            seqs.insert(at, (new, length))
            pr = T.Problem(seqs, fmt, hq=hq, hkv=1, d=64, seed=49 + at, max_new=max(new, 3), max_len=1000)
            table = torch.full((3, 63), -7, dtype=torch.int32)                # (the same limits every time)
            table[:, :pr.table.shape[1]] = pr.table
            pr.table, pr.d_table, pr.p.max_pages = table, table.cuda(), 63
            # the sequence's own tokens, the same every time
            own = torch.Generator().manual_seed(50)
            for t in pr.cache():
                if t is None:
                    continue
                for e in range(-(-length // pr.page)):
                    page = int(pr.table[at, e])
                    if t.dtype == torch.bfloat16:
                        t[page] = torch.randn(t[page].shape, generator=own).bfloat16()
                    elif t.shape[-1] == 2:
                        t[page] = torch.randint(118, 124, t[page].shape, generator=own).to(torch.uint8)
                    else:
                        t[page] = torch.randint(0, 126, t[page].shape, generator=own).to(torch.uint8)
            Q = pr.randn(pr.n_tokens, hq, 64)
            row = int(pr.cu[at])
            Q[row:row + new] = q
            O, LSE = pr.run_attn(Q.cuda())
            got = O[row:row + new].clone(), LSE[row:row + new].clone()
            assert torch.isfinite(got[0]).all()
            if first is None:
                first = got
            assert torch.equal(first[0].view(torch.int16), got[0].view(torch.int16)) and torch.equal(first[1], got[1]), (at, seqs)
            assert int(pr.status.item()) == 0


