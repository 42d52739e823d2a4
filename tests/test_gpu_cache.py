"""The paged cache on the GPU against its plain statement in 64 bits (cache_testlib): what is written and read back bit for bit, attention
within the tolerances derived there."""
import numpy as np
import pytest
import torch

import cache_testlib as T
from paper_2607_15105_b200 import binding

pytestmark = pytest.mark.gpu
FMTS = ("bf16", "mx8", "mx4")


def tricky(pr, *shape):
    """numbers of every size, zeros, subnormal blocks, borders between two codes"""
    x = pr.randn(*shape)
    flat = x.view(-1, 32)
    n = flat.shape[0]
    exps = torch.randint(-60, 60, (n, 1), generator=pr.g)
    flat.mul_(torch.exp2(exps.float()).bfloat16())
    flat[0] = 0
    flat[1 % n] = torch.arange(32).bfloat16() * 2.0 ** -133                 # bf16's smallest
    flat[2 % n] = (torch.arange(32) - 16).bfloat16() * 0.25                 # halves of e2m1's steps
    flat[3 % n, 3] = 3.3895313892515355e38                                  # the largest bf16 number
    flat[4 % n, 0] = 448.0
    flat[5 % n, 7] = -456.0
    flat[6 % n] = (torch.arange(32) * 0.0625 + 1).bfloat16()                # ties of e4m3
    flat[7 % n] = -0.0
    return x


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("d,hkv,page,order,seqs", [
    (64, 2, 16, "head", [(1, 1), (3, 20), (5, 5)]),
    (128, 3, 8, "token", [(7, 33), (1, 64), (0, 12), (17, 17)]),
    (128, 8, 48, "head", [(100, 100)]),
    (64, 1, 128, "token", [(1, 129)] * 9)])
def test_write_then_read_bit_for_bit(fmt, d, hkv, page, order, seqs):
    pr = T.Problem(seqs, fmt, hq=hkv, hkv=hkv, d=d, page=page, seed=5, order=order, spare_rows=2)
    K, V = tricky(pr, pr.n_tokens, hkv, d), tricky(pr, pr.n_tokens, hkv, d)
    want = {}
    for name, x in (("K", K), ("V", V)):
        t = getattr(pr, name).cpu().clone()
        sc = None if fmt == "bf16" else getattr(pr, name + "_scale").cpu().clone()
        for row, pg, r in pr.new_slots():
            if fmt == "bf16":
                t[pg, :, r] = x[row]
            else:
                codes, scales = T.quantise(T.f64(x[row]), fmt)
                t[pg, :, r], sc[pg, :, r] = torch.from_numpy(T.pack(codes, fmt)), torch.from_numpy(scales)
        want[name] = t, sc
    binding.hga_cache_write(pr.p, K.cuda(), V.cuda(), pr.d_cu, pr.d_lens, pr.d_table, *pr.cache(), pr.status)
    for name in "KV":
        t, sc = want[name]
        got = getattr(pr, name).cpu()
        if fmt == "bf16":
            assert torch.equal(got.view(torch.int16), t.contiguous().view(torch.int16))
        else:
            assert torch.equal(getattr(pr, name + "_scale").cpu(), sc)
            assert torch.equal(got, t)
    most = max(t for _, t in seqs)
    for begin, end in ((0, most), (3, max(most - 2, 3)), (most + 1, most + 9)):
        out = {n: torch.full((len(seqs), hkv, end - begin, d), 9.0, dtype=torch.bfloat16, device="cuda") for n in "KV"}
        binding.hga_cache_read(pr.p, begin, end, pr.d_lens, pr.d_table, *pr.cache(), out["K"], out["V"], pr.status)
        for name in "KV":
            values = pr.values(name)
            for i, (_, t) in enumerate(seqs):
                real = pr.resident(values, i)[:, begin:min(t, end)]
                got = T.f64(out[name][i])
                assert np.array_equal(got[:, :real.shape[1]], real), name
                assert (got[:, real.shape[1]:] == 9).all(), "rows behind the sequence were written"
    assert int(pr.status.item()) == 0


@pytest.mark.parametrize("fmt", FMTS)
def test_only_keys_or_only_values_and_strides(fmt):
    pr = T.Problem([(4, 9), (2, 30)], fmt, hq=2, hkv=2, d=64, seed=2)
    before = pr.K.cpu().clone()
    # new values inside a wider tensor, read back into one
    wide = pr.randn(pr.n_tokens, 2, 3, 64).cuda()
    V = wide[:, :, 1]
    pr.p.vn_stride[:] = V.stride()[:2]
    binding.hga_cache_write(pr.p, None, V, pr.d_cu, pr.d_lens, pr.d_table, None, pr.V, None, pr.V_scale, pr.status)
    assert torch.equal(pr.K.cpu(), before)
    out = torch.full((2, 30, 2, 128), 9.0, dtype=torch.bfloat16, device="cuda")
    O = out.transpose(1, 2)[..., 64:]
    pr.p.out_stride[:] = O.stride()[:3]
    binding.hga_cache_read(pr.p, 0, 30, pr.d_lens, pr.d_table, None, pr.V, None, pr.V_scale, None, O, pr.status)
    values = pr.values("V")
    for i, t in enumerate((9, 30)):
        assert np.array_equal(T.f64(O[i])[:, :t], pr.resident(values, i))
        assert (T.f64(O[i])[:, t:] == 9).all()
    assert (T.f64(out[..., :64]) == 9).all()
    for i, (n, t) in enumerate(((4, 9), (2, 30))):
        got = pr.resident(values, i)[:, t - n:]
        x = T.f64(V.cpu())[int(pr.cu[i]):int(pr.cu[i]) + n].transpose(1, 0, 2)
        assert np.array_equal(got, x if fmt == "bf16" else T.held(*T.quantise(x, fmt), fmt))


@pytest.mark.parametrize("fmt", ("mx8", "mx4"))
def test_blocks_with_infinities_read_back_as_nan(fmt):
    pr = T.Problem([(3, 3)], fmt, hq=1, hkv=1, d=64, seed=3)
    K = pr.randn(3, 1, 64)
    K[0, 0, 5], K[1, 0, 40], K[2, 0, 63] = float("inf"), float("nan"), -float("inf")
    binding.hga_cache_write(pr.p, K.cuda(), None, pr.d_cu, pr.d_lens, pr.d_table, pr.K, None, pr.K_scale, None, pr.status)
    out = torch.zeros(1, 1, 3, 64, dtype=torch.bfloat16, device="cuda")
    binding.hga_cache_read(pr.p, 0, 3, pr.d_lens, pr.d_table, pr.K, None, pr.K_scale, None, out, None, pr.status)
    nan = torch.isnan(out[0, 0]).cpu()
    want = torch.zeros(3, 64, dtype=torch.bool)
    want[0, :32] = want[1, 32:] = want[2, 32:] = True
    assert torch.equal(nan, want)


def test_write_leaves_out_what_has_no_place():
    """more new tokens than resident ones, a page that is none, limits that cu_q and seq_lens pass"""
    pr = T.Problem([(5, 3), (4, 40), (2, 10)], "bf16", hq=1, hkv=1, d=64, page=8, seed=4)
    pr.table[1, 4] = pr.n_pages                                             # where tokens 32..39 would lie
    pr.d_table = pr.table.cuda()
    K = pr.randn(pr.n_tokens, 1, 64)
    want = pr.K.cpu().clone()
    for row, pg, r in pr.new_slots():
        want[pg, :, r] = K[row]
    binding.hga_cache_write(pr.p, K.cuda(), None, pr.d_cu, pr.d_lens, pr.d_table, pr.K, None, None, None, pr.status)
    assert torch.equal(pr.K.cpu().view(torch.int16), want.view(torch.int16))
    assert int(pr.status.item()) == binding.HGA_STATUS_BAD_INDEX
    # limits
    for change in (dict(max_new=3), dict(max_len=38)):
        pr = T.Problem([(2, 9), (4, 40)], "bf16", hq=1, hkv=1, d=64, page=8, seed=4, **change)
        K = pr.randn(pr.n_tokens, 1, 64)
        want = pr.K.cpu().clone()
        for row, pg, r in pr.new_slots():
            pos = 36 + row - 2
            if row < 2 or (row - 2 < pr.p.max_new and pos < pr.p.max_len):
                want[pg, :, r] = K[row]
        binding.hga_cache_write(pr.p, K.cuda(), None, pr.d_cu, pr.d_lens, pr.d_table, pr.K, None, None, None, pr.status)
        assert torch.equal(pr.K.cpu().view(torch.int16), want.view(torch.int16)), change
        assert int(pr.status.item()) == binding.HGA_STATUS_BAD_INDEX


# ----------------------------------------------------------------------------- attention

ATTN = [
    # (seqs, hq, hkv, d, page)
    ([(1, 1)], 1, 1, 64, 8),
    ([(1, 8)], 4, 1, 128, 8),
    ([(1, 257), (1, 256), (1, 255)], 8, 2, 128, 16),
    ([(1, 130)] * 3, 9, 1, 64, 128),                       # nine rows: two tiles of eight, or one of sixteen
    ([(2, 2), (5, 300), (1, 77)], 7, 1, 128, 48),
    ([(3, 200), (0, 50), (4, 4), (1, 1)], 6, 2, 64, 16),
    ([(16, 16)], 2, 1, 128, 16),
    ([(33, 161)], 4, 2, 64, 64),
    ([(40, 40), (64, 200)], 4, 1, 128, 24),
    ([(130, 130)], 2, 2, 64, 16),
    ([(70, 400), (1, 9), (129, 260)], 3, 1, 128, 8),
    ([(150, 700)], 5, 1, 64, 32),
    ([(300, 300)], 1, 1, 128, 4096),
    ([(9, 1500)], 16, 1, 64, 16),                          # keys in several parts
    ([(1, 3001), (1, 700)], 2, 1, 128, 16),
    ([(5, 5), (200, 1100)], 12, 2, 128, 64),
    ([(3, 140)], 128, 1, 64, 16),                          # one key/value head for 128 query heads
]


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("case", range(len(ATTN)))
def test_attention(fmt, case):
    seqs, hq, hkv, d, page = ATTN[case]
    pr = T.Problem(seqs, fmt, hq=hq, hkv=hkv, d=d, page=page, seed=case, order="token" if case % 3 == 1 else "head", spare_rows=case % 2)
    Q = pr.randn(pr.n_tokens, hq, d)
    O, LSE = pr.run_attn(Q.cuda())
    pr.check_attn(Q, O, LSE)
    assert int(pr.status.item()) == 0
    again, _ = pr.run_attn(Q.cuda(), lse=False)
    assert torch.equal(O.view(torch.int16), again.view(torch.int16))


@pytest.mark.parametrize("fmt", ("bf16", "mx4"))
@pytest.mark.parametrize("n_seq,most", ((40, 90), (600, 90), (40, 3), (1500, 2)))
def test_many_sequences(fmt, n_seq, most):
    """sequences without new tokens among them; more than a warp, a block and 32 x 32 of them"""
    r = np.random.RandomState(n_seq)
    seqs = [(int(r.choice((0, 0, 1, 2))), int(r.randint(2, 40))) for _ in range(n_seq)]
    seqs[n_seq // 3], seqs[n_seq - 2], seqs[5] = (most, most + 50), (most - 1, most + 1), (0, 0)
    pr = T.Problem(seqs, fmt, hq=2, hkv=1, d=64, page=8, seed=21)
    K, V = pr.randn(pr.n_tokens, 1, 64), pr.randn(pr.n_tokens, 1, 64)
    binding.hga_cache_write(pr.p, K.cuda(), V.cuda(), pr.d_cu, pr.d_lens, pr.d_table, *pr.cache(), pr.status)
    values = pr.values("K")
    for row, pg, slot in pr.new_slots():
        x = T.f64(K[row, 0])
        assert np.array_equal(values[pg, 0, slot], x if fmt == "bf16" else T.held(*T.quantise(x[None], fmt), fmt)[0])
    Q = pr.randn(pr.n_tokens, 2, 64)
    O, LSE = pr.run_attn(Q.cuda())
    pr.check_attn(Q, O, LSE)
    assert int(pr.status.item()) == 0


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("new,length,parts", ((20, 7000, 2), (40, 9000, None), (56, 16000, 2), (37, 5000, None), (8, 3000, None), (64, 2000, 0)))
def test_chunks_whose_keys_are_shared_out(fmt, new, length, parts):
    """one sequence whose units are fewer than SMs, or leave a part of them idle in the last round: two uneven parts, several even ones, none.
    128 query heads per key/value head make a unit of two tokens."""
    hq, hkv, d = 1024, 8, 64
    pr = T.Problem([(new, length)], fmt, hq=hq, hkv=hkv, d=d, page=64, seed=32)
    need = binding.hga_cache_workspace_bytes(pr.p)
    if parts is None:
        assert need > 0
    else:
        units = (new + 1) // 2
        tokens = min((units - units * hkv // 148 * 148 // hkv) * 2, new)      # of the units that are shared out
        assert need == parts * tokens * hq * (d + 4) * 4
    Q = pr.randn(new, hq, d)
    O, LSE = pr.run_attn(Q.cuda())
    assert int(pr.status.item()) == 0
    # as Problem.attend, a key/value head at a time, with matrix products in 64 bits; tolerances as there
    K, V = (torch.from_numpy(pr.resident(pr.values(n), 0)).cuda() for n in "KV")
    hidden = torch.arange(length, device="cuda")[None] > length - new + torch.arange(new, device="cuda")[:, None]
    for h in range(hkv):
        q = Q[:, h * 128:(h + 1) * 128].cuda().double()
        x = (q @ K[h].T / 8).masked_fill(hidden[:, None], -np.inf)
        lse = torch.logsumexp(x, -1)
        w = torch.exp(x - lse[..., None])
        want, a = w @ V[h], w @ V[h].abs()
        size = (q.abs() @ K[h].abs().T / 8).masked_fill(hidden[:, None], 0).amax(-1)
        off = (d + 4) * 2.0 ** -23 * size + 2.0 ** -21
        tol = 2.0 ** -8 * (a + 2 * want.abs()) + 2 * (off + 2.0 ** -23 * 4096)[..., None] * (a + want.abs()) + 2.0 ** -92
        if fmt != "bf16":
            tol += 2.0 ** -31 * w.amax(-1)[..., None] * V[h].abs().sum(0)
        got = O[:, h * 128:(h + 1) * 128].double()
        assert ((got - want).abs() <= tol).all(), ((got - want).abs() / tol).max()
        tol_l = 2 * off + 2.0 ** -23 * 4096 + 2.0 ** -22 * lse.abs()
        assert ((LSE[:, h * 128:(h + 1) * 128].double() - lse).abs() <= tol_l).all()


@pytest.mark.parametrize("fmt", FMTS)
def test_kernels_are_the_ones_meant(fmt):
    """tiles of 16 rows for few of them, of 128 for more; parts joined in a cluster or by a kernel of its own"""
    for new, length, hq, rows, tensor in ((1, 100, 8, 1, 0), (1, 700, 8, 1, 0), (1, 9000, 8, 2, 0), (12, 300, 4, 1, 0), (70, 300, 4, 0, 1), (70, 9000, 4, 1, 1)):
        pr = T.Problem([(new, length)], fmt, hq=hq, hkv=1, d=64, page=64, seed=22)
        Q = pr.randn(pr.n_tokens, hq, 64).cuda()
        before = binding.hga_kernel_launch_counts()
        pr.run_attn(Q)
        ran = [b - a for a, b in zip(before, binding.hga_kernel_launch_counts())]
        assert ran[binding.HGA_KERNELS_CACHE_ROWS] == rows and ran[binding.HGA_KERNELS_CACHE_TENSOR] == tensor, (new, length, ran)
        assert sum(ran) == rows + tensor


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("seqs", ([(4, 2), (3, 0), (2, 300), (6, 5)], [(200, 90), (70, 0), (130, 300)]))
def test_rows_without_keys(fmt, seqs):
    pr = T.Problem(seqs, fmt, hq=4, hkv=2, d=64, seed=8, max_len=400)
    Q = pr.randn(pr.n_tokens, 4, 64)
    O, LSE = pr.run_attn(Q.cuda())
    pr.check_attn(Q, O, LSE)
    assert int(pr.status.item()) == 0


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("seqs,hq", (([(6, 50), (4, 300)], 2), ([(100, 140), (64, 64)], 4)))
def test_what_a_row_does_not_see_has_no_influence(fmt, seqs, hq):
    """NaN and infinities in keys and values behind a row, in the rest of its last page and in pages of nobody"""
    d = 64
    pr = T.Problem(seqs, fmt, hq=hq, hkv=1, d=d, seed=9)
    Q = pr.randn(pr.n_tokens, hq, d)
    # unwritten slots: all bits set
    used = set()
    for i, (_, t) in enumerate(seqs):
        used |= {(int(pr.table[i, x // pr.page]), x % pr.page) for x in range(t)}
    for pg in range(pr.n_pages):
        for r in range(pr.page):
            if (pg, r) not in used:
                for t in pr.cache():
                    if t is not None:
                        t[pg, :, r] = float("nan") if fmt == "bf16" else 255
    # the newest tokens but one are not finite
    slots = {row: (pg, r) for row, pg, r in pr.new_slots()}
    for i, (n, t) in enumerate(seqs):
        for back, name, value in ((1, "K", float("nan")), (2, "V", float("inf")), (2, "K", float("-inf")), (n - 2, "V", float("nan"))):
            pg, r = slots[int(pr.cu[i]) + n - back]
            if fmt == "bf16":
                getattr(pr, name)[pg, :, r, 3::7] = value
            else:
                getattr(pr, name + "_scale")[pg, :, r, 0] = 255
    O, LSE = pr.run_attn(Q.cuda())
    want, lse, tol, tol_l = pr.attend(Q)
    got = T.f64(O)
    for i, (n, t) in enumerate(seqs):
        clean = slice(int(pr.cu[i]), int(pr.cu[i]) + 2)                      # these see none of it
        assert np.isfinite(want[clean]).all()
        assert (np.abs(got - want)[clean] <= tol[clean]).all()
        middle = slice(int(pr.cu[i]) + 2, int(pr.cu[i]) + n - 2)            # these see one value that is NaN in some columns
        for row in range(middle.start, middle.stop):
            nan = np.isnan(want[row])
            assert nan.any() and not nan.all()
            assert np.isnan(got[row][nan]).all()
            assert (np.abs(got - want)[row][~nan] <= tol[row][~nan]).all()
            assert (np.abs(T.f64(LSE)[row] - lse[row]) <= tol_l[row]).all()
        assert np.isnan(got[int(pr.cu[i]) + n - 1]).any()


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("seqs", ([(2, 100), (1, 40)], [(90, 200), (40, 40)]))
def test_pages_that_are_none_count_as_zeros(fmt, seqs):
    pr = T.Problem(seqs, fmt, hq=4, hkv=1, d=128, seed=10, page=16)
    pr.table[0, 2], pr.table[0, 5], pr.table[1, 0] = -1, pr.n_pages, 0x7fffffff
    pr.d_table = pr.table.cuda()
    Q = pr.randn(pr.n_tokens, 4, 128)
    O, LSE = pr.run_attn(Q.cuda())
    pr.check_attn(Q, O, LSE)
    assert int(pr.status.item()) == binding.HGA_STATUS_BAD_INDEX
    out = torch.full((2, 1, 100, 128), 9.0, dtype=torch.bfloat16, device="cuda")
    pr.status.zero_()
    binding.hga_cache_read(pr.p, 0, 100, pr.d_lens, pr.d_table, *pr.cache(), out, None, pr.status)
    n = min(100, seqs[0][1])
    assert np.array_equal(T.f64(out[0])[:, :n], pr.resident(pr.values("K"), 0)[:, :n])
    assert int(pr.status.item()) == binding.HGA_STATUS_BAD_INDEX


@pytest.mark.parametrize("seqs", ([(2, 90), (3, 50)], [(70, 90), (66, 200)]))
def test_limits_hold(seqs):
    """what cu_q and seq_lens say beyond max_new and max_len is left out and reported"""
    n1 = seqs[1][0]
    pr = T.Problem(seqs, "bf16", hq=4, hkv=2, d=64, seed=12, max_new=n1 - 1)
    Q = pr.randn(pr.n_tokens, 4, 64)
    O, LSE = pr.run_attn(Q.cuda())
    want, lse, tol, tol_l = pr.attend(Q)
    got = T.f64(O)
    for i, (n, _) in enumerate(seqs):
        a, m = int(pr.cu[i]), min(n, n1 - 1)
        assert (np.abs(got - want)[a:a + m] <= tol[a:a + m]).all()
        assert (got[a + m:a + n] == 7).all() and (T.f64(LSE)[a + m:a + n] == 7).all()
    assert int(pr.status.item()) == binding.HGA_STATUS_BAD_INDEX
    # keys at or behind max_len
    pr = T.Problem(seqs, "bf16", hq=4, hkv=2, d=64, seed=12, max_len=seqs[1][1] - 5)
    Q = pr.randn(pr.n_tokens, 4, 64)
    O, LSE = pr.run_attn(Q.cuda())
    values = pr.values("K"), pr.values("V")
    i, (n, t) = 1, seqs[1]
    K, V = (pr.resident(v, i) for v in values)
    for j in range(n):
        end = min(t - n + j + 1, t - 5)
        for h in range(4):
            x = K[h // 2, :end] @ T.f64(Q)[int(pr.cu[1]) + j, h] / 8
            w = np.exp(x - x.max())
            o = w @ V[h // 2, :end] / w.sum()
            assert np.abs(T.f64(O)[int(pr.cu[1]) + j, h] - o).max() < 0.05
    assert int(pr.status.item()) == binding.HGA_STATUS_BAD_INDEX


@pytest.mark.parametrize("cu", ([0, 9, 4, 12], [-3, 4, 8, 12], [0, 4, 8, 99], [5, 5, 5, 5], [0, 0x7fffffff, -0x7fffffff, 12]))
@pytest.mark.parametrize("op", ("write", "attn"))
def test_broken_prefix_sums_stay_inside(cu, op):
    """no result is promised for these, but nothing outside the tensors is touched and the call returns"""
    pr = T.Problem([(4, 30), (4, 40), (4, 20)], "mx8", hq=32, hkv=2, d=64, seed=13, max_new=12)
    pr.d_cu = torch.tensor(cu, dtype=torch.int32, device="cuda")
    pr.d_lens = torch.tensor([30, -5, 0x7fffffff], dtype=torch.int32, device="cuda")
    pr.p.max_len = 48
    if op == "write":
        guard = [torch.full((64, 2, 64), 3.0, dtype=torch.bfloat16, device="cuda") for _ in "KV"]
        binding.hga_cache_write(pr.p, guard[0], guard[1], pr.d_cu, pr.d_lens, pr.d_table, *pr.cache(), pr.status)
    else:
        O = torch.full((64, 32, 64), 7.0, dtype=torch.bfloat16, device="cuda")
        Q = pr.randn(64, 32, 64).cuda()
        pr.run_attn(Q, O=O)
        assert (O[12:] == 7).all()
    torch.cuda.synchronize()
    assert int(pr.status.item()) == binding.HGA_STATUS_BAD_INDEX


def test_lengths_below_zero_are_read_as_none():
    pr = T.Problem([(4, 30), (4, 40)], "mx8", hq=2, hkv=2, d=64, seed=31)
    pr.d_lens = torch.tensor([-0x80000000, 40], dtype=torch.int32, device="cuda")
    out = torch.full((2, 2, 25, 64), 9.0, dtype=torch.bfloat16, device="cuda")
    binding.hga_cache_read(pr.p, 10, 35, pr.d_lens, pr.d_table, *pr.cache(), out, None, pr.status)
    assert (out[0] == 9).all() and np.array_equal(T.f64(out[1]), pr.resident(pr.values("K"), 1)[:, 10:35])
    assert int(pr.status.item()) == binding.HGA_STATUS_BAD_INDEX


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("seqs", ([(1, 300)], [(90, 300)]))
def test_large_logits_in_any_order(fmt, seqs):
    """a row's largest logit comes late, early, and far above the rest"""
    pr = T.Problem(seqs, fmt, hq=4, hkv=1, d=64, seed=14, spread=8.0)
    Q = pr.randn(pr.n_tokens, 4, 64) * 6
    O, LSE = pr.run_attn(Q.cuda())
    pr.check_attn(Q, O, LSE)


@pytest.mark.parametrize("fmt", ("mx8", "mx4"))
@pytest.mark.parametrize("seqs,hq", (([(1, 300), (2, 90)], 4), ([(100, 300), (40, 40)], 4)))
@pytest.mark.parametrize("which", ("K tiny", "V tiny", "V huge", "K huge", "V mixed", "all"))
def test_scales_of_every_size(fmt, seqs, hq, which):
    """quantised pages are multiplied as fp16 where their scales allow: here some or all do not"""
    pr = T.Problem(seqs, fmt, hq=hq, hkv=2, d=64, seed=20)
    up = {"K tiny": (-40, 0), "V tiny": (0, -60), "V huge": (0, 60), "K huge": (30, 0), "V mixed": (0, 0), "all": (-70, 40)}[which]
    for name, by in zip("KV", up):
        sc = getattr(pr, name + "_scale")
        sc += by
        if name == "V" and which == "V mixed":
            sc[:, :, 3::5] += 30
            sc[:, :, 4::7] -= 45
    Q = pr.randn(pr.n_tokens, hq, 64)
    Q = (Q.float() * 2.0 ** -up[0]).bfloat16()                               # logits of ordinary size
    Q[1] *= 2.0 ** -20
    O, LSE = pr.run_attn(Q.cuda())
    pr.check_attn(Q, O, LSE)
    assert int(pr.status.item()) == 0


def test_scale_and_strides_of_q_and_o():
    pr = T.Problem([(3, 70), (80, 90)], "mx8", hq=4, hkv=2, d=128, seed=15)
    wide = pr.randn(pr.n_tokens, 3, 4, 128)
    Q = wide[:, 1]
    out = torch.full((4, pr.n_tokens, 136), 7.0, dtype=torch.bfloat16, device="cuda")
    O = out.transpose(0, 1)[..., :128]
    pr.p.q_stride[:], pr.p.o_stride[:] = Q.stride()[:2], O.stride()[:2]
    pr.p.softmax_scale = 0.25
    pr.run_attn(wide.cuda()[:, 1], O=O)
    want, lse, tol, _ = pr.attend(Q, scale=0.25)
    assert (np.abs(T.f64(O) - want) <= tol).all()
    assert (out[..., 128:] == 7).all()


@pytest.mark.parametrize("seqs", ([(1, 600)] * 2, [(100, 400)] * 2))
def test_captured_and_replayed_with_other_contents(seqs):
    """write and attention of a step in one graph; replays see what is in the tensors then"""
    pr = T.Problem([(n, t + 40) for n, t in seqs], "mx8", hq=4, hkv=2, d=128, seed=16)
    K, V, Q = (torch.zeros(pr.n_tokens, h, 128, dtype=torch.bfloat16, device="cuda") for h in (2, 2, 4))
    O, LSE, ws = torch.zeros_like(Q), torch.zeros(Q.shape[:2], device="cuda"), pr.workspace()

    def step():
        binding.hga_cache_write(pr.p, K, V, pr.d_cu, pr.d_lens, pr.d_table, *pr.cache(), pr.status)
        binding.hga_cache_attn(pr.p, Q, pr.d_cu, pr.d_lens, pr.d_table, *pr.cache(), O, LSE, ws, pr.status)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(3):
        pr.seqs = [(n, t + 40 - 11 * k) for n, t in seqs]
        pr.lens = torch.tensor([t for _, t in pr.seqs], dtype=torch.int32)
        pr.d_lens.copy_(pr.lens)
        q = pr.randn(*Q.shape)
        Q.copy_(q)
        K.copy_(pr.randn(*K.shape))
        V.copy_(pr.randn(*V.shape))
        graph.replay()
        torch.cuda.synchronize()
        pr.check_attn(q, O, LSE)
    assert int(pr.status.item()) == 0


def test_two_streams_with_workspaces_of_their_own():
    probs = [T.Problem([(1, 900), (1, 1300)], f, hq=8, hkv=2, d=128, seed=17 + i) for i, f in enumerate(("mx8", "bf16"))]
    Qs = [pr.randn(pr.n_tokens, 8, 128) for pr in probs]
    dev = [q.cuda() for q in Qs]
    streams = [torch.cuda.Stream() for _ in probs]
    ws = [pr.workspace() for pr in probs]
    torch.cuda.synchronize()
    outs = []
    for _ in range(20):
        outs = []
        for pr, q, st, w in zip(probs, dev, streams, ws):
            with torch.cuda.stream(st):
                outs.append(pr.run_attn(q, workspace=w))
    torch.cuda.synchronize()
    for pr, q, (O, LSE) in zip(probs, Qs, outs):
        pr.check_attn(q, O, LSE)


@pytest.mark.parametrize("new,length", ((1, 90), (1, 700), (1, 9000), (70, 200), (70, 3000)))
@pytest.mark.parametrize("sign", (-1, 1))
def test_large_logits_all_alike(new, length, sign):
    """all logits at +-2^25: the mean of the values, whatever the way (one CTA, a cluster, parts, tiles)"""
    pr = T.Problem([(new, length)], "bf16", hq=2, hkv=1, d=64, page=64, seed=25)
    pr.K.fill_(2.0 ** 12)
    Q = torch.full((pr.n_tokens, 2, 64), sign * 2.0 ** 10, dtype=torch.bfloat16, device="cuda")
    O, LSE = pr.run_attn(Q)
    V = pr.resident(pr.values("V"), 0)[0]
    for j in (0, new - 1):
        v = V[:length - new + j + 1]
        # equal weights, each rounded alike; sums of up to 9000 values below 5 in fp32, the tensor pipe cutting off; O's rounding
        off = 2.0 ** -8 * np.abs(v.mean(0)) + len(v) * 2.0 ** -23 * np.abs(v).mean(0)
        assert (np.abs(T.f64(O[j, 0]) - v.mean(0)) <= off).all()
        assert abs(LSE[j, 0].item() / (sign * 2.0 ** 25) - 1) < 1e-5


def test_a_pool_that_is_not_on_the_current_device_is_refused():
    pr = T.Problem([(1, 9)], "bf16", hq=1, hkv=1, d=64, seed=23, device="cpu")
    with pytest.raises(ValueError, match="current device"):
        pr.run_attn(pr.randn(1, 1, 64))
    with pytest.raises(ValueError, match="current device"):
        binding.hga_cache_write(pr.p, None, pr.V_values, pr.d_cu, pr.d_lens, pr.d_table, None, pr.V)
    with pytest.raises(ValueError, match="current device"):
        binding.hga_cache_read(pr.p, 0, 9, pr.d_lens, pr.d_table, pr.K, None, None, None, pr.K_values, None)


def test_writes_are_seen_by_the_calls_behind_them():
    """write, read and attention one straight behind the other, with other contents every time: the kernels start before the one ahead has ended"""
    for fmt in FMTS:
        pr = T.Problem([(1, 300)] * 8, fmt, hq=4, hkv=2, d=128, page=16, seed=24)
        n = 20
        K, V = pr.randn(n, 8, 2, 128).cuda(), pr.randn(n, 8, 2, 128).cuda()
        Q = pr.randn(8, 4, 128)
        Qd, ws = Q.cuda(), pr.workspace()
        O = torch.zeros(n, 8, 4, 128, dtype=torch.bfloat16, device="cuda")
        out = torch.zeros(n, 8, 2, 300, 128, dtype=torch.bfloat16, device="cuda")
        torch.cuda.synchronize()
        for i in range(n):
            binding.hga_cache_write(pr.p, K[i], V[i], pr.d_cu, pr.d_lens, pr.d_table, *pr.cache(), pr.status)
            binding.hga_cache_attn(pr.p, Qd, pr.d_cu, pr.d_lens, pr.d_table, *pr.cache(), O[i], None, ws, pr.status)
            binding.hga_cache_write(pr.p, None, K[n - 1 - i], pr.d_cu, pr.d_lens, pr.d_table, None, pr.V, None, pr.V_scale, pr.status)
            binding.hga_cache_read(pr.p, 0, 300, pr.d_lens, pr.d_table, None, pr.V, None, pr.V_scale, None, out[i], pr.status)
        torch.cuda.synchronize()
        for i in range(n):
            x = T.f64(K[n - 1 - i])
            want = x if fmt == "bf16" else T.held(*T.quantise(x, fmt), fmt)
            assert np.array_equal(T.f64(out[i])[:, :, 299], want)
        again = torch.zeros_like(O)
        for i in range(n):
            binding.hga_cache_write(pr.p, K[i], V[i], pr.d_cu, pr.d_lens, pr.d_table, *pr.cache(), pr.status)
            torch.cuda.synchronize()
            binding.hga_cache_attn(pr.p, Qd, pr.d_cu, pr.d_lens, pr.d_table, *pr.cache(), again[i], None, ws, pr.status)
            torch.cuda.synchronize()
        assert torch.equal(O.view(torch.int16), again.view(torch.int16))
        pr.check_attn(Q, again[n - 1], None)


def test_offsets_beyond_32_bits():
    """a pool whose last page lies more than 2^32 bytes (and elements) behind its first"""
    d, hkv, page = 128, 8, 64
    n_pages = (1 << 32) // (hkv * page * d) + 40                              # bytes of a one-byte format pass 2^32
    for fmt in ("mx8", "bf16"):
        dt = torch.uint8 if fmt == "mx8" else torch.bfloat16
        K = torch.zeros(n_pages, hkv, page, d, dtype=dt, device="cuda")
        V = torch.zeros_like(K)
        sc = [torch.full((n_pages, hkv, page, d // 32), 127, dtype=torch.uint8, device="cuda") if fmt == "mx8" else None for _ in "KV"]
        small = T.Problem([(1, 100), (70, 130)], fmt, hq=8, hkv=hkv, d=d, page=page, seed=18)
        far = torch.arange(n_pages - small.n_pages, n_pages)
        big = torch.where(small.table >= 0, small.table + (n_pages - small.n_pages), small.table).int().cuda()
        p = binding.make_cache_params(2, 8, hkv, d, page, n_pages, big.shape[1], T.FORMATS[fmt], small.n_tokens, 70, 130)
        # the small pool's tokens are read back densely and written to the far pages
        out = [torch.zeros(2, hkv, 130, d, dtype=torch.bfloat16, device="cuda") for _ in "KV"]
        binding.hga_cache_read(small.p, 0, 130, small.d_lens, small.d_table, *small.cache(), *out, small.status)
        new = [torch.cat([o[0, :, :100], o[1]], 1).transpose(0, 1).contiguous() for o in out]
        cu = torch.tensor([0, 100, 230], dtype=torch.int32, device="cuda")
        pw = binding.make_cache_params(2, 8, hkv, d, page, n_pages, big.shape[1], T.FORMATS[fmt], 230, 130, 130)
        binding.hga_cache_write(pw, *new, cu, small.d_lens, big, K, V, *sc, small.status)
        assert int((K[far.cuda()] != 0).sum()) > 0
        Q = small.randn(small.n_tokens, 8, d)
        O, LSE = torch.full_like(Q, 7).cuda(), torch.full(Q.shape[:2], 7.0, device="cuda")
        ws = torch.empty(binding.hga_cache_workspace_bytes(p), dtype=torch.uint8, device="cuda")
        binding.hga_cache_attn(p, Q.cuda(), small.d_cu, small.d_lens, big, K, V, *sc, O, LSE, ws, small.status)
        small.check_attn(Q, O, LSE)
        assert int(small.status.item()) == 0
        del K, V, sc


@pytest.mark.parametrize("fmt", FMTS)
def test_a_document_through_cache_routing_and_attention(fmt):
    """The operators together, and with the calls that are there: a prompt goes into the cache in chunks that attend to what is resident, then
    tokens one by one; the cache is read back and serves summaries, routing and routed attention."""
    hq, hkv, d, total = 8, 2, 128, 384
    pr = T.Problem([(total, total)], fmt, hq=hq, hkv=hkv, d=d, page=16, seed=19)
    K, V, Q = pr.randn(total, hkv, d), pr.randn(total, hkv, d), pr.randn(total, hq, d)
    O, LSE = torch.zeros(total, hq, d, dtype=torch.bfloat16, device="cuda"), torch.zeros(total, hq, device="cuda")
    dK, dV, dQ = K.cuda(), V.cuda(), Q.cuda()
    steps = [(0, 200), (200, 381)] + [(t, t + 1) for t in range(381, total)]
    for a, b in steps:
        p = binding.make_cache_params(1, hq, hkv, d, 16, pr.n_pages, pr.table.shape[1], T.FORMATS[fmt], b - a, b - a, b)
        cu = torch.tensor([0, b - a], dtype=torch.int32, device="cuda")
        lens = torch.tensor([b], dtype=torch.int32, device="cuda")
        binding.hga_cache_write(p, dK[a:b], dV[a:b], cu, lens, pr.d_table, *pr.cache(), pr.status)
        ws = torch.empty(binding.hga_cache_workspace_bytes(p), dtype=torch.uint8, device="cuda")
        binding.hga_cache_attn(p, dQ[a:b], cu, lens, pr.d_table, *pr.cache(), O[a:b], LSE[a:b], ws, pr.status)
    pr.check_attn(Q, O, LSE)
    # read back: [B, Hkv, L, d] as the routed path takes it; with every chunk opened it attends to the same keys
    from paper_2607_15105_b200.workloads import HgaConfig
    cfg = HgaConfig("cache", batch=1, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, total_len=total, seg_len=64, chunk=64, group=8, q_block=64,
                    topk_chunks=4, topk_groups=8, sink=64, local=64, topics=4, needles=0, backward=False, seed=1)
    Kd, Vd = (torch.zeros(1, hkv, total, d, dtype=torch.bfloat16, device="cuda") for _ in "KV")
    lens = torch.tensor([total], dtype=torch.int32, device="cuda")
    binding.hga_cache_read(pr.p, 0, total, lens, pr.d_table, *pr.cache(), Kd, Vd, pr.status)
    buf = binding.HgaLayerBuffers(cfg, backward=False)
    Qs = dQ[total - 64:].transpose(0, 1).contiguous()[None]
    buf.build_summaries(Kd, 0, total)
    buf.route(Qs)
    buf.attn_fwd(Qs, Kd, Vd)
    torch.cuda.synchronize()
    assert int(buf.status.item()) == 0 and int(pr.status.item()) == 0
    dense = O[total - 64:].transpose(0, 1).float()
    # two kernels of the same sums: each within 2^-8 (sum w |v| + 2 |O|) of the value, with |v| < 5 and |O| < 2
    assert (buf.O[0].float() - dense).abs().max().item() <= 2 * 2.0 ** -8 * (5 + 2 * 2)
