"""What the paged cache's calls refuse of tensors, and what they take, on the GPU."""
import pytest
import torch

import cache_testlib as T
from paper_2607_15105_b200 import binding

pytestmark = pytest.mark.gpu


def arguments(pr):
    """the three calls and their arguments by name"""
    n, h, d = pr.n_tokens, pr.hkv, pr.d
    pool = dict(seq_lens=pr.d_lens, block_table=pr.d_table, K_cache=pr.K, V_cache=pr.V, K_scale=pr.K_scale, V_scale=pr.V_scale, status_word=pr.status)
    new, rows = (lambda: torch.zeros(n, h, d, dtype=torch.bfloat16, device="cuda")), torch.zeros(n, pr.hq, d, dtype=torch.bfloat16, device="cuda")
    dense = torch.zeros(len(pr.seqs), h, 40, d, dtype=torch.bfloat16, device="cuda")
    return {binding.hga_cache_write: dict(pool, K_new=new(), V_new=new(), cu_q=pr.d_cu),
            binding.hga_cache_read: dict(pool, tok_begin=0, tok_end=40, K_out=dense, V_out=dense.clone()),
            binding.hga_cache_attn: dict(pool, Q=rows, O=rows.clone(), LSE=torch.zeros(n, pr.hq, device="cuda"), cu_q=pr.d_cu,
                                         workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))}


@pytest.mark.parametrize("fmt", ("bf16", "mx8"))
def test_any_tensor_on_the_host_is_refused(fmt):
    pr = T.Problem([(2, 40), (1, 30)], fmt, hq=4, hkv=2, d=64, seed=61)
    before = binding.hga_kernel_launch_count()
    for call, args in arguments(pr).items():
        for name, t in args.items():
            if isinstance(t, torch.Tensor):
                with pytest.raises(ValueError, match="current device"):
                    call(pr.p, **dict(args, **{name: t.cpu()}))
    assert binding.hga_kernel_launch_count() == before
    for call, args in arguments(pr).items():
        call(pr.p, **args)
        call(pr.p, **dict(args, status_word=None))
        call(pr.p, **{k: t.data_ptr() if isinstance(t, torch.Tensor) and k != "workspace" else t for k, t in args.items()})
    torch.cuda.synchronize()
    assert binding.hga_kernel_launch_count() == before + 9 and int(pr.status.item()) == 0


@pytest.mark.parametrize("fmt", ("bf16", "mx8"))
def test_tensors_that_are_not_dense_are_refused_without_their_strides(fmt):
    pr = T.Problem([(2, 40), (1, 30)], fmt, hq=4, hkv=2, d=64, seed=62)
    for s in (pr.p.k_stride, pr.p.v_stride):
        s[:] = (0, 0, 0)
    before = binding.hga_kernel_launch_count()
    for call, args in arguments(pr).items():
        for name, t in args.items():
            if isinstance(t, torch.Tensor) and t.numel() > 1:
                wide = torch.zeros(*t.shape, 2, dtype=t.dtype, device="cuda")[..., 0]
                with pytest.raises(ValueError, match="strides"):
                    call(pr.p, **dict(args, **{name: wide}))
    assert binding.hga_kernel_launch_count() == before


def test_a_step_without_tokens():
    pr = T.Problem([(0, 40), (0, 30)], "mx8", hq=4, hkv=2, d=64, seed=63)
    before = binding.hga_kernel_launch_count()
    none = torch.empty(0, 2, 64, dtype=torch.bfloat16, device="cuda")
    binding.hga_cache_write(pr.p, none, none, pr.d_cu, pr.d_lens, pr.d_table, *pr.cache(), pr.status)
    rows = torch.empty(0, 4, 64, dtype=torch.bfloat16, device="cuda")
    binding.hga_cache_attn(pr.p, rows, pr.d_cu, pr.d_lens, pr.d_table, *pr.cache(), rows, torch.empty(0, 4, device="cuda"), pr.workspace(), pr.status)
    out = torch.empty(2, 2, 0, 64, dtype=torch.bfloat16, device="cuda")
    binding.hga_cache_read(pr.p, 7, 7, pr.d_lens, pr.d_table, *pr.cache(), out, out, pr.status)
    assert binding.hga_kernel_launch_count() == before
