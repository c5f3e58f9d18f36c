"""Decode attention on a problem that has no budgets, nor a window or an aggregation to compress with."""
import pytest
import torch

from paper_2609_31395_amd import actkv

pytestmark = pytest.mark.gpu
DEV = "cuda"


def test_a_problem_without_what_a_compression_takes():
    g = torch.Generator(device=DEV).manual_seed(11)
    kv = torch.randn(2, 30, 16, 2, 64, device=DEV, dtype=torch.bfloat16, generator=g)
    table = torch.randperm(30, device=DEV, generator=g).int().view(2, 15)
    q = torch.randn(3, 14, 64, device=DEV, dtype=torch.bfloat16, generator=g)
    kw = dict(seq_lens=[240, 33], q_lens=[1, 2], num_q_heads=14, num_kv_heads=2, head_dim=64, num_pages=30, bt_stride=15)
    want = actkv.attend(actkv.Problem(budgets=[0] * 4, **kw).to_device(DEV), q, kv, table)
    p = actkv.Problem(budgets=[], pool_window=4, agg="max_mean", **kw)
    p.seq_lens_d, p.q_lens_d = torch.from_numpy(p.seq_lens).to(DEV), torch.from_numpy(p.q_lens).to(DEV)
    got = actkv.attend(p, q, kv, table, ws=actkv.attend_workspace(p))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
