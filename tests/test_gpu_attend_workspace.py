"""Attention of batches that shrink, in a workspace made for the largest."""
import pytest
import torch

from paper_2609_31395_amd import actkv

pytestmark = pytest.mark.gpu
DEV = "cuda"


def test_fewer_tokens_requests_and_entries_in_one_workspace():
    Hq, H, D, R, length, most = 64, 8, 64, 16, 9000, 6
    pages = -(-length // 16)
    g = torch.Generator(device=DEV).manual_seed(7)
    kv = torch.randn(2, R * pages, 16, H, D, device=DEV, dtype=torch.bfloat16, generator=g)
    table = torch.randperm(R * pages, device=DEV, generator=g).int().view(R, pages)
    ws = None
    for n, reqs, m in [(most, R, length), (5, R, length), (4, R, length), (1, R, length), (3, 9, 7000), (6, 2, 300), (1, 1, 20)]:
        p = actkv.Problem(seq_lens=[m] * reqs, q_lens=[n] * reqs, budgets=[0] * (reqs * H), num_q_heads=Hq, num_kv_heads=H,
                          head_dim=D, num_pages=R * pages, bt_stride=pages).to_device(DEV)
        if ws is None:
            size = actkv.attend_workspace(p).numel()
            ws = torch.empty(size + 256, dtype=torch.uint8, device=DEV)
        ws[size:] = 77
        q = torch.randn(n * reqs, Hq, D, device=DEV, dtype=torch.bfloat16, generator=g)
        got = actkv.attend(p, q, kv, table[:reqs], ws=ws[:size])
        want = actkv.attend(p, q, kv, table[:reqs])
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), (n, reqs, m)
        assert (ws[size:] == 77).all()
