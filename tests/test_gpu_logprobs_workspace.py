"""Log probabilities of batches that shrink, in a workspace made for the largest."""
import ctypes

import pytest
import torch

from paper_2609_31395_amd import actkv

pytestmark = pytest.mark.gpu
DEV = "cuda"


def test_a_batch_that_shrinks_in_one_workspace():
    rows, vocab = 64, 151936
    n = ctypes.c_size_t()
    assert actkv.load_library().actkv_token_logprobs_workspace(rows, vocab, 64, ctypes.byref(n)) == 0
    ws = torch.empty(n.value + 64, dtype=torch.uint8, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(1)
    logits = torch.randn(rows, vocab, device=DEV, generator=g) * 3
    tokens = torch.randint(0, vocab, (rows,), device=DEV, generator=g)
    for r, v, k in [(64, vocab, 64), (64, vocab, 20), (52, vocab, 20), (51, vocab, 20), (32, vocab, 26), (51, 100000, 40),
                    (7, 50000, 64), (1, vocab, 20)]:
        x = logits[:r, :v]
        t = tokens[:r] % v
        ws[n.value:] = 77
        got = actkv.token_logprobs(x, t, top_k=k, ws=ws[:n.value])
        want = actkv.token_logprobs(x, t, top_k=k)
        for key in want:
            assert torch.equal(got[key], want[key]), (r, v, k, key)
        assert torch.equal(got["top_tokens"], torch.sort(x, dim=1, descending=True, stable=True).indices[:, :k])
        assert (ws[n.value:] == 77).all()
