"""The decode-step operators called for the null stream by its raw handle, 0: what they make belongs to
that stream, whichever stream is current."""
import pytest
import torch

from paper_2609_31395_amd import actkv

pytestmark = pytest.mark.gpu
DEV = "cuda"


def stream_of(t):
    """The stream whose pool t's memory comes from."""
    return next(s["stream"] for s in torch.cuda.memory_snapshot()
                if s["address"] <= t.data_ptr() < s["address"] + s["total_size"])


@pytest.mark.parametrize("side_is_current", [False, True])
def test_the_null_stream_by_its_handle(side_is_current):
    g = torch.Generator(device=DEV).manual_seed(3)
    p = actkv.Problem(seq_lens=[40, 17], q_lens=[1, 1], budgets=[0] * 4, num_q_heads=8, num_kv_heads=2,
                      head_dim=64, num_pages=8, bt_stride=3).to_device(DEV)
    kv = torch.randn(2, 8, 16, 2, 64, device=DEV, dtype=torch.bfloat16, generator=g)
    q = torch.randn(2, 8, 64, device=DEV, dtype=torch.bfloat16, generator=g)
    table = torch.tensor([[3, 1, 7], [0, 5, -1]], dtype=torch.int32, device=DEV)
    refs = torch.ones(8, dtype=torch.int32, device=DEV)
    logits = torch.randn(3, 1000, device=DEV, generator=g)
    tokens = torch.zeros(3, dtype=torch.int64, device=DEV)
    want = [*actkv.attend(p, q, kv, table), *actkv.release_pages(table, refs.clone()),
            *actkv.token_logprobs(logits, tokens, top_k=3).values()]
    torch.cuda.synchronize()
    counts = refs.clone()
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream() if side_is_current else torch.cuda.default_stream()):
        got = [*actkv.attend(p, q, kv, table, stream=0), *actkv.release_pages(table, counts, stream=0),
               *actkv.token_logprobs(logits, tokens, top_k=3, stream=0).values()]
    torch.cuda.synchronize()
    assert [stream_of(t) for t in got] == [0] * len(got)
    for a, b in zip(got, want):
        assert torch.equal(a, b)
