"""Token log probabilities, entropy and top alternatives (actkv_token_logprobs) against fp64.

Tolerances.  With d_v = x_v - max, e^d carries a relative error of at most (|d| + 2) 2^-23 (the
argument's rounding and exp2's), the chunk sums one of 80 2^-24 (64 terms of a thread and the tree), so
log S is off by at most E|d| 2^-23 + 84 2^-24 <= 1e-5 for the rows here (E|d| <= 30), U / S by at most
E[d^2] 2^-23 + 84 2^-24 E|d|, and every result is rounded once to fp32 (2^-24 relative).  Tokens and
their order are exact.
"""
import math

import numpy as np
import pytest
import torch

from paper_2609_31395_amd import actkv

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = [torch.float32, torch.bfloat16, torch.float16]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a HIP device"
    actkv.load_library()


def check(logits, tokens, k, got):
    x = logits.double()
    rows, V = x.shape
    m = x.amax(1, keepdim=True)
    none = torch.isneginf(m)[:, 0]
    d = torch.where(torch.isneginf(x), -1e9, x - torch.where(none[:, None], 0.0, m))
    e = torch.where(torch.isneginf(x), 0.0, torch.exp(d))
    S = e.sum(1)
    lse = torch.where(none, 0.0, m[:, 0] + torch.log(S))
    mean, square = (e * -d).sum(1) / S, (e * d * d).sum(1) / S
    H = torch.where(none, 0.0, torch.log(S) + mean)
    mean, square = torch.where(none, 0.0, mean), torch.where(none, 0.0, square)
    assert float(mean.max()) <= 30
    tol = 1e-5 + 84 * 2.0 ** -24 * mean + 2.0 ** -23 * square + 2.0 ** -24 * H
    assert ((got["entropy"].double() - H).abs() <= tol).all()

    def close(a, b):
        same = a.double() == b
        return (same | ((a.double() - b).abs() <= 1e-5 + 2.0 ** -24 * b.abs())).all()
    if tokens is not None:
        inside = (tokens >= 0) & (tokens < V)
        want = x.gather(1, tokens.clamp(0, V - 1)[:, None])[:, 0] - lse
        assert close(got["logprobs"][inside], want[inside])
        assert (got["logprobs"][tokens < 0] == 0).all() and torch.isnan(got["logprobs"][tokens >= V]).all()
    if k:
        order = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :k]
        n = order.shape[1]
        assert torch.equal(got["top_tokens"][:, :n], order)
        assert close(got["top_logprobs"][:, :n], x.gather(1, order) - lse[:, None])
        assert (got["top_tokens"][:, n:] == -1).all() and torch.isneginf(got["top_logprobs"][:, n:]).all()


def rows_of(V, dtype, seed, rows=7):
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.randn(rows, V, device=DEV, generator=g) * 3
    x[1, int(torch.randint(0, V, (1,)))] += 25            # one near-certain token
    x[2].masked_fill_(torch.rand(V, device=DEV, generator=g) < 0.4, -math.inf)
    x[3] = torch.round(x[3])                               # equal values
    x[4] = 1.25                                            # all equal
    x[5] = -math.inf                                       # masked but for two tokens, if it has them
    x[5, V // 2], x[5, V - 1] = -1.0, 2.0
    if rows > 6:
        x[6] = torch.round(x[6] / 4)                       # few values, zeros of both signs
        x[6, ::3] = -0.0
    return x.to(dtype), torch.randint(0, V, (rows,), device=DEV, generator=g)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [1, 2, 7, 63, 64, 65, 1000, 16383, 16384, 16385, 40001, 151936, 262144])
def test_rows_and_alternatives(V, dtype):
    x, t = rows_of(V, dtype, V)
    for k in (0, 1, 5, 20, 64):
        check(x, t, k, actkv.token_logprobs(x, t, top_k=k))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shift", [0, 1, 3, 8])
def test_rows_that_are_part_of_a_wider_array(dtype, shift):
    V = 20003
    x, t = rows_of(V, dtype, shift)
    wide = torch.full((7, V + 13), math.nan, dtype=dtype, device=DEV)
    part = wide[:, shift:shift + V]
    part.copy_(x)
    check(x, t, 9, actkv.token_logprobs(part, t, top_k=9))
    wide = torch.full((7, V + 13 + (-(V + 13)) % 16), math.nan, dtype=dtype, device=DEV)
    wide[:, :V] = x
    check(x, t, 9, actkv.token_logprobs(wide[:, :V], t, top_k=9))


def test_tokens_outside_the_vocabulary_and_masked_rows():
    x, _ = rows_of(5000, torch.float32, 1)
    x[0] = -math.inf
    t = torch.tensor([3, -1, 5000, 1 << 40, -(1 << 60), 2500, 0], device=DEV)
    got = actkv.token_logprobs(x, t, top_k=4)
    check(x, t, 4, got)
    assert torch.isneginf(got["logprobs"][0]) and got["entropy"][0] == 0
    assert got["top_tokens"][0].tolist() == [0, 1, 2, 3] and torch.isneginf(got["top_logprobs"][0]).all()


def test_only_what_is_asked_for_is_written():
    x, t = rows_of(3000, torch.bfloat16, 2)
    r = actkv.token_logprobs(x)
    assert r["logprobs"] is None and r["top_tokens"] is None
    check(x, None, 0, r)
    e = torch.full((9,), 5.0, device=DEV)
    p = torch.full((9,), 5.0, device=DEV)
    r = actkv.token_logprobs(x, t, entropy=e, logprobs=p)
    assert r["entropy"] is e and (e[7:] == 5).all() and (p[7:] == 5).all()
    check(x, t, 0, dict(entropy=e[:7], logprobs=p[:7]))


def test_values_that_are_not_numbers_never_leave_the_vocabulary():
    x = torch.randn(4, 9000, device=DEV)
    x[0, ::2], x[1, 5], x[2] = math.nan, math.inf, math.nan
    x[3, 7] = -math.nan
    r = actkv.token_logprobs(x, torch.zeros(4, dtype=torch.int64, device=DEV), top_k=64)
    assert ((r["top_tokens"] >= -1) & (r["top_tokens"] < 9000)).all()


def test_many_rows():
    x = (torch.randn(3000, 1500, device=DEV) * 2).bfloat16()
    t = torch.randint(0, 1500, (3000,), device=DEV)
    check(x, t, 3, actkv.token_logprobs(x, t, top_k=3))
    r = actkv.token_logprobs(torch.empty(0, 10, device=DEV), torch.empty(0, dtype=torch.int64, device=DEV), top_k=2)
    assert r["logprobs"].shape == (0,) and r["top_tokens"].shape == (0, 2)


def test_the_token_confidence_is_the_mean_of_the_alternatives():
    """T = -(1/k) sum of the k largest log probabilities (Sec. 6.1)."""
    x, t = rows_of(50000, torch.float32, 4)
    x = x[[0, 1, 3, 6]]
    r = actkv.token_logprobs(x, t[:4], top_k=20)
    conf = actkv.token_confidence(x, top_k=20)
    assert ((conf.double() + r["top_logprobs"].double().mean(1)).abs() <= 4e-5).all()


def test_replayed_from_a_graph():
    x, t = rows_of(40000, torch.float32, 8)
    out = dict(logprobs=torch.empty(7, device=DEV), entropy=torch.empty(7, device=DEV),
               top_tokens=torch.empty(7, 5, dtype=torch.int64, device=DEV), top_logprobs=torch.empty(7, 5, device=DEV))
    ws = torch.empty(1 << 16, dtype=torch.uint8, device=DEV)

    def body():
        actkv.token_logprobs(x, t, top_k=5, ws=ws, **out)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        body()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        body()
    for rep in range(3):
        x.copy_(rows_of(40000, torch.float32, 20 + rep)[0])
        for v in out.values():
            v.fill_(-3)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        check(x, t, 5, out)
