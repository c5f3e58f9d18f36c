"""Decode attention (actkv_attend) against the formula in fp64.

Tolerances.  A logit is an fp32-accumulated sum of D exact bf16 products, scaled in fp32: its error
is at most d = (D + 16) 2^-24 A with A = sm_scale max_t sum_i |q_i k_ti|.  A probability then has a
relative error of at most 2 d plus a few units of 2^-24 from exp2 and the sums and 2^-17 from the two
bf16 values that carry it into the second product (2^-16 covers both), so out is off by at most
(2 d + 2^-16) sum_t p_t |v_t|, and by half a bf16 step, 2^-8 |out|, from its rounding.  The LSE is off
by at most d + 2^-20 (1 + |LSE|).
"""
import math

import numpy as np
import pytest
import torch

from paper_2609_31395_amd import actkv

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a HIP device"
    actkv.load_library()


class Batch:
    """Random requests; every slot that holds no entry is NaN."""

    def __init__(self, heads, lens, tokens, seed, *, per_head=None, causal=True, room=0, rising=False,
                 num_pages=None, sm_scale=0.0):
        self.Hq, self.H, self.D = heads
        rng = np.random.default_rng(seed)
        R = len(lens)
        self.n = np.array(tokens, np.int32)
        L = np.array(lens, np.int32)
        self.lens = np.repeat(L[:, None], self.H, 1) if per_head is None else np.array(per_head, np.int32)
        pages = -(-(L + room) // 16)
        total = num_pages or int(pages.sum()) + 5
        self.bt = np.full((R, max(1, int(pages.max(initial=0)))), -1, np.int32)
        ids = rng.permutation(total)[:int(pages.sum())] if num_pages is None else \
            total - 1 - np.arange(int(pages.sum()))
        at = 0
        for r in range(R):
            self.bt[r, :pages[r]] = ids[at:at + pages[r]]
            at += pages[r]
        g = torch.Generator(device=DEV).manual_seed(seed)

        def randn(*shape):
            return torch.randn(*shape, device=DEV, dtype=torch.bfloat16, generator=g)
        self.kv = torch.empty(2, total, 16, self.H, self.D, dtype=torch.bfloat16, device=DEV)
        if num_pages is None:
            self.kv.fill_(math.nan)
        else:
            self.kv[:, torch.from_numpy(np.sort(ids)).to(DEV)] = math.nan
        for r in range(R):
            for h in range(self.H):
                m = int(self.lens[r, h])
                k, v = randn(m, self.D), randn(m, self.D)
                if rising:
                    k *= torch.linspace(0.1, 6, max(m, 1), device=DEV)[:m, None].bfloat16()
                t = np.arange(m)
                page = torch.from_numpy(self.bt[r, t // 16].astype(np.int64)).to(DEV)
                self.kv[0, page, torch.from_numpy(t % 16).to(DEV), h] = k
                self.kv[1, page, torch.from_numpy(t % 16).to(DEV), h] = v
        self.q = randn(int(self.n.sum()), self.Hq, self.D)
        self.p = actkv.Problem(seq_lens=L + room, q_lens=self.n, budgets=np.zeros(R * self.H),
                               num_q_heads=self.Hq, num_kv_heads=self.H, head_dim=self.D,
                               num_pages=total, bt_stride=self.bt.shape[1], causal=causal,
                               sm_scale=sm_scale).to_device(DEV)
        self.bt_d = torch.from_numpy(self.bt).to(DEV)
        self.lens_d = torch.from_numpy(self.lens.reshape(-1).copy()).to(DEV)

    def reference(self, lens=None, bt=None):
        """out, lse, and how far the kernel's may be from them."""
        lens = self.lens if lens is None else lens
        bt = self.bt if bt is None else bt
        N, D, G = int(self.n.sum()), self.D, self.Hq // self.H
        scale = self.p.sm_scale or 1.0 / math.sqrt(D)
        out = torch.zeros(N, self.Hq, D, dtype=torch.float64, device=DEV)
        lse = torch.full((N, self.Hq), -math.inf, dtype=torch.float64, device=DEV)
        tol, tol_lse = torch.zeros_like(out), torch.zeros_like(lse)
        off = 0
        for r, n in enumerate(self.n):
            for h in range(self.H):
                m = int(lens[r, h])
                t = np.arange(m)
                page = bt[r, t // 16].astype(np.int64)
                good = torch.from_numpy((page >= 0) & (page < self.kv.shape[1])).to(DEV)
                page = torch.from_numpy(np.where((page >= 0) & (page < self.kv.shape[1]), page, 0)).to(DEV)
                slot = torch.from_numpy(t % 16).to(DEV)
                k = torch.where(good[:, None], self.kv[0, page, slot, h].double(), 0.0)
                v = torch.where(good[:, None], self.kv[1, page, slot, h].double(), 0.0)
                for j in range(n):
                    see = min(m, m - int(n) + j + 1) if self.p.causal else m
                    if see < 1:
                        continue
                    q = self.q[off + j, h * G:h * G + G].double()
                    x = q @ k[:see].T * scale
                    p = torch.softmax(x, 1)
                    d = (D + 16) * 2.0 ** -24 * scale * (q.abs() @ k[:see].abs().T).amax(1)
                    hs = slice(h * G, h * G + G)
                    out[off + j, hs] = p @ v[:see]
                    lse[off + j, hs] = torch.logsumexp(x, 1)
                    tol[off + j, hs] = ((2 * d + 2.0 ** -16)[:, None] * (p @ v[:see].abs())
                                        + 2.0 ** -8 * out[off + j, hs].abs())
                    tol_lse[off + j, hs] = d + 2.0 ** -20 * (1 + lse[off + j, hs].abs())
            off += int(n)
        return out, lse, tol, tol_lse

    def check(self, got, lens=None, bt=None):
        out, lse, tol, tol_lse = self.reference(lens, bt)
        assert torch.equal(torch.isinf(got[1]), torch.isinf(lse))
        err = (got[0].double() - out).abs() - tol
        worst = math.nan if torch.isnan(got[0]).any() else float(err.max() if err.numel() else 0)
        assert worst <= 0, \
            f"out off by {worst} more than allowed"
        fine = torch.isfinite(lse)
        err = (got[1].double() - lse)[fine].abs() - tol_lse[fine]
        assert float(err.max() if err.numel() else 0) <= 0, "lse"


HEADS = [(8, 2, 64), (32, 4, 128), (4, 4, 128), (28, 4, 128), (6, 3, 64), (40, 2, 64), (64, 1, 128),
         (17, 1, 128)]


@pytest.mark.parametrize("heads", HEADS)
def test_lengths_around_pages_steps_and_units(heads):
    lens = [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 257, 700]
    b = Batch(heads, lens, [1] * len(lens), 3)
    got = actkv.attend(b.p, b.q, b.kv, b.bt_d)
    b.check(got)
    again = actkv.attend(b.p, b.q, b.kv, b.bt_d)
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("heads", HEADS[:6])
def test_several_tokens_and_a_length_per_head(heads, causal):
    Hq, H, D = heads
    most = 64 // (Hq // H)
    tokens = [1, 0, min(most, 3), most, 2 if most > 1 else 1, 0]
    lens = [300, 40, 1000, 190, 33, 0]
    rng = np.random.default_rng(7)
    per = np.stack([rng.integers(0, m + 1, H) for m in lens])
    per[0, 0], per[2, -1], per[3, 0] = 0, 1, min(most, 190) - 1   # no entry; fewer than tokens
    b = Batch(heads, lens, tokens, 11, per_head=per, causal=causal)
    b.check(actkv.attend(b.p, b.q, b.kv, b.bt_d, kv_lens=b.lens_d))


@pytest.mark.parametrize("heads,lens", [((32, 4, 128), [40000]), ((8, 1, 64), [30001]),
                                        ((16, 8, 128), [9000, 5, 12345, 600]),
                                        ((4, 2, 64), [37 + 11 * i for i in range(300)])])
def test_split_over_the_length_and_joined(heads, lens):
    b = Batch(heads, lens, [1] * len(lens), 5)
    b.check(actkv.attend(b.p, b.q, b.kv, b.bt_d))


@pytest.mark.parametrize("append", [False, True])
@pytest.mark.parametrize("per_head", [False, True])
@pytest.mark.parametrize("heads,tokens", [((32, 4, 128), [2, 1, 0, 3, 1]), ((12, 12, 64), [5, 1, 0, 33, 2]),
                                          ((16, 2, 128), [8, 1, 0, 1, 8]), ((24, 3, 128), [5, 2, 0, 1, 1]),
                                          ((64, 8, 64), [6, 1, 0, 1, 8])])
def test_split_pieces_of_every_kind(heads, tokens, per_head, append):
    """Long requests beside short and empty ones, in shares that begin and end inside them."""
    Hq, H, D = heads
    lens = [9001, 300, 77, 17005, 64]
    rng = np.random.default_rng(4)
    per = None
    if per_head:
        per = np.stack([rng.integers(min(t, m) if append else 0, m + 1, H) for m, t in zip(lens, tokens)])
        per[1, 0], per[3, -1] = tokens[1] if append else 0, 17005
    b = Batch(heads, lens, tokens, 47, per_head=per)
    k = v = None
    if append:
        N = int(b.n.sum())
        k = torch.randn(N, H, D, device=DEV, dtype=torch.bfloat16)
        v = torch.randn(N, H, D, device=DEV, dtype=torch.bfloat16)
    got = actkv.attend(b.p, b.q, b.kv, b.bt_d, kv_lens=b.lens_d if per_head else None, k_new=k, v_new=v)
    if append:
        off = 0
        for r, n in enumerate(tokens):
            for h in range(H):
                t = np.arange(int(b.lens[r, h]) - n, int(b.lens[r, h]))
                page = torch.from_numpy(b.bt[r, t // 16].astype(np.int64)).to(DEV)
                slot = torch.from_numpy(t % 16).to(DEV)
                assert torch.equal(b.kv[0, page, slot, h], k[off:off + n, h])
                assert torch.equal(b.kv[1, page, slot, h], v[off:off + n, h])
            off += n
    b.check(got)


@pytest.mark.parametrize("heads", [(32, 4, 128), (40, 2, 64)])
def test_logits_that_keep_rising(heads):
    b = Batch(heads, [23001, 64, 500], [1, 1, 1], 9, rising=True, sm_scale=0.7)
    b.check(actkv.attend(b.p, b.q, b.kv, b.bt_d))


@pytest.mark.parametrize("fused", [False, True])
@pytest.mark.parametrize("heads", [(8, 2, 64), (32, 4, 128), (40, 2, 64)])
def test_newest_tokens_are_written_first(heads, fused):
    Hq, H, D = heads
    lens, tokens = [1, 200, 130, 50, 16, 3], [1, 1, 2, 0, 1, 3]
    rng = np.random.default_rng(2)
    per = np.stack([rng.integers(min(t, m), m + 1, H) for m, t in zip(lens, tokens)])
    b = Batch(heads, lens, tokens, 13, per_head=per)
    N = int(b.n.sum())
    row = torch.randn(N, Hq + 2 * H, D, device=DEV, dtype=torch.bfloat16)
    b.q, k, v = row[:, :Hq], row[:, Hq:Hq + H], row[:, Hq + H:]
    if not fused:
        b.q, k, v = b.q.contiguous(), k.contiguous(), v.contiguous()
    want = b.kv.clone()
    off = 0
    for r, n in enumerate(tokens):
        for j in range(n):
            for h in range(H):
                t = int(per[r, h]) - n + j
                if t >= 0:
                    want[0, int(b.bt[r, t // 16]), t % 16, h] = k[off + j, h]
                    want[1, int(b.bt[r, t // 16]), t % 16, h] = v[off + j, h]
        off += n
    for r, n in enumerate(tokens):   # the entries to come hold anything before
        for h in range(H):
            for t in range(max(0, int(per[r, h]) - n), int(per[r, h])):
                b.kv[:, int(b.bt[r, t // 16]), t % 16, h] = math.nan
    got = actkv.attend(b.p, b.q, b.kv, b.bt_d, kv_lens=b.lens_d, k_new=k, v_new=v)
    assert torch.equal(b.kv.view(torch.int16), want.view(torch.int16))
    b.check(got)


def test_pages_outside_the_pool_read_as_zero_and_are_not_written():
    for lens in ([300, 20, 100], [22300, 20, 100]):
        _check_bad_pages(Batch((8, 2, 64), lens, [1, 1, 2], 17))


def _check_bad_pages(b):
    bt = b.bt.copy()
    bt[0, 3], bt[0, b.bt.shape[1] - 1], bt[1, 1], bt[2, 6], bt[2, 0] = -1, b.kv.shape[1], 1 << 30, -7, -(1 << 31)
    bt_d = torch.from_numpy(bt).to(DEV)
    b.check(actkv.attend(b.p, b.q, b.kv, bt_d), bt=bt)
    before = b.kv.clone()
    k = torch.randn(4, 2, 64, device=DEV, dtype=torch.bfloat16)
    actkv.attend(b.p, b.q, b.kv, bt_d, k_new=k, v_new=k)
    assert torch.equal(b.kv.view(torch.int16), before.view(torch.int16))   # every last page is a bad one


def test_lengths_outside_the_row_are_taken_as_its_ends():
    b = Batch((8, 2, 64), [100, 40], [1, 1], 19)
    lens = torch.tensor([1000, -5, 40, 41], dtype=torch.int32, device=DEV)
    b.check(actkv.attend(b.p, b.q, b.kv, b.bt_d, kv_lens=lens),
            lens=np.array([[100, 0], [40, 40]], np.int32))


def test_page_offsets_past_32_bits():
    b = Batch((16, 8, 128), [1000, 77], [1, 1], 23, num_pages=140_000)   # 4.6 GB a plane
    k = torch.randn(2, 8, 128, device=DEV, dtype=torch.bfloat16)
    got = actkv.attend(b.p, b.q, b.kv, b.bt_d, k_new=k, v_new=k)
    assert torch.equal(b.kv[0, int(b.bt[1, 4]), 12], k[1]) and torch.equal(b.kv[1, int(b.bt[0, 62]), 7], k[0])
    b.check(got)


def test_outputs_beyond_the_batch_stay_and_the_lse_feeds_the_scoring():
    b = Batch((32, 4, 128), [700, 90, 2000], [1, 1, 1], 29)
    out = torch.full((5, 32, 128), 7.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((5, 32), 7.0, device=DEV)
    got = actkv.attend(b.p, b.q, b.kv, b.bt_d, out=out, lse=lse)
    assert got[0] is out and (out[3:] == 7).all() and (lse[3:] == 7).all()
    b.check((out[:3], lse[:3]))
    # the scoring's own LSE of the same rows, and the scores from it: probabilities that sum to one
    # per query row, G rows to a head
    ref = actkv.lse(b.p, b.q, b.kv, b.bt_d)
    assert float((ref - lse[:3]).abs().max()) <= 2e-4
    acc = torch.zeros(actkv.num_scores(b.p), device=DEV)
    actkv.score_accumulate(b.p, b.q, b.kv, b.bt_d, acc, lse=lse[:3].contiguous())
    off = 0
    for m in (700, 90, 2000):
        sums = acc[off * 4:(off + m) * 4].view(4, m).double().sum(1)
        assert float((sums - 8).abs().max()) <= 8 * 2e-3
        off += m


@pytest.mark.parametrize("longest", [500, 16370])
def test_replayed_from_a_graph_with_lengths_that_grow(longest):
    """seq_lens are what the rows hold at most; the lengths are read on the device."""
    b = Batch((32, 4, 128), [longest, 60], [1, 1], 31, room=40)
    k = torch.randn(2, 4, 128, device=DEV, dtype=torch.bfloat16)
    ws = actkv.attend_workspace(b.p)
    out = torch.empty(2, 32, 128, dtype=torch.bfloat16, device=DEV)
    lse = torch.empty(2, 32, device=DEV)
    lens = b.lens_d.clone()

    def body():
        actkv.attend(b.p, b.q, b.kv, b.bt_d, kv_lens=lens, k_new=k, v_new=k, out=out, lse=lse, ws=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        body()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        body()
    for step in range(1, 5):
        k.copy_(torch.randn(2, 4, 128, device=DEV))
        lens += 7 if step == 3 else 1
        if step == 3:   # the entries that were skipped
            for r in range(2):
                for t in range(int(lens[4 * r]) - 7, int(lens[4 * r]) - 1):
                    b.kv[:, int(b.bt[r, t // 16]), t % 16] = 0.5
        out.fill_(9)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        b.check((out, lse), lens=lens.view(2, 4).cpu().numpy())
        eager = actkv.attend(b.p, b.q, b.kv, b.bt_d, kv_lens=lens, k_new=k, v_new=k)
        assert torch.equal(eager[0], out) and torch.equal(eager[1], lse)


def test_on_a_stream_of_its_own():
    b = Batch((8, 2, 64), [900, 33], [1, 1], 37)
    want = actkv.attend(b.p, b.q, b.kv, b.bt_d)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for stream in (side, side.cuda_stream):
        got = actkv.attend(b.p, b.q, b.kv, b.bt_d, stream=stream)
        other = torch.full((1 << 18,), 3.0, device=DEV)   # may not take the workspace's memory
        side.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and (other == 3).all()


def test_nothing_to_attend():
    b = Batch((8, 2, 64), [40, 20], [0, 0], 41)
    out, lse = actkv.attend(b.p, b.q, b.kv, b.bt_d)
    assert out.shape == (0, 8, 64) and lse.shape == (0, 8)
    b = Batch((8, 2, 64), [0, 0], [1, 2], 43, causal=False)
    out, lse = actkv.attend(b.p, b.q, b.kv, b.bt_d)
    assert (out == 0).all() and torch.isneginf(lse).all()
