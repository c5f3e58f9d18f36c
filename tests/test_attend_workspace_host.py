"""Sizes of the attention's workspace: one made for an engine's largest problem serves every smaller one."""
import ctypes

import numpy as np
import pytest

from paper_2609_31395_amd import actkv


def size(heads, lens, tokens):
    Hq, H, D = heads
    p = actkv.Problem(seq_lens=lens, q_lens=np.full(len(lens), tokens), budgets=np.zeros(len(lens) * H), num_q_heads=Hq,
                      num_kv_heads=H, head_dim=D, num_pages=1 << 20, bt_stride=1 << 12)
    n = ctypes.c_size_t()
    assert actkv.load_library().actkv_attend_workspace(ctypes.byref(p.cstruct()), ctypes.byref(n)) == 0
    return n.value


HEADS = [(8, 2, 64), (32, 4, 128), (32, 8, 128), (64, 8, 64), (12, 12, 64), (16, 16, 128), (28, 4, 128)]


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("lens", [[60], [2048] * 4, [16000], [9000, 12000] * 8, [35000] * 32])
def test_it_never_falls_as_tokens_grow(heads, lens):
    sizes = [size(heads, lens, n) for n in range(0, min(64 // (heads[0] // heads[1]), min(lens)) + 1)]
    assert sizes == sorted(sizes)


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("tokens", [1, 3, 7])
def test_it_never_falls_as_requests_or_lengths_grow(heads, tokens):
    sizes = [size(heads, [length] * 16, tokens) for length in (8, 33, 100, 700, 3000, 9000, 20000, 60000)]
    assert sizes == sorted(sizes)
    sizes = [size(heads, [5000] * r, tokens) for r in (1, 2, 3, 8, 15, 40, 100, 300)]
    assert sizes == sorted(sizes)
