"""Decode attention takes nothing of a problem but its requests' lengths, heads and pages: what the
compression reads beside them (budgets, pooling window, aggregation) may be anything, or absent."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2609_31395_amd import actkv

FAKE = 0x10000   # never dereferenced: every call below fails before any launch
INVALID, SMALL = -1, -3


def problem(**over):
    kw = dict(seq_lens=[40, 17], q_lens=[1, 2], budgets=[0] * 4, num_q_heads=14, num_kv_heads=2, head_dim=64,
              num_pages=16, bt_stride=3)
    kw.update(over)
    return actkv.Problem(**kw)


def need(c):
    n = ctypes.c_size_t()
    code = actkv.load_library().actkv_attend_workspace(ctypes.byref(c), ctypes.byref(n))
    return code, n.value


def no_budgets(c):
    c.budgets_h = None


def negative_budgets(c):
    c.kept = np.full(4, -1, np.int32)
    c.budgets_h = c.kept.ctypes.data


def window(c):
    c.pool_window = 4


def aggregation(c):
    c.agg = 1    # MAX_MEAN, which the scoring has not for 7 query heads to a KV head


def other_aggregation(c):
    c.agg = 9


@pytest.mark.parametrize("change", [no_budgets, negative_budgets, window, aggregation, other_aggregation])
def test_fields_of_the_compression_alone(change):
    p = problem()
    c = p._make_cstruct(p.seq_lens, p.q_lens, p.budgets)
    want = need(c)
    assert want[0] == 0
    change(c)
    assert need(c) == want
    c.seq_lens_d = c.q_lens_d = FAKE
    got = actkv.load_library().actkv_attend(ctypes.byref(c), FAKE, 14 * 64, FAKE, FAKE, None, None, None, 0, FAKE, None, FAKE,
                                            64, None)
    assert got == SMALL   # past the problem's checks


@pytest.mark.parametrize("over", [dict(seq_lens=[-1, 17]), dict(q_lens=[-1, 1]), dict(bt_stride=2), dict(num_q_heads=13),
                                  dict(sm_scale=-1.0), dict(sm_scale=float("nan")), dict(num_pages=0), dict(q_lens=[41, 1]), dict(flags=1 << 20)])
def test_its_own_fields_are_checked(over):
    assert need(problem(**over).cstruct())[0] == INVALID


@pytest.mark.parametrize("over", [dict(budgets=[]), dict(pool_window=4), dict(agg="max_mean")])
def test_the_binding_needs_no_budgets(over):
    p = problem(**over)
    ws = actkv.attend_workspace(p, "cpu")
    p.seq_lens_d, p.q_lens_d = torch.from_numpy(p.seq_lens.copy()), torch.from_numpy(p.q_lens.copy())
    ok = dict(q=torch.zeros(3, 14, 64, dtype=torch.bfloat16), kv_cache=torch.zeros(2, 16, 16, 2, 64, dtype=torch.bfloat16),
              block_table=torch.zeros(2, 3, dtype=torch.int32), ws=ws)
    with pytest.raises(ValueError, match="on the GPU"):
        actkv.attend(p, **ok)
    for key, bad in [("q_lens_d", p.q_lens_d[:1]), ("seq_lens_d", None)]:
        old = getattr(p, key)
        setattr(p, key, bad)
        with pytest.raises(ValueError, match=key):
            actkv.attend(p, **ok)
        setattr(p, key, old)
    with pytest.raises(ValueError, match="q_lens"):
        actkv.attend_workspace(problem(q_lens=[1]), "cpu")
