"""The forms of decode attention that few problems take, against the formula in fp64 (tolerances as in
test_gpu_attend); test_attend_forms_host has that these problems take them."""
import pytest
import torch

import attend_forms
from paper_2609_31395_amd import actkv
from test_gpu_attend import Batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("append", [False, True])
@pytest.mark.parametrize("name", attend_forms.FORMS)
def test_against_the_formula(name, append):
    f = attend_forms.FORMS[name]
    Hq, H, D = f["heads"]
    b = Batch(f["heads"], f["lens"], f["tokens"], 53, causal=f["causal"])
    k = v = None
    if append:
        k = torch.randn(int(b.n.sum()), H, D, device="cuda", dtype=torch.bfloat16)
        v = torch.randn(int(b.n.sum()), H, D, device="cuda", dtype=torch.bfloat16)
    got = actkv.attend(b.p, b.q, b.kv, b.bt_d, k_new=k, v_new=v)
    again = actkv.attend(b.p, b.q, b.kv, b.bt_d, k_new=k, v_new=v)
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])
    if append:   # written where the formula reads them
        off = 0
        for r, n in enumerate(b.n):
            here = range(max(0, int(n) - int(b.lens[r, 0])), int(n))
            for j in here:
                t = int(b.lens[r, 0]) - int(n) + j
                page = int(b.bt[r, t // 16])
                assert torch.equal(b.kv[0, page, t % 16], k[off + j]) and torch.equal(b.kv[1, page, t % 16], v[off + j])
            off += int(n)
    b.check(got)
