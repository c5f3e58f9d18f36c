"""Decode attention of large values: V scaled by a power of two scales the output by exactly that, as
long as the sums before the division stay within fp32."""
import pytest
import torch

from paper_2609_31395_amd import actkv
from test_gpu_attend import Batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lens", [[700, 40, 33], [40000, 300]])
@pytest.mark.parametrize("heads", [(32, 4, 128), (40, 2, 64)])
def test_large_values(heads, lens):
    """|V| below 8 before it is scaled (randn in bf16, checked), so below 2^88 after."""
    b = Batch(heads, lens, [1] * len(lens), 61, rising=True)
    assert float(torch.nan_to_num(b.kv[1].float()).abs().max()) < 8
    want, lse = actkv.attend(b.p, b.q, b.kv, b.bt_d)
    b.kv[1] *= 2.0 ** 85
    got, lse2 = actkv.attend(b.p, b.q, b.kv, b.bt_d)
    assert torch.equal(lse, lse2)
    assert torch.equal(got.double(), want.double() * 2.0 ** 85)
