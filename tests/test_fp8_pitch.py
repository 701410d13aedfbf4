"""The 8-bit product into rows of a wider pitch: what lies between them is the caller's."""
import pytest
import torch

from paper_2411_02581_b200 import binding as B
from test_fp8 import activations

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,ldo", [(150, 152), (150, 151), (149, 160), (144, 152), (257, 264)])
@pytest.mark.parametrize("dt", [0, 1])
@pytest.mark.parametrize("m", [200, 20000])
def test_columns_behind_the_result_are_left_alone(m, n, ldo, dt):
    from paper_2411_02581_b200 import moe
    dtype = (torch.float32, torch.bfloat16)[dt]
    q, s = moe.fp8_quantize(activations(m, 144, 1).cuda())
    v, t = moe.fp8_quantize(activations(n, 144, 2).cuda(), "tiles")
    want = moe.fp8_matmul(q, s, v, t, out_dtype=dtype)
    out = torch.full((m, ldo), 7.0, dtype=dtype, device="cuda")
    assert B.lib().tuna_fp8_matmul(q.data_ptr(), s.data_ptr(), m, 144, v.data_ptr(), t.data_ptr(), 2, n, 144, 144, 1, None, out.data_ptr(), dt, ldo, None) == 0
    torch.cuda.synchronize()
    assert torch.equal(out[:, :n], want) and bool((out[:, n:] == 7).all())
