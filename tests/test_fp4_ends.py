"""4-bit operands where they end: scales behind the last row."""
import pytest
import torch

from test_fp4_experts import layer
from test_fp8 import activations


def spoiled(s13, inter):
    """The scales with NaN (byte 255) for the rows behind each matrix's last one, whose values do not matter."""
    s = s13.clone()
    row = torch.arange(128, device=s.device)
    behind = (row >= (inter - 1) % 128 + 1).view(4, 32).t()                       # at [row % 32][row / 32] of a tile
    last = s.view(torch.uint8)[:, :, -1]                                          # [experts, 2, runs, 32, 4, 4]
    last[:] = torch.where(behind[None, None, None, :, :, None], torch.full_like(last, 255), last)
    return s


# (rows, experts, hidden, inter): a block alone with a tile, clusters of 4 and 2 that share one, pairs of blocks
FORMS = {"alone": (700, 3, 288, 160), "wide inter": (300, 2, 256, 416), "fours": (5, 3, 2048, 160), "twos": (90, 8, 4096, 352), "pairs": (6000, 3, 160, 2592)}


@pytest.mark.gpu
@pytest.mark.parametrize("form", list(FORMS))
def test_scales_behind_the_last_row_may_be_nan(form):
    from paper_2411_02581_b200 import moe
    rows, e, d, i = FORMS[form]
    w13, s13, w2, s2 = layer(e, d, i)
    bad = spoiled(s13, i)
    assert bool((bad.view(torch.uint8) == 255).any())
    x = activations(rows, d, 7).cuda()
    offsets = torch.linspace(0, rows, e + 1).long().cuda()
    want = moe.fp4_expert_rows(x, offsets, w13, s13, w2, s2)
    assert bool(torch.isfinite(want).all()) and torch.equal(moe.fp4_expert_rows(x, offsets, w13, bad, w2, s2), want)
    ids = (torch.arange(rows, dtype=torch.int32, device="cuda") % e)[:, None].contiguous()
    w = torch.rand(rows, 1, generator=torch.Generator().manual_seed(1)).cuda()
    assert torch.equal(moe.fp4_experts(x, ids, w, w13, bad, w2, s2), moe.fp4_experts(x, ids, w, w13, s13, w2, s2))
    assert moe.device_status() == 0
