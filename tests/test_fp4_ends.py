"""4-bit operands where they end: scales behind the last row, rows outside every group."""
import pytest
import torch

from paper_2411_02581_b200 import binding as B
from paper_2411_02581_b200 import build as build_mod
from test_fp4_experts import layer, plain_rows
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


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,code", [(torch.float32, 0), (torch.bfloat16, 1)])
@pytest.mark.parametrize("entry", ["fp4", "fp8"])
@pytest.mark.parametrize("offsets", [None, [30, 200, 200, 471], [-5, 1, 1, 1 << 40], [499, 500, 500, 500], [0, 0, 0, 0]])
def test_an_empty_sum_leaves_rows_of_no_group_alone(entry, offsets, dtype, code):
    """k = 0: rows of the groups are zero, others as they were."""
    m, n, pitch, groups = 500, 37, 41, 3
    y = torch.full((m + 2, pitch), 7.0, dtype=dtype, device="cuda")
    off = None if offsets is None else torch.tensor(offsets, device="cuda")
    at, out = None if off is None else off.data_ptr(), y[1:].data_ptr()
    if entry == "fp4":
        rc = B.lib().tuna_fp4_matmul(None, None, m, 16, None, None, n, 16, 0, 0 if off is None else groups, at, out, code, pitch, None)
    else:
        rc = B.lib().tuna_fp8_matmul(None, None, m, 16, None, None, 2, n, 16, 0, 1 if off is None else groups, at, out, code, pitch, None)
    torch.cuda.synchronize()
    lo, hi = (0, m) if offsets is None else (max(offsets[0], 0), min(offsets[-1], m))
    want = torch.full_like(y, 7.0)
    want[1 + lo:1 + hi, :n] = 0
    assert rc == 0 and torch.equal(y, want)


def test_offsets_off_eight_bytes_are_refused():
    """On the host, before any GPU work (pointers are never followed), with an empty sum too."""
    build_mod.build()
    for k in (0, 64):
        assert B.lib().tuna_fp4_matmul(256, 256, 5, 64, 256, 256, 7, 64, k, 2, 260, 256, 0, 8, None) == -1
        assert B.lib().tuna_fp8_matmul(256, 256, 5, 64, 256, 256, 2, 7, 64, k, 2, 260, 256, 0, 8, None) == -1


@pytest.mark.gpu
@pytest.mark.parametrize("t,e,k,d,i", [(1, 8, 2, 1024, 256), (1, 4, 1, 512, 128), (16, 6, 2, 512, 256), (130, 5, 4, 256, 64)])
def test_experts_rows_are_rounded_once_before_the_sum(t, e, k, d, i):
    """The weighted sum adds rows of bf16 in 32 bits.  Against those of 64 bits, rounded, a value differs only where the 32-bit sums cross the middle of two
    bf16 values (a product's sum is off by some 2^-22 of its terms, so one in 2^10 at most, and then by 2^-8: 2^-13 in all) or of two 4-bit ones (one in
    2^16 of h, by a quarter of itself: 2^-10 of all rows, if there is one at all)."""
    from paper_2411_02581_b200 import moe
    parts = layer(e, d, i, 11)
    x = activations(t, d, 12).cuda()
    g = torch.Generator().manual_seed(13)
    ids = torch.rand(t, e, generator=g).argsort(1)[:, :k].to(torch.int32)
    w = torch.rand(t, k, generator=g)
    want = torch.zeros(t, d, dtype=torch.float64)
    for j in range(e):
        at, slot = (ids == j).nonzero(as_tuple=True)
        if at.numel():
            y, _ = plain_rows(x[at].cpu(), *[p[j] for p in parts])
            want.index_add_(0, at, y.to(torch.bfloat16).double() * w[at, slot].double()[:, None])
    want = want.to(torch.bfloat16).double()
    got = moe.fp4_experts(x, ids.cuda(), w.cuda(), *parts).cpu().double()
    assert float((got - want).norm()) <= 2.0 ** -10 * float(want.norm())
