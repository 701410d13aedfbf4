"""The balance loss where its inputs end: tokens of no segment, masked rows, and gradients that are not finite."""
import pytest
import torch

from test_moe_balance import F32, agree, agree_gradient, made, plain

SCORINGS = ["softmax", "sigmoid"]


@pytest.mark.gpu
@pytest.mark.parametrize("scoring", SCORINGS)
def test_blocks_of_nobodys_tokens(scoring):
    """Whole blocks before the first segment and behind the last one: they have asked for their tokens' choices and leave nothing."""
    from paper_2411_02581_b200 import moe
    t, e, k = 60000, 64, 4
    z, ids = made(t, e, k, F32, 3)
    bounds = [29000, 29500, 30001]
    offsets = torch.tensor(bounds, device="cuda")
    one = torch.tensor([1.0, 2.0])
    want = plain(z, ids, k, scoring, bounds, one, one)
    z, ids = z.cuda(), ids.cuda()
    for _ in range(3):
        got = moe.balance(z, ids, scoring=scoring, offsets=offsets)
        d = moe.balance_backward(z, got.counts, got.tokens, k, one.cuda(), one.cuda(), scoring=scoring, offsets=offsets)
    agree(got, want)
    agree_gradient(d, *want[5:], F32)
    assert bool((d[:29000] == 0).all()) and bool((d[30001:] == 0).all())
    none = moe.balance(z, ids, scoring=scoring, offsets=torch.tensor([t, t, t], device="cuda"))
    assert all(bool((p == 0).all()) for p in none)
