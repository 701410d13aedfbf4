"""The balance loss where its inputs end: tokens of no segment, masked rows, and gradients that are not finite."""
import pytest
import torch

from paper_2411_02581_b200 import binding as B
from paper_2411_02581_b200 import build as build_mod
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


@pytest.mark.gpu
@pytest.mark.parametrize("scoring", SCORINGS)
@pytest.mark.parametrize("e", [5, 24, 64, 160, 300])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("which", ["loss", "z"])
def test_a_gradient_that_is_not_finite_stays_in_its_segment(which, bad, e, scoring):
    """Masked logits, masked rows and tokens of no segment get zeros, and other segments what they get without it."""
    from paper_2411_02581_b200 import moe
    t, k = 3000, 3
    z, ids = made(t, e, k, F32, 4)
    z[700:760], z[1500], z[2500:] = -float("inf"), float("nan"), -float("inf")
    z[::7, 1], z[3::11, 4], ids[2500:] = -float("inf"), float("nan"), -1
    z, ids = z.cuda(), ids.cuda()
    offsets = torch.tensor([100, 600, 2000, 2600], device="cuda")
    got = moe.balance(z, ids, scoring=scoring, offsets=offsets)
    fine = torch.tensor([1.0, 2.0, 3.0], device="cuda")
    odd = fine.clone()
    odd[1] = bad
    args = dict(scoring=scoring, offsets=offsets)
    for dz in ((None, fine) if which == "loss" else (odd,)):
        d = moe.balance_backward(z, got.counts, got.tokens, k, odd if which == "loss" else fine, dz, **args)
        want = moe.balance_backward(z, got.counts, got.tokens, k, fine, None if dz is None else fine, **args)
        inside = torch.zeros(t, dtype=torch.bool, device="cuda")
        inside[600:2000] = True
        assert torch.equal(d[~inside], want[~inside])
        masked = torch.isnan(z) | (z == -float("inf"))
        assert bool((d[masked] == 0).all())
        assert not bool(torch.isfinite(d[inside][~masked[inside]]).any())


def test_pointers_off_their_values_boundaries_are_refused():
    """On the host, before any GPU work (pointers are never followed)."""
    build_mod.build()
    L = B.lib()

    def loss(off=256, out=256, z=256, counts=256, mass=256, live=256):
        return L.tuna_moe_balance(256, 0, 8, 16, 16, 256, 2, 0, 2, off, out, z, counts, mass, live, 256, 0, None)
    assert [loss(off=260), loss(out=258), loss(z=257), loss(counts=260), loss(mass=258), loss(live=252)] == [-1] * 6

    def grad(off=256, counts=256, live=256, dloss=256, dz=256):
        return L.tuna_moe_balance_backward(256, 0, 8, 16, 16, 2, 0, 2, off, counts, live, dloss, dz, 256, 16, None)
    assert [grad(off=260), grad(counts=260), grad(live=252), grad(dloss=258), grad(dz=257)] == [-1] * 5


@pytest.mark.gpu
def test_slots_a_token_are_not_wrapped():
    """An integer that does not fit 32 bits is refused, below as above."""
    from paper_2411_02581_b200 import moe
    z, ids = (p.cuda() for p in made(8, 16, 2, F32))
    b = moe.balance(z, ids)
    one = torch.ones(1, device="cuda")
    with pytest.raises(B.TunaError, match="TUNA_ERR_INVALID_ARG"):
        moe.balance_backward(z, b.counts, b.tokens, 2 - (1 << 32), one)
    with pytest.raises(B.TunaError, match="TUNA_ERR_RANGE"):
        moe.balance_backward(z, b.counts, b.tokens, 2 + (1 << 32), one)


@pytest.mark.gpu
def test_choices_of_masked_rows_are_counted():
    """ids may come from another choice than route's and name experts for rows without live logits: they are counted as any other, and the loss is
    that of the formula, over 1 when all is even.  With -1 there (as route has it) they are not."""
    from paper_2411_02581_b200 import moe
    t, e, k = 640, 8, 2
    z = torch.zeros(t, e)
    z[::4] = -float("inf")
    ids = torch.stack([torch.arange(t) % e, (torch.arange(t) + 3) % e], 1).to(torch.int32)
    got = moe.balance(z.cuda(), ids.cuda())
    agree(got, plain(z, ids, k, "softmax", [0, t]))
    assert abs(float(got.loss) - 4 / 3) < 1e-6 and int(got.counts.sum()) == t * k and int(got.tokens) == t * 3 // 4
    ids[::4] = -1
    got = moe.balance(z.cuda(), ids.cuda())
    agree(got, plain(z, ids, k, "softmax", [0, t]))
