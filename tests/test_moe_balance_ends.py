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


@pytest.mark.gpu
@pytest.mark.parametrize("scoring", SCORINGS)
def test_infinite_logits_have_no_part_of_z(scoring):
    """A row that holds +inf gets the loss's gradient and none of z's; the others get both."""
    from paper_2411_02581_b200 import moe
    t, e, k = 500, 40, 2
    z, ids = made(t, e, k, F32, 5)
    z[3, 7], z[3, 30], z[400, 0] = float("inf"), float("inf"), float("inf")
    one = torch.ones(1)
    calm = torch.where(torch.isinf(z), torch.full_like(z, 200.0), z)              # (the same shares, and a finite z)
    want = plain(calm, ids, k, scoring, [0, t], one, 0.3 * one)
    alone = plain(calm, ids, k, scoring, [0, t], one)
    got = moe.balance(z.cuda(), ids.cuda(), scoring=scoring)
    assert float(got.z) == float("inf") and int(got.tokens) == t and torch.equal(got.counts.cpu(), want[2])
    d = moe.balance_backward(z.cuda(), got.counts, got.tokens, k, one.cuda(), 0.3 * one.cuda(), scoring=scoring).cpu()
    rows = torch.ones(t, dtype=torch.bool)
    rows[[3, 400]] = False
    agree_gradient(d[rows], want[5][rows], want[6][rows], F32)
    agree_gradient(d[~rows], alone[5][~rows], alone[6][~rows], F32)



@pytest.mark.gpu
@pytest.mark.parametrize("scoring", SCORINGS)
@pytest.mark.parametrize("t,segments", [(200, 3), (9000, 4)])
def test_without_z(t, segments, scoring):
    """The C entry without a place for z: the rest is the same, bit for bit."""
    from paper_2411_02581_b200 import moe
    e, k = 50, 2
    z, ids = (p.cuda() for p in made(t, e, k, F32, 6))
    offsets = torch.linspace(0, t, segments + 1).long().cuda()
    want = moe.balance(z, ids, scoring=scoring, offsets=offsets)
    loss, counts, mass, live = (torch.empty_like(p) for p in (want.loss, want.counts, want.mass, want.tokens))
    ws = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
    assert B.lib().tuna_moe_balance(z.data_ptr(), 0, t, e, e, ids.data_ptr(), k, SCORINGS.index(scoring), segments, offsets.data_ptr(), loss.data_ptr(),
                                    None, counts.data_ptr(), mass.data_ptr(), live.data_ptr(), ws.data_ptr(), ws.numel(), None) == 0
    torch.cuda.synchronize()
    assert torch.equal(loss, want.loss) and torch.equal(counts, want.counts) and torch.equal(mass, want.mass) and torch.equal(live, want.tokens)



@pytest.mark.gpu
def test_sums_of_a_huge_segment():
    """4 million tokens of even logits: each adds 2^-9 to every expert, so that a lane's sums (of 900 tokens at most) and a block's are exact, and
    the sum of 600 blocks' is off by 600 * 2^-24 of itself at most; the first one's choices are counted to the last."""
    from paper_2411_02581_b200 import moe
    t, e, k = (1 << 22) + 777, 512, 2
    z = torch.zeros(t, e, dtype=torch.bfloat16, device="cuda")
    ids = torch.zeros(t, k, dtype=torch.int32, device="cuda")
    ids[:, 1] = torch.arange(t, device="cuda") % e
    got = moe.balance(z, ids)
    want = torch.bincount(ids[:, 1].long(), minlength=e)
    want[0] += t
    assert torch.equal(got.counts[0], want) and int(got.tokens) == t
    assert bool(((got.mass[0].double() - t / e).abs() <= 2.0 ** -14 * t / e).all())
    assert abs(float(got.loss) - 1) <= 2.0 ** -13
    del z
    torch.cuda.empty_cache()
