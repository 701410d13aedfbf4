"""The balance loss and its gradient against a plain implementation in 64 bits.

Tolerances.  Logits are below 2^4 in magnitude: z - top is off by 2^-20 at most, exp and the division by a few 2^-23,
so a probability is within 2^-18 of itself.  Sums: a lane adds at most 70 tokens, a block 8 warps, a segment 300 blocks, each
addition off by 2^-24 of the sum: 2^-15 in all for mass, loss and z.  A gradient is p (G - sum p G) + dz' lse p: its two
terms are each within 2^-17 of their magnitude, and the result is rounded to the logits' type.
"""
import ctypes

import pytest
import torch

from paper_2411_02581_b200 import binding as B
from paper_2411_02581_b200 import build as build_mod

F32, BF16 = torch.float32, torch.bfloat16
HALF = {F32: 2.0 ** -24, BF16: 2.0 ** -8}


def made(t, e, k, dtype, seed=0, spread=1.5):
    g = torch.Generator().manual_seed(seed * 1000 + t + e)
    z = (spread * torch.randn(t, e, generator=g)).clamp(-15, 15).to(dtype)
    ids = torch.rand(t, e, generator=g).argsort(1)[:, :k].to(torch.int32)
    return z, ids


def plain(z, ids, k, scoring, bounds, dloss=None, dz=None):
    """(loss, z, counts, mass, live[, dlogits, its size]) in 64 bits."""
    z = z.double()
    z = torch.where(torch.isnan(z), torch.full_like(z, -float("inf")), z)
    t, e = z.shape
    loss, zs, counts, mass, live = [], [], [], [], []
    d, size = torch.zeros_like(z), torch.zeros_like(z)
    for g, (lo, hi) in enumerate(zip(bounds[:-1], bounds[1:])):
        named = ids[lo:hi].reshape(-1).long()
        c = torch.bincount(named[(named >= 0) & (named < e)], minlength=e)
        rows = z[lo:hi]
        at = (rows > -float("inf")).any(1)
        n = int(at.sum())
        rows = rows[at]
        soft = torch.softmax(rows, 1)
        lse = torch.logsumexp(rows, 1)
        if scoring == "softmax":
            p, rest = soft, None
        else:
            logs = torch.nn.functional.logsigmoid(rows)          # (sigmoids that underflow still have shares)
            p, rest = torch.softmax(logs, 1), torch.sigmoid(-rows)
        counts.append(c), live.append(n), mass.append(p.sum(0))
        per = e / (k * n * n) if n else 0.0
        loss.append(per * float((c * mass[-1]).sum())), zs.append(float((lse * lse).mean()) if n else 0.0)
        if dloss is not None and n:
            pull = float(dloss[g]) * per * c.double()
            one, two = p * (pull - (p * pull).sum(1, keepdim=True)), p * (pull.abs() + (p * pull.abs()).sum(1, keepdim=True))
            if rest is not None:
                one, two = one * rest, two * rest
            part = (float(dz[g]) * 2 / n * lse)[:, None] * soft if dz is not None else torch.zeros_like(soft)
            full, mag = torch.zeros(hi - lo, e, dtype=torch.float64), torch.zeros(hi - lo, e, dtype=torch.float64)
            full[at], mag[at] = one + part, two + part.abs()
            d[lo:hi], size[lo:hi] = full, mag
    out = [torch.tensor(loss, dtype=torch.float64), torch.tensor(zs, dtype=torch.float64), torch.stack(counts), torch.stack(mass), torch.tensor(live)]
    return out + [d, size]


def agree(got, want):
    loss, z, counts, mass, live = [p.cpu() for p in got]
    assert torch.equal(counts, want[2]) and torch.equal(live, want[4])
    for a, b in ((loss, want[0]), (z, want[1]), (mass, want[3])):
        assert bool(((a.double() - b).abs() <= 2.0 ** -15 * b.abs() + 1e-30).all())


def agree_gradient(got, want, size, dtype):
    assert got.dtype == dtype
    got = got.cpu().double()
    assert bool(((got - want).abs() <= 2.0 ** -17 * size + HALF[dtype] * want.abs() + 1e-37).all())


def cut_at(t, segments, seed=1):
    if segments == 1:
        return [0, t]
    g = torch.Generator().manual_seed(seed)
    cuts = sorted(torch.randint(0, t + 1, (segments - 1,), generator=g).tolist())
    if segments > 3:
        cuts[1] = cuts[0]                                  # a segment without tokens
    return [0] + cuts + [t]


SIZES = [(1, 1, 1, 1), (1, 8, 2, 1), (2, 3, 3, 2), (63, 60, 4, 5), (500, 8, 2, 1), (257, 33, 5, 4), (1000, 64, 2, 8), (5003, 160, 6, 37), (20000, 64, 8, 3),
         (700, 128, 4, 700), (333, 256, 8, 2), (90, 300, 10, 3), (40, 512, 32, 4), (65, 511, 1, 1), (30011, 9, 2, 1), (100, 64, 2, 9), (100, 64, 2, 8), (50, 16, 2, 3000), (9000, 24, 2, 4000), (8200, 256, 4, 2)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
@pytest.mark.parametrize("t,e,k,segments", SIZES)
def test_loss_and_gradient(t, e, k, segments, scoring, dtype):
    from paper_2411_02581_b200 import moe
    z, ids = made(t, e, k, dtype)
    bounds = cut_at(t, segments)
    offsets = torch.tensor(bounds, device="cuda") if segments > 1 else None
    g = torch.Generator().manual_seed(5)
    dloss, dz = torch.randn(segments, generator=g), torch.randn(segments, generator=g)
    want = plain(z, ids, k, scoring, bounds, dloss, dz)
    got = moe.balance(z.cuda(), ids.cuda(), scoring=scoring, offsets=offsets)
    agree(got, want)
    d = moe.balance_backward(z.cuda(), got.counts, got.tokens, k, dloss.cuda(), dz.cuda(), scoring=scoring, offsets=offsets)
    agree_gradient(d, *want[5:], dtype)
    want = plain(z, ids, k, scoring, bounds, dloss)
    d = moe.balance_backward(z.cuda(), got.counts, got.tokens, k, dloss.cuda(), scoring=scoring, offsets=offsets)
    agree_gradient(d, *want[5:], dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
@pytest.mark.parametrize("t", [90, 3000])
def test_masked_logits_rows_and_choices(t, scoring):
    from paper_2411_02581_b200 import moe
    e, k = 24, 3
    z, ids = made(t, e, k, F32, 2)
    low = torch.finfo(F32).min
    z[3, 5], z[4, :20], z[5, 1] = -float("inf"), -float("inf"), float("nan")
    z[6] = -float("inf")
    z[7] = float("nan")
    z[40:44] = -float("inf")                                # a whole segment of them
    z[8, 2:] = low                                          # the lowest finite value is a logit like any other
    z[9, :4] = -90.0                                        # (its sigmoid is near the end of the range)
    ids[6:8], ids[40:44], ids[10, 1], ids[11, 0], ids[12] = -1, -1, -1, e + 5, -(1 << 31)
    ids[13] = ids[13, 0]                                    # the same expert thrice
    bounds = [0, 12, 40, 44, 44, t]
    offsets = torch.tensor(bounds, device="cuda")
    dloss, dz = torch.linspace(0.5, 2, 5), torch.linspace(1, -1, 5)
    want = plain(z, ids, k, scoring, bounds, dloss, dz)
    got = moe.balance(z.cuda(), ids.cuda(), scoring=scoring, offsets=offsets)
    agree(got, want)
    assert float(got.loss[2]) == 0 and float(got.z[3]) == 0 and got.tokens.tolist()[2:4] == [0, 0]
    d = moe.balance_backward(z.cuda(), got.counts, got.tokens, k, dloss.cuda(), dz.cuda(), scoring=scoring, offsets=offsets)
    agree_gradient(d, *want[5:], F32)
    assert bool((d[6:8] == 0).all()) and bool((d[40:44] == 0).all()) and float(d[3, 5]) == 0 and float(d[5, 1]) == 0


@pytest.mark.gpu
def test_sigmoids_that_underflow_keep_their_shares():
    from paper_2411_02581_b200 import moe
    z = torch.tensor([[-200.0, -201.0, -400.0, -200.0], [-1e30, -1e30, -1e30, -3e38], [300.0, 200.0, -300.0, 0.0]])
    ids = torch.tensor([[0], [1], [2]], dtype=torch.int32)
    got = moe.balance(z.cuda(), ids.cuda(), scoring="sigmoid")
    logs = torch.nn.functional.logsigmoid(z.double())
    assert torch.allclose(got.mass.cpu().double(), torch.softmax(logs, 1).sum(0)[None], rtol=2.0 ** -16, atol=1e-30)
    d = moe.balance_backward(z.cuda(), got.counts, got.tokens, 1, torch.ones(1, device="cuda"), scoring="sigmoid")
    assert bool(torch.isfinite(d).all())


@pytest.mark.gpu
def test_infinite_logits_share_the_softmax():
    from paper_2411_02581_b200 import moe
    z = torch.zeros(40, 16)
    z[1, 3], z[1, 9] = float("inf"), float("inf")
    ids = torch.zeros(40, 1, dtype=torch.int32)
    got = moe.balance(z.cuda(), ids.cuda())
    want = torch.full((16,), 39 / 16)
    want[3] += 0.5
    want[9] += 0.5
    assert torch.allclose(got.mass.cpu()[0], want) and float(got.z[0]) == float("inf") and int(got.tokens[0]) == 40
    d = moe.balance_backward(z.cuda(), got.counts, got.tokens, 1, torch.ones(1, device="cuda"))
    assert bool(torch.isfinite(d).all())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("e,pitch,at", [(60, 67, 3), (64, 72, 0), (33, 48, 8), (130, 131, 1)])
def test_strided_rows(e, pitch, at, dtype):
    from paper_2411_02581_b200 import moe
    z, ids = made(700, e, 4, dtype, 3)
    wide = torch.full((700, pitch), 9.0, dtype=dtype, device="cuda")
    wide[:, at:at + e] = z.cuda()
    a, b = moe.balance(z.cuda(), ids.cuda()), moe.balance(wide[:, at:at + e], ids.cuda())
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    dl = torch.ones(1, device="cuda")
    assert torch.equal(moe.balance_backward(z.cuda(), a.counts, a.tokens, 4, dl, dl), moe.balance_backward(wide[:, at:at + e], a.counts, a.tokens, 4, dl, dl))
    # through the C entry, into rows of a pitch of their own: what lies between them stays
    out = torch.full((700, pitch), 7.0, dtype=dtype, device="cuda")
    assert B.lib().tuna_moe_balance_backward(z.cuda().contiguous().data_ptr(), {F32: 0, BF16: 1}[dtype], 700, e, e, 4, 0, 1, None, a.counts.data_ptr(),
                                             a.tokens.data_ptr(), dl.data_ptr(), dl.data_ptr(), out[:, at:].data_ptr(), pitch, None) == 0
    torch.cuda.synchronize()
    assert torch.equal(out[:, at:at + e], moe.balance_backward(z.cuda(), a.counts, a.tokens, 4, dl, dl))
    assert bool((out[:, :at] == 7).all()) and bool((out[:, at + e:] == 7).all())


@pytest.mark.gpu
def test_tokens_of_no_segment_and_offsets_that_are_no_offsets():
    from paper_2411_02581_b200 import moe
    z, ids = made(900, 40, 2, F32, 4)
    bounds = [100, 350, 800]
    dl = torch.tensor([1.0, 2.0])
    want = plain(z, ids, 2, "softmax", bounds, dl, dl)
    offsets = torch.tensor(bounds, device="cuda")
    got = moe.balance(z.cuda(), ids.cuda(), offsets=offsets)
    agree(got, want)
    d = moe.balance_backward(z.cuda(), got.counts, got.tokens, 2, dl.cuda(), dl.cuda(), offsets=offsets)
    agree_gradient(d, *want[5:], F32)
    assert bool((d[:100] == 0).all()) and bool((d[800:] == 0).all())
    # cut to the tokens
    got = moe.balance(z.cuda(), ids.cuda(), offsets=torch.tensor([-(1 << 62), 350, 1 << 62], device="cuda"))
    agree(got, plain(z, ids, 2, "softmax", [0, 350, 900]))
    # falling ones: nothing outside the arrays is touched, and the calls end (their results mean nothing)
    space = torch.full((64 + 900 * 40 + 64,), 7.0, device="cuda")
    off = torch.tensor([500, 20, -5, 1 << 40, 10, 0], device="cuda")
    b = moe.balance(z.cuda(), ids.cuda(), offsets=off)
    five = torch.ones(5, device="cuda")
    assert B.lib().tuna_moe_balance_backward(z.cuda().data_ptr(), 0, 900, 40, 40, 2, 0, 5, off.data_ptr(), b.counts.data_ptr(), b.tokens.data_ptr(),
                                             five.data_ptr(), None, space[64:].data_ptr(), 40, None) == 0
    torch.cuda.synchronize()
    assert bool((space[:64] == 7).all()) and bool((space[64 + 900 * 40:] == 7).all())


@pytest.mark.gpu
def test_no_tokens_and_no_live_ones():
    from paper_2411_02581_b200 import moe
    got = moe.balance(torch.zeros(0, 12, device="cuda"), torch.zeros(0, 2, dtype=torch.int32, device="cuda"), offsets=torch.zeros(4, dtype=torch.int64, device="cuda"))
    assert [tuple(p.shape) for p in got] == [(3,), (3,), (3, 12), (3, 12), (3,)] and all(bool((p == 0).all()) for p in got)
    assert moe.balance_backward(torch.zeros(0, 12, device="cuda"), got.counts, got.tokens, 2, got.loss, offsets=torch.zeros(4, dtype=torch.int64, device="cuda")).shape == (0, 12)
    z = torch.full((700, 12), -float("inf"), device="cuda")
    got = moe.balance(z, torch.full((700, 2), -1, dtype=torch.int32, device="cuda"))
    assert all(bool((p == 0).all()) for p in got)
    assert bool((moe.balance_backward(z, got.counts, got.tokens, 2, got.loss + 1, got.loss + 1) == 0).all())


@pytest.mark.gpu
def test_gradient_against_differences():
    from paper_2411_02581_b200 import moe
    z, ids = made(120, 16, 2, F32, 6)
    bounds = [0, 50, 120]
    offsets = torch.tensor(bounds, device="cuda")
    dl, dz = torch.tensor([1.0, 3.0]), torch.tensor([0.5, 0.2])
    step = 1e-3 * torch.randn(120, 16, generator=torch.Generator().manual_seed(1), dtype=torch.float64)
    for scoring in ("softmax", "sigmoid"):
        got = moe.balance(z.cuda(), ids.cuda(), scoring=scoring, offsets=offsets)
        d = moe.balance_backward(z.cuda(), got.counts, got.tokens, 2, dl.cuda(), dz.cuda(), scoring=scoring, offsets=offsets).cpu().double()

        def value(at):
            p = plain(at, ids, 2, scoring, bounds)
            return float((p[0] * dl.double()).sum() + (p[1] * dz.double()).sum())
        rise = (value(z.double() + step) - value(z.double() - step)) / 2
        # the third derivative's part is about 1e-6 of the step's; the gradient is within 2^-17 of its terms
        assert abs(rise - float((d * step).sum())) <= 1e-4 * float((d * step).abs().sum())


@pytest.mark.gpu
def test_ranks_that_add_up_their_sums():
    """The loss of a batch in two parts: counts, mass and live tokens added up, and the gradient of each part with them."""
    from paper_2411_02581_b200 import moe
    z, ids = made(1000, 32, 2, F32, 7)
    whole = moe.balance(z.cuda(), ids.cuda())
    parts = [moe.balance(z[s].cuda(), ids[s].cuda()) for s in (slice(0, 300), slice(300, 1000))]
    counts, mass, live = (sum(getattr(p, f) for p in parts) for f in ("counts", "mass", "tokens"))
    assert torch.equal(counts, whole.counts) and torch.equal(live, whole.tokens)
    loss = 32 / (2 * live.double() ** 2) * (counts.double() * mass.double()).sum(1)
    assert torch.allclose(loss, whole.loss.double(), rtol=2.0 ** -15)
    one = torch.ones(1, device="cuda")
    d = torch.cat([moe.balance_backward(z[s].cuda(), counts, live, 2, one) for s in (slice(0, 300), slice(300, 1000))])
    assert torch.equal(d, moe.balance_backward(z.cuda(), whole.counts, whole.tokens, 2, one))


@pytest.mark.gpu
def test_one_answer_however_often_captured_or_on_another_stream():
    from paper_2411_02581_b200 import moe
    z, ids = (p.cuda() for p in made(30000, 64, 2, BF16, 8))
    offsets = torch.tensor([0, 7, 9000, 30000], device="cuda")
    dl = torch.ones(3, device="cuda")

    def call(**kw):
        b = moe.balance(z, ids, offsets=offsets, **kw)
        return [*b, moe.balance_backward(z, b.counts, b.tokens, 2, dl, dl, offsets=offsets, **kw)]
    want = call()
    for _ in range(5):
        assert all(torch.equal(a, b) for a, b in zip(call(), want))
    graphs, outs = [torch.cuda.CUDAGraph() for _ in range(2)], []
    for graph in graphs:
        with torch.cuda.graph(graph):
            outs.append(call())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        graphs[0].replay()
        with torch.cuda.stream(side):
            graphs[1].replay()
    torch.cuda.synchronize()
    for out in outs:
        assert all(torch.equal(a, b) for a, b in zip(out, want))
    torch.cuda._sleep(20_000_000)
    got = call(stream=side)
    junk = [torch.full((n,), 0x5a, dtype=torch.uint8, device="cuda") for n in (512 << i for i in range(15))]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    del junk


@pytest.mark.gpu
def test_beside_the_router():
    """The router's choice, its loss and both gradients: the order as a training step makes them, against autograd in 64 bits."""
    from paper_2411_02581_b200 import moe
    t, e, k = 600, 24, 3
    z, _ = made(t, e, k, F32, 9)
    r = moe.route(z.cuda(), k, renormalize=True)
    b = moe.balance(z.cuda(), r.ids)
    assert torch.equal(b.counts, r.counts) and int(b.tokens[0]) == t
    dw = torch.randn(t, k, generator=torch.Generator().manual_seed(3))
    coef = torch.tensor([0.7])
    d = moe.route_backward(z.cuda(), r.ids, dw.cuda(), renormalize=True) + moe.balance_backward(z.cuda(), b.counts, b.tokens, k, coef.cuda(), coef.cuda())
    x = z.double().requires_grad_(True)
    p = torch.softmax(x, 1)
    w = p.gather(1, r.ids.cpu().long())
    w = w / w.sum(1, keepdim=True)
    loss = e * (b.counts.cpu()[0] / (k * t) * p.mean(0)).sum() + torch.logsumexp(x, 1).square().mean()
    (0.7 * loss + (w * dw.double()).sum()).backward()
    assert torch.allclose(d.cpu().double(), x.grad, rtol=1e-4, atol=1e-6)     # (the router's part is off by some 2^-20 of 1)


@pytest.mark.gpu
def test_more_values_than_32_bits_count():
    from paper_2411_02581_b200 import moe
    t, e = (1 << 22) + 777, 512                             # 2^31 values and more, the last ones like the first
    head, ids0 = made(777, e, 1, BF16, 10)
    z = torch.full((t, e), 0.0, dtype=BF16, device="cuda")
    z[-777:] = head.cuda()
    ids = torch.zeros(t, 1, dtype=torch.int32, device="cuda")
    ids[-777:] = ids0.cuda()
    offsets = torch.tensor([0, t - 777, t], device="cuda")
    got = moe.balance(z, ids, offsets=offsets)
    want = plain(head, ids0, 1, "softmax", [0, 777], torch.ones(1), None)
    assert torch.equal(got.counts[1].cpu(), want[2][0]) and got.tokens.tolist() == [t - 777, 777]
    assert bool(((got.mass[1].cpu().double() - want[3][0]).abs() <= 2.0 ** -15 * want[3][0]).all())
    assert torch.allclose(got.mass[0].cpu().double(), torch.full((e,), (t - 777) / e, dtype=torch.float64), rtol=2.0 ** -11)  # (14000 additions a lane)
    d = moe.balance_backward(z, got.counts, got.tokens, 1, torch.ones(2, device="cuda"), offsets=offsets)
    agree_gradient(d[-777:], *want[5:], BF16)
    del z, d
    torch.cuda.empty_cache()


@pytest.mark.gpu
def test_python_refusals():
    from paper_2411_02581_b200 import moe
    z, ids = (p.cuda() for p in made(8, 16, 2, F32))
    b = moe.balance(z, ids)
    one = torch.ones(1, device="cuda")
    with pytest.raises(ValueError, match="scoring"):
        moe.balance(z, ids, scoring="tanh")
    with pytest.raises(ValueError, match="logits"):
        moe.balance(z.half(), ids)
    with pytest.raises(ValueError, match="logits: rows must be contiguous"):
        moe.balance(z.t(), ids)
    with pytest.raises(ValueError, match="ids"):
        moe.balance(z, ids.long())
    with pytest.raises(ValueError, match="ids"):
        moe.balance(z, ids[:4])
    with pytest.raises(ValueError, match="offsets"):
        moe.balance(z, ids, offsets=torch.zeros(1, dtype=torch.int64, device="cuda"))
    with pytest.raises(ValueError, match="offsets"):
        moe.balance(z, ids, offsets=torch.zeros(3, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError, match="counts"):
        moe.balance_backward(z, b.mass, b.tokens, 2, one)
    with pytest.raises(ValueError, match="dz"):
        moe.balance_backward(z, b.counts, b.tokens, 2, one, one.double())
    with pytest.raises(B.TunaError, match="TUNA_ERR_RANGE"):
        moe.balance_backward(z, b.counts, b.tokens, 33, one)
    with pytest.raises(B.TunaError, match="TUNA_ERR_INVALID_ARG"):
        moe.balance_backward(z, b.counts, b.tokens, 0, one)


def test_balance_refusals():
    """Refused on the host, before any GPU work (pointers are never followed)."""
    build_mod.build()
    L = B.lib()

    def loss(z=256, dtype=0, t=8, e=16, ld=16, ids=256, k=2, scoring=0, seg=1, off=None, out=256, counts=256, mass=256, live=256, ws=256, n=1 << 20):
        return L.tuna_moe_balance(z, dtype, t, e, ld, ids, k, scoring, seg, off, out, None, counts, mass, live, ws, n, None)
    assert loss(dtype=2) == -1 and loss(ld=15) == -1 and loss(scoring=2) == -1 and loss(seg=2) == -1 and loss(seg=0) == -1 and loss(k=0) == -1
    assert loss(z=None) == -1 and loss(z=258) == -1 and loss(ids=None) == -1 and loss(out=None) == -1 and loss(counts=None) == -1 and loss(mass=None) == -1
    assert loss(live=None) == -1 and loss(t=-1) == -1 and loss(e=0, ld=0) == -1
    assert loss(e=513, ld=513) == -9 and loss(k=33) == -9 and loss(seg=32769, off=256) == -9 and loss(t=1 << 31) == -9
    assert loss(t=1 << 20, ws=None) == -6 and loss(t=1 << 20, n=100) == -6 and loss(t=1 << 20, ws=264) == -6

    def grad(z=256, dtype=0, t=8, e=16, ld=16, k=2, scoring=0, seg=1, off=None, counts=256, live=256, dloss=256, out=256, ldd=16):
        return L.tuna_moe_balance_backward(z, dtype, t, e, ld, k, scoring, seg, off, counts, live, dloss, None, out, ldd, None)
    assert grad(dtype=3) == -1 and grad(ld=15) == -1 and grad(ldd=15) == -1 and grad(scoring=-1) == -1 and grad(seg=3) == -1 and grad(counts=None) == -1
    assert grad(live=None) == -1 and grad(dloss=None) == -1 and grad(out=None) == -1 and grad(out=257) == -1 and grad(t=0) == 0 and grad(k=33) == -9
    n = ctypes.c_size_t()
    assert L.tuna_moe_balance_workspace_bytes(1 << 20, 64, 1, None) == -1 and L.tuna_moe_balance_workspace_bytes(-1, 64, 1, ctypes.byref(n)) == -1
    assert L.tuna_moe_balance_workspace_bytes(0, 64, 1, ctypes.byref(n)) == 0 and n.value == 0
    assert L.tuna_moe_balance_workspace_bytes(1 << 20, 64, 3, ctypes.byref(n)) == 0 and n.value > 0
