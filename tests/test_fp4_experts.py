"""Experts with 4-bit weights against a plain implementation in 64 bits.

The bound follows the values.  A gate or up sum is within (d / 64 + 8) * 2^-23 of its terms' magnitude (test_fp4.py), so h =
silu(gate) * up moves by at most 1.1 eg |u| + |silu(g)| eu + 1.1 eg eu (silu rises by 1.1 at most), by 2^-19 of itself for the
exponential and the division, and by |g| 2^-23 of itself for the exponential's argument, g log2(e) with a constant that is off by 2^-25 and a
product by 2^-24 of themselves: e^-g is off by |g| 1.5 * 2^-24 of itself, 1 / (1 + e^-g) by no more.  What its 4-bit form may then be lies between those of h a little larger and a little smaller, in
either of the scales that they give; a row of the down product moves linearly with it, by its own sum's share and by its rounding to
bf16 (2^-8), the weighted sum by those of its slots, by k + 1 roundings of 2^-24, and by its own rounding to bf16.
"""
import pytest
import torch

from paper_2411_02581_b200 import binding as B
from paper_2411_02581_b200 import build as build_mod
from test_fp4 import FP4, POWER, plain_quantize, stored, value
from test_fp8 import activations


def weights(count, rows, cols, seed):
    from paper_2411_02581_b200 import moe
    g = torch.Generator().manual_seed(seed)
    parts = [moe.fp4_quantize((torch.randn(rows, cols, generator=g) * cols ** -0.5).cuda()) for _ in range(count)]
    return torch.stack([p[0].contiguous() for p in parts]), torch.stack([p[1] for p in parts])


def layer(e, d, i, seed=1):
    w13, s13 = weights(2 * e, i, d, seed)
    w2, s2 = weights(e, d, i, seed + 1)
    return w13.view(e, 2, i, d // 2), s13.view(e, 2, *s13.shape[1:]), w2, s2


def rounded(h, by):
    """h in 4 bits with the scales of `by`."""
    _, byte = plain_quantize(by)
    s = torch.exp2(byte.double() - 127).repeat_interleave(32, 1)[:, :h.shape[1]]
    v = (h / s).abs()
    step = torch.where(v < 2, 0.5, torch.where(v < 4, 1.0, 2.0))
    return torch.clamp(torch.round(v / step) * step, max=6) * s * h.sign()


def plain_rows(x, w13, s13, w2, s2):
    """One expert's rows and how far off each value may be, in 64 bits."""
    d, i = x.shape[1], w2.shape[1] * 2
    a, gate, up, down = stored(x), value(w13[0], s13[0], d), value(w13[1], s13[1], d), value(w2, s2, i)
    g, u = a @ gate.t(), a @ up.t()
    eg, eu = ((d / 64 + 8) * 2.0 ** -23 * (a.abs() @ m.abs().t()) for m in (gate, up))
    s = torch.nn.functional.silu(g)
    h = s * u
    off = 1.1 * eg * u.abs() + s.abs() * eu + 1.1 * eg * eu + (2.0 ** -19 + 2.0 ** -23 * g.abs()) * h.abs()
    more, less = h + off * h.sign(), torch.where(off < h.abs(), h - off * h.sign(), torch.zeros_like(h))
    held = stored(h)
    slack = torch.stack([(rounded(v, by) - held).abs() for v in (more, less) for by in (more, less)]).amax(0)
    y = held @ down.t()
    return y, slack @ down.abs().t() + (i / 64 + 8) * 2.0 ** -23 * ((held.abs() + slack) @ down.abs().t()) + 2.0 ** -8 * y.abs()


def plain_experts(x, ids, w, *parts):
    e, k = parts[0].shape[0], ids.shape[1]
    ids, w = ids.cpu().long(), w.cpu().double()
    out, off, size = (torch.zeros(x.shape, dtype=torch.float64) for _ in range(3))
    for j in range(e):
        t, slot = (ids == j).nonzero(as_tuple=True)
        if t.numel():
            y, dy = plain_rows(x[t].cpu(), *[p[j] for p in parts])
            by = w[t, slot][:, None]
            out.index_add_(0, t, y * by), off.index_add_(0, t, dy * by.abs()), size.index_add_(0, t, (y * by).abs())
    return out, off + (k + 1) * 2.0 ** -24 * size + 2.0 ** -8 * (out.abs() + off) + 1e-30


def near(got, want, off):
    return got.shape == want.shape and bool(((got.cpu().double() - want).abs() <= off).all())


SIZES = [(1, 4, 2, 128, 128), (1, 64, 2, 1024, 512), (3, 8, 2, 256, 160), (70, 16, 4, 288, 416), (300, 5, 1, 512, 256), (513, 60, 6, 1024, 96),
         (0, 4, 2, 128, 128), (1000, 3, 3, 160, 512), (2, 4, 4, 32, 32), (900, 2, 1, 4096, 64), (260, 4, 2, 64, 2080), (1500, 3, 2, 1056, 800), (4000, 4, 2, 288, 1056), (6000, 3, 1, 160, 2592), (64, 512, 2, 96, 64), (40, 300, 3, 2080, 32), (32, 3, 3, 64, 64), (128, 1, 1, 128, 96), (43, 5, 3, 64, 32)]


@pytest.mark.gpu
@pytest.mark.parametrize("t,e,k,d,i", SIZES)
def test_experts(t, e, k, d, i):
    from paper_2411_02581_b200 import moe
    g = torch.Generator().manual_seed(t + d)
    x = activations(t, d, t + 1).cuda()
    parts = layer(e, d, i)
    ids = torch.rand(t, e, generator=g).argsort(1)[:, :k].to(torch.int32)
    ids[torch.rand(t, k, generator=g) < 0.1] = -1
    ids[ids == e - 1] = 0 if e > 3 else -1                 # an expert that nobody chose (and one that may come twice)
    if t > 2:
        ids[1] = -1                                        # a token without experts
    w = torch.rand(t, k, generator=g)
    ids, w = ids.cuda(), w.cuda()
    got = moe.fp4_experts(x, ids, w, *parts)
    assert near(got, *plain_experts(x, ids, w, *parts))
    if t > 2:
        assert bool((got[1] == 0).all())
    if t:
        counts, offsets, rows, pos = moe.order(ids, e)
        y = moe.fp4_expert_rows(x[rows.clamp(min=0)], offsets, *parts)
        assert torch.equal(moe.combine(y, w, pos), got)
    assert moe.device_status() == 0


@pytest.mark.gpu
def test_rows_of_no_expert_are_left_alone():
    from paper_2411_02581_b200 import moe
    e, d, i = 3, 96, 160
    parts = layer(e, d, i)
    x = activations(500, d, 3).cuda()
    bounds = [30, 200, 200, 471]
    off = torch.tensor(bounds, device="cuda")
    y = torch.full((500, 104), 7.0, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
    assert B.lib().tuna_fp4_expert_rows(x.data_ptr(), d, 500, e, off.data_ptr(), d, i, *[p.data_ptr() for p in parts], y.data_ptr(), 104, ws.data_ptr(),
                                        ws.numel(), None) == 0
    torch.cuda.synchronize()
    assert bool((y[:30] == 7).all()) and bool((y[471:] == 7).all()) and bool((y[:, d:] == 7).all())
    for j in (0, 2):
        at = slice(bounds[j], bounds[j + 1])
        want, off = plain_rows(x[at].cpu(), *[p[j] for p in parts])
        assert near(y[at, :d], want, off)


@pytest.mark.gpu
def test_values_that_are_large_small_or_not_finite():
    from paper_2411_02581_b200 import moe
    e, d, i = 2, 128, 64
    parts = layer(e, d, i)
    x = activations(8, d, 5)
    x[1] = 0
    x[2] *= 1e15
    x[3] *= 1e-15
    x[4, 7], x[5, 9] = float("nan"), float("inf")
    ids, w = torch.zeros(8, 1, dtype=torch.int32).cuda(), torch.ones(8, 1).cuda()
    got = moe.fp4_experts(x.cuda(), ids, w, *parts)
    fine = [0, 1, 2, 3, 6, 7]
    want, off = plain_experts(x[fine], ids[fine], w[fine], *parts)
    assert near(got[fine], want, off) and bool((got[1] == 0).all()) and bool(torch.isnan(got[4:6]).all())


@pytest.mark.gpu
def test_strided_rows_workspace_stream_and_graph():
    from paper_2411_02581_b200 import moe
    e, k, d, i, t = 8, 2, 160, 96, 300
    parts = layer(e, d, i)
    g = torch.Generator().manual_seed(1)
    x = activations(t, d, 2).cuda()
    r = moe.route(torch.randn(t, e, generator=g).cuda(), k)
    want = moe.fp4_experts(x, r.ids, r.weights, *parts)
    wide = torch.zeros(t, d + 5, dtype=torch.bfloat16, device="cuda")
    wide[:, 3:3 + d] = x
    assert torch.equal(moe.fp4_experts(wide[:, 3:3 + d], r.ids, r.weights, *parts), want)
    ws = torch.full((1 << 24,), 0xff, dtype=torch.uint8, device="cuda")      # (what a workspace held before does not matter)
    assert torch.equal(moe.fp4_experts(x, r.ids, r.weights, *parts, workspace=ws), want)
    rows = x[r.rows]
    want_rows = moe.fp4_expert_rows(rows, r.offsets, *parts)
    ws.fill_(0xff)
    assert torch.equal(moe.fp4_expert_rows(rows, r.offsets, *parts, workspace=ws), want_rows)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
    got = moe.fp4_experts(x, r.ids, r.weights, *parts, stream=side), moe.fp4_expert_rows(rows, r.offsets, *parts, stream=side)
    junk = [torch.full((n,), 0x5a, dtype=torch.uint8, device="cuda") for n in (512 << i for i in range(15)) for _ in range(3)]
    torch.cuda.synchronize()
    assert torch.equal(got[0], want) and torch.equal(got[1], want_rows)
    del junk
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = moe.fp4_experts(x, r.ids, r.weights, *parts)
    x.mul_(2)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, moe.fp4_experts(x, r.ids, r.weights, *parts))


@pytest.mark.gpu
def test_layer_of_the_new_operators_together():
    """Router, its loss, experts in 4 bits, and the gradients of the gate: a training step's calls in their order.  The
    experts' rows, their weighted sum and its gradient are compared with those of the product entry on the same rows."""
    from paper_2411_02581_b200 import moe
    e, k, d, i, t = 6, 2, 256, 128, 400
    parts = layer(e, d, i)
    x = activations(t, d, 2).cuda()
    router = (torch.randn(e, d, generator=torch.Generator().manual_seed(3)) * d ** -0.5).cuda()
    z = x.float() @ router.t()
    r = moe.route(z, k, renormalize=True)
    b = moe.balance(z, r.ids)
    assert torch.equal(b.counts, r.counts)
    rows = x[r.rows]
    y = moe.fp4_expert_rows(rows, r.offsets, *parts)
    out = moe.combine(y, r.weights, r.pos)
    assert torch.equal(out, moe.fp4_experts(x, r.ids, r.weights, *parts))
    # the gate product of every expert by the grouped entry: what the experts' own first step is made of
    q, s = moe.fp4_quantize(rows, offsets=r.offsets)
    gate = moe.fp4_matmul(q, s, parts[0][:, 0].contiguous(), parts[1][:, 0].contiguous(), offsets=r.offsets, out_dtype=torch.float32)
    for j in range(e):
        at = slice(int(r.offsets[j]), int(r.offsets[j + 1]))
        a, m = stored(rows[at].cpu()), value(parts[0][j, 0], parts[1][j, 0])
        assert bool(((gate[at].cpu().double() - a @ m.t()).abs() <= 12 * 2.0 ** -23 * (a.abs() @ m.abs().t()) + 1e-37).all())
    dout = torch.randn(t, d, generator=torch.Generator().manual_seed(4)).to(torch.bfloat16).cuda()
    dy, dw = moe.combine_backward(dout, y, r.weights, r.pos)
    dz = moe.route_backward(z, r.ids, dw, renormalize=True) + moe.balance_backward(z, b.counts, b.tokens, k, torch.full_like(b.loss, 0.01), torch.full_like(b.z, 0.001))
    zc = z.cpu().double().requires_grad_(True)
    p = torch.softmax(zc, 1)
    w = p.gather(1, r.ids.cpu().long())
    w = w / w.sum(1, keepdim=True)
    pick = (y.cpu().double()[r.pos.cpu()] * dout.cpu().double()[:, None]).sum(2)
    loss = 0.01 * e * (b.counts.cpu()[0] / (k * t) * p.mean(0)).sum() + 0.001 * torch.logsumexp(zc, 1).square().mean()
    (loss + (w * pick).sum()).backward()
    assert torch.allclose(dz.cpu().double(), zc.grad, rtol=1e-4, atol=1e-5 * float(pick.abs().max()))
    assert moe.device_status() == 0


@pytest.mark.gpu
def test_python_refusals():
    from paper_2411_02581_b200 import moe
    e, d, i = 4, 64, 32
    w13, s13, w2, s2 = layer(e, d, i)
    x, off = activations(6, d, 1).cuda(), torch.tensor([0, 1, 2, 3, 6], device="cuda")
    ids, w = torch.zeros(6, 2, dtype=torch.int32, device="cuda"), torch.ones(6, 2, device="cuda")
    for bad, match in (((w13[:, :1], s13, w2, s2), "w13"), ((w13, s13[:3], w2, s2), "s13"), ((w13, s13, w2[:3], s2), "w2"), ((w13, s13, w2, s2.view(torch.uint8)), "s2")):
        with pytest.raises(ValueError, match=match):
            moe.fp4_expert_rows(x, off, *bad)
        with pytest.raises(ValueError, match=match):
            moe.fp4_experts(x, ids, w, *bad)
    with pytest.raises(ValueError, match="x: a CUDA matrix of bfloat16"):
        moe.fp4_experts(x.float(), ids, w, w13, s13, w2, s2)
    with pytest.raises(ValueError, match="offsets"):
        moe.fp4_expert_rows(x, off[:4], w13, s13, w2, s2)
    with pytest.raises(ValueError, match="weights"):
        moe.fp4_experts(x, ids, w.double(), w13, s13, w2, s2)
    with pytest.raises(B.TunaError, match="TUNA_ERR_WORKSPACE"):
        moe.fp4_experts(x, ids, w, w13, s13, w2, s2, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
    with pytest.raises(B.TunaError, match="TUNA_ERR_INVALID_ARG"):     # 48 is no multiple of 32
        bad = layer(e, d, 48)
        moe.fp4_experts(x, ids, w, *bad)


def test_expert_refusals():
    """Refused on the host, before any GPU work (pointers are never followed)."""
    import ctypes
    build_mod.build()
    L = B.lib()

    def rows(x=256, ldx=64, m=5, e=4, off=256, d=64, i=32, w13=256, s13=256, w2=256, s2=256, y=256, ldy=64, ws=256, n=1 << 30):
        return L.tuna_fp4_expert_rows(x, ldx, m, e, off, d, i, w13, s13, w2, s2, y, ldy, ws, n, None)
    assert rows(ldx=63) == -1 and rows(ldy=63) == -1 and rows(d=48, ldx=48) == -1 and rows(i=16) == -1 and rows(e=0) == -1 and rows(m=-1) == -1
    assert rows(x=None) == -1 and rows(off=None) == -1 and rows(off=260) == -1 and rows(w13=264) == -1 and rows(s13=264) == -1 and rows(w2=None) == -1
    assert rows(s2=8) == -1 and rows(y=257) == -1 and rows(ws=None) == -6 and rows(ws=264) == -6 and rows(n=64) == -6 and rows(m=0) == 0
    assert rows(e=513) == -9 and rows(m=(1 << 24) + 1) == -9 and rows(i=(1 << 20) + 32) == -9

    def many(x=256, ldx=64, t=5, ids=256, w=256, k=2, e=4, d=64, i=32, w13=256, s13=256, w2=256, s2=256, out=256, ldo=64, ws=256, n=1 << 30):
        return L.tuna_fp4_experts(x, ldx, t, ids, w, k, e, d, i, w13, s13, w2, s2, out, ldo, ws, n, None)
    assert many(ldx=63) == -1 and many(k=5) == -1 and many(k=0) == -1 and many(ids=None) == -1 and many(w=None) == -1 and many(w=258) == -1
    assert many(out=None) == -1 and many(t=-1) == -1 and many(t=0) == 0 and many(ws=None) == -6 and many(n=64) == -6 and many(t=1 << 25) == -9
    n = ctypes.c_size_t()
    assert L.tuna_fp4_experts_workspace_bytes(5, 4, 2, 64, 32, None) == -1 and L.tuna_fp4_expert_rows_workspace_bytes(5, 4, 64, 48, ctypes.byref(n)) == -1
    assert L.tuna_fp4_experts_workspace_bytes(0, 4, 2, 64, 32, ctypes.byref(n)) == 0
