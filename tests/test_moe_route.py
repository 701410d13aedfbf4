"""Router, order and combine against plain 64-bit implementations, with their gradients.

Tolerances: a weight is a quotient of sums of at most E exponentials, each within 2 units of
2^-24 and summed in 32 bits, so its relative error stays below (E + 8) * 2^-24 < 1e-4 for
E = 512; gradients lose a further cancellation of the same size against |dw| <= max; bf16
results add half a unit of 2^-8.
"""
import numpy as np
import pytest
import torch

from paper_2411_02581_b200 import binding as B
from paper_2411_02581_b200 import build as build_mod
from paper_2411_02581_b200 import workloads as W

EPS32, EPS16 = 1e-4, 2.0 ** -8


def plain_route(logits, k, scoring, renormalize, scale, ranks):
    z = logits.double()
    z = torch.where(torch.isnan(z), torch.full_like(z, -np.inf), z)
    t, e = z.shape
    # a stable descending sort keeps the lower index of a tie first
    order = torch.sort(z, dim=1, descending=True, stable=True)
    ids, zs = order.indices[:, :k].clone(), order.values[:, :k]
    there = zs != -np.inf
    ids[~there] = -1
    top = z.amax(1, keepdim=True) if e else z
    ex = torch.where(z == top, torch.ones_like(z), torch.exp(z - top))
    ex = torch.where(z == -np.inf, torch.zeros_like(z), ex)
    if scoring == "softmax":
        p = ex / ex.sum(1, keepdim=True).clamp(min=1e-300)
    else:
        p = torch.sigmoid(z)
    w = torch.where(there, p.gather(1, ids.clamp(min=0)), torch.zeros_like(zs))
    if renormalize:
        w = w / w.sum(1, keepdim=True).clamp(min=1e-300)
    return ids, w * scale


def plain_order(ids, experts, ranks):
    t, k = ids.shape
    i = ids.numpy().reshape(-1)
    rank = np.repeat(np.arange(t) // max(t // ranks, 1), k)
    ok = (i >= 0) & (i < experts)
    entries = np.flatnonzero(ok)
    at = entries[np.lexsort((entries, i[entries], rank[entries]))]
    rows = np.full(t * k, -1, dtype=np.int64)
    rows[:at.size] = at // k
    pos = np.full(t * k, -1, dtype=np.int64)
    pos[at] = np.arange(at.size)
    counts = np.zeros((ranks, experts), dtype=np.int64)
    np.add.at(counts, (rank[entries], i[entries]), 1)
    offsets = np.concatenate([[0], np.cumsum(counts.reshape(-1))])
    return counts, offsets, rows, pos.reshape(t, k)


def make_logits(t, e, dtype, seed, kind):
    g = torch.Generator().manual_seed(seed)
    z = torch.randn(t, e, generator=g)
    if kind == "ties":
        z = torch.round(z)
    if kind == "masked" and t:
        z[torch.rand(t, e, generator=g) < 0.5] = -np.inf
        z[0] = -np.inf                                        # a row that the mask leaves empty
        z[-1] = np.nan
        z[t // 2] = torch.finfo(dtype).min                    # the lowest value everywhere: an ordinary tie
        if t > 2:
            z[1, e // 2] = np.inf
            z[1, 0] = np.inf
    return z.to(dtype)


SHAPES = [(1, 1, 1, 1), (1, 64, 2, 1), (7, 5, 3, 1), (64, 64, 8, 1), (129, 60, 2, 1), (1000, 256, 8, 4), (96, 100, 9, 8),
          (333, 512, 32, 3), (5000, 8, 1, 1), (40000, 64, 2, 64), (4096, 3, 2, 4096), (9000, 512, 4, 300), (2050, 130, 17, 1)]


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["normal", "ties", "masked"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("t,e,k,ranks", SHAPES)
def test_route_matches_plain(t, e, k, ranks, dtype, kind):
    from paper_2411_02581_b200 import moe
    z = make_logits(t, e, dtype, t * 31 + e, kind)
    for scoring, renormalize, scale in (("softmax", False, 1.0), ("softmax", True, 2.5), ("sigmoid", False, 1.0), ("sigmoid", True, 0.5)):
        r = moe.route(z.cuda(), k, scoring=scoring, renormalize=renormalize, scale=scale, ranks=ranks)
        ids, w = plain_route(z, k, scoring, renormalize, scale, ranks)
        assert torch.equal(r.ids.cpu().long(), ids)
        assert torch.allclose(r.weights.cpu().double(), w, rtol=EPS32, atol=1e-30)
        counts, offsets, rows, pos = plain_order(ids, e, ranks)
        assert np.array_equal(r.counts.cpu().numpy(), counts)
        assert np.array_equal(r.offsets.cpu().numpy(), offsets)
        assert np.array_equal(r.rows.cpu().numpy(), rows)
        assert np.array_equal(r.pos.cpu().numpy(), pos)
        c2, o2, r2, p2 = moe.order(r.ids, e, ranks=ranks)
        assert torch.equal(c2, r.counts) and torch.equal(o2, r.offsets) and torch.equal(r2, r.rows) and torch.equal(p2, r.pos)


@pytest.mark.gpu
def test_route_takes_strided_rows_and_odd_addresses():
    from paper_2411_02581_b200 import moe
    z = make_logits(200, 64, torch.bfloat16, 5, "normal")
    big = torch.zeros(200, 71, dtype=torch.bfloat16, device="cuda")
    big[:, 3:67] = z.cuda()
    a, b = moe.route(z.cuda(), 4), moe.route(big[:, 3:67], 4)
    for x, y in zip(a, b):
        assert torch.equal(x, y)
    dw = torch.randn(200, 4, device="cuda")
    assert torch.equal(moe.route_backward(z.cuda(), a.ids, dw), moe.route_backward(big[:, 3:67], a.ids, dw))


@pytest.mark.gpu
def test_order_leaves_out_ids_outside_the_experts():
    from paper_2411_02581_b200 import moe
    g = torch.Generator().manual_seed(1)
    ids = torch.randint(-3, 20, (500, 4), generator=g, dtype=torch.int32)   # repeated ids in a row are allowed
    got = moe.order(ids.cuda(), 16, ranks=5)
    for x, y in zip(got, plain_order(ids.long(), 16, 5)):
        assert np.array_equal(x.cpu().numpy(), y)
    none = moe.order(torch.full((40, 2), -1, dtype=torch.int32, device="cuda"), 16)
    assert int(none[0].sum()) == 0 and bool((none[2] == -1).all()) and bool((none[3] == -1).all())


@pytest.mark.gpu
def test_route_is_the_dispatch_of_the_c4_generator():
    """rows / counts are the gather map and the count matrix of a top-2 dispatch, experts = ranks."""
    from paper_2411_02581_b200 import moe
    P, tokens, seed = 8, 48, 11
    first, second = W.moe_top2_routing(seed, P, tokens)
    ids = torch.from_numpy(np.stack([first, second], 2).reshape(P * tokens, 2)).to(torch.int32)
    counts, offsets, rows, pos = moe.order(ids.cuda(), P, ranks=P)
    gather, _ = W.moe_row_maps(first, second)
    assert np.array_equal(rows.cpu().numpy(), gather)
    assert np.array_equal(counts.cpu().numpy(), W.moe_top2_counts(seed, P, tokens))


@pytest.mark.gpu
@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalize", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("t,e,k", [(1, 64, 2), (33, 60, 6), (130, 256, 8), (50, 500, 20), (9, 7, 7)])
def test_route_gradient(t, e, k, dtype, renormalize, scoring):
    from paper_2411_02581_b200 import moe
    z = make_logits(t, e, dtype, e, "normal")
    if t > 2:
        z[0] = -np.inf
        z[1, : e // 2] = -np.inf
    dw = torch.randn(t, k, generator=torch.Generator().manual_seed(2))
    r = moe.route(z.cuda(), k, scoring=scoring, renormalize=renormalize, scale=1.5)
    got = moe.route_backward(z.cuda(), r.ids, dw.cuda(), scoring=scoring, renormalize=renormalize, scale=1.5).cpu().double()
    ids, there = r.ids.cpu().long().clamp(min=0), (r.ids.cpu() >= 0).double()

    def value(x):
        p = torch.sigmoid(x) if scoring == "sigmoid" else torch.softmax(x, 1)
        w = torch.nan_to_num(p.gather(1, ids)) * there
        if renormalize:
            w = w / w.sum(1, keepdim=True).clamp(min=1e-300)
        return 1.5 * w

    x = z.double().clone()
    live = torch.isfinite(x).any(1)
    x = x[live].requires_grad_()
    ids, there = ids[live], there[live]
    want = torch.zeros(t, e, dtype=torch.float64)
    (value(x) * dw[live].double()).sum().backward()
    want[live] = torch.nan_to_num(x.grad)
    tol = EPS32 * 8 + (EPS16 if dtype == torch.bfloat16 else 0)
    assert float((got - want).abs().max()) <= tol * max(1.0, float(want.abs().max()))
    # and against differences, along a random direction
    if dtype == torch.float32:
        step = torch.randn(x.shape, dtype=torch.float64, generator=torch.Generator().manual_seed(3))
        step[~torch.isfinite(x.detach())] = 0
        h = 1e-5
        rise = ((value(x.detach() + h * step) - value(x.detach() - h * step)) * dw[live].double()).sum() / (2 * h)
        assert abs(float(rise) - float((got[live] * step).sum())) <= 1e-3 * max(1.0, float((want[live] * step).abs().sum()))


@pytest.mark.gpu
@pytest.mark.parametrize("y_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("t,k,d", [(1, 1, 8), (1, 2, 4096), (77, 3, 100), (40, 6, 257), (300, 2, 1024)])
def test_combine_and_its_gradient(t, k, d, y_dtype, out_dtype):
    from paper_2411_02581_b200 import moe
    g = torch.Generator().manual_seed(t + d)
    rows = t * k + 5
    y = torch.randn(rows, d, generator=g).to(y_dtype)
    pos = torch.randperm(rows, generator=g)[:t * k].view(t, k)
    pos[torch.rand(t, k, generator=g) < 0.2] = -1
    if t > 1:
        pos[0] = -1                                           # a token with no expert left
    w = torch.rand(t, k, generator=g)
    live = (pos >= 0)[:, :, None].double()
    yd = y.double()[pos.clamp(min=0)] * live
    want = (w.double()[:, :, None] * yd).sum(1)
    got = moe.combine(y.cuda(), w.cuda(), pos.cuda(), out_dtype=out_dtype).cpu().double()
    tol = EPS32 + (EPS16 if out_dtype == torch.bfloat16 else 0)
    assert torch.allclose(got, want, rtol=tol, atol=1e-5)
    dout = torch.randn(t, d, generator=g).to(out_dtype)
    dy, dw = moe.combine_backward(dout.cuda(), y.cuda(), w.cuda(), pos.cuda())
    want_dy = torch.zeros(rows, d, dtype=torch.float64)
    ok = pos >= 0
    want_dy[pos[ok]] = (w.double()[:, :, None] * dout.double()[:, None, :])[ok]
    tol = EPS32 + (EPS16 if y_dtype == torch.bfloat16 else 0)
    assert torch.allclose(dy.cpu().double(), want_dy, rtol=tol, atol=1e-6)
    assert torch.allclose(dw.cpu().double(), (yd * dout.double()[:, None, :]).sum(2), rtol=1e-4, atol=1e-5 * d ** 0.5 * 4)


@pytest.mark.gpu
def test_combine_gradient_of_rows_without_columns():
    """<dout, y> of empty rows is zero, and written."""
    from paper_2411_02581_b200 import moe
    L = B.lib()
    w, pos, dw = torch.ones(5, 3, device="cuda"), torch.arange(15, device="cuda"), torch.full((5, 3), 7.0, device="cuda")
    assert L.tuna_moe_combine_backward(None, 0, 0, None, 0, 15, 0, 0, w.data_ptr(), pos.data_ptr(), 5, 3, None, 0, dw.data_ptr(), None) == 0
    torch.cuda.synchronize()
    assert int(torch.count_nonzero(dw)) == 0
    assert L.tuna_moe_combine_backward(None, 0, 0, None, 0, 15, 0, 0, w.data_ptr(), pos.data_ptr(), 5, 3, None, 0, None, None) == -1
    dy, dw = moe.combine_backward(torch.empty(5, 0, device="cuda"), torch.empty(15, 0, device="cuda"), w, pos.view(5, 3))
    assert dy.shape == (15, 0) and int(torch.count_nonzero(dw)) == 0


@pytest.mark.gpu
def test_no_tokens():
    from paper_2411_02581_b200 import moe
    r = moe.route(torch.empty(0, 64, device="cuda"), 2)
    assert r.ids.shape == (0, 2) and int(r.counts.abs().sum()) == 0 and int(r.offsets.abs().sum()) == 0
    assert moe.combine(torch.empty(0, 8, device="cuda"), r.weights, r.pos).shape == (0, 8)
    assert moe.route_backward(torch.empty(0, 64, device="cuda"), r.ids, r.weights).shape == (0, 64)


@pytest.mark.gpu
def test_route_on_another_stream_and_in_a_graph():
    from paper_2411_02581_b200 import moe
    z = make_logits(300, 64, torch.float32, 9, "normal").cuda()
    want = moe.route(z, 2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = moe.route(z, 2, stream=side)
    side.synchronize()
    for x, y in zip(want, got):
        assert torch.equal(x, y)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = moe.route(z, 2)
    z.copy_(make_logits(300, 64, torch.float32, 10, "ties"))
    graph.replay()
    for x, y in zip(moe.route(z, 2), held):
        assert torch.equal(x, y)


def test_route_refusals():
    """Refused on the host, before any GPU work (no GPU needed: pointers are never followed)."""
    build_mod.build()
    L = B.lib()
    n = B.ctypes.c_size_t()
    size = lambda *a: L.tuna_moe_order_workspace_bytes(*a, B.ctypes.byref(n))  # noqa: E731
    assert size(64, 64, 2, 1) == 0 and n.value > 0 and n.value % 256 == 0
    assert size(-1, 64, 2, 1) == -1 and size(64, 0, 2, 1) == -1 and size(64, 64, 0, 1) == -1
    assert size(64, 64, 2, 0) == -1 and size(64, 64, 2, 3) == -1          # 3 ranks do not divide 64 tokens
    assert size(64, 8, 9, 1) == -1                                         # more slots than experts
    assert size(8192, 64, 2, 8192) == -9 and size(64, 513, 2, 1) == -9 and size(64, 64, 33, 1) == -9 and size(1 << 31, 64, 2, 1) == -9

    def route(p=256, dtype=0, t=64, e=64, ld=64, k=2, ranks=1, scoring=0, ws=256, ws_bytes=1 << 30):
        return L.tuna_moe_route(p, dtype, t, e, ld, k, ranks, scoring, 0, 1.0, p, p, p, p, p, p, ws, ws_bytes, None)
    assert route(p=None) == -1 and route(dtype=2) == -1 and route(ld=63) == -1 and route(scoring=7) == -1
    assert route(ws=None, ranks=2) == -6 and route(ws=257, ranks=2) == -6 and route(ws_bytes=8, ranks=2) == -6
    need = lambda *a: (L.tuna_moe_route_workspace_bytes(*a, B.ctypes.byref(n)), n.value)  # noqa: E731
    assert need(64, 64, 2, 1) == (0, 0) and need(64, 64, 2, 2)[1] > 0 and need(5000, 64, 2, 1)[1] > 0   # a few tokens need none
    assert route(p=257) == -1                                              # logits off their own alignment
    assert L.tuna_moe_order(None, 64, 64, 2, 1, None, None, None, None, None, 0, None) == -1
    assert L.tuna_moe_route_backward(None, 0, 64, 64, 64, 2, 0, 0, 1.0, None, None, None, 64, None) == -1
    assert L.tuna_moe_combine(None, 0, 4, 8, 7, None, None, 2, 2, None, 0, 8, None) == -1          # ldy < dim
    assert L.tuna_moe_combine(None, 2, 4, 8, 8, None, None, 2, 2, None, 0, 8, None) == -1          # e4m3 rows
    assert L.tuna_moe_combine(256, 0, 4, 8, 8, 256, 256, 2, 33, 256, 0, 8, None) == -9
    assert L.tuna_ops_device_status(None) == -1


def test_python_refusals():
    from paper_2411_02581_b200 import moe
    with pytest.raises(ValueError, match="logits"):
        moe.route(torch.zeros(4, 4), 2)                                    # not on the GPU
    with pytest.raises(ValueError, match="scoring"):
        moe._scoring("softplus")
