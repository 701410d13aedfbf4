"""Experts of many tokens and the few-token layer against plain 64-bit implementations.

Tolerances, as a share of the row's norm.  Both round the result to bf16 (2^-9).  `experts`
rounds each expert's row to bf16 as well, and its 8-bit intermediate may fall to the other side
of a rounding boundary where the 32-bit sums differ from the 64-bit ones by 1e-6: such a value
moves by up to 2^-3 of itself, one in ~1e4 of them does, which is 2^-3 * 1e-2 of the norm; with
both 2^-9 together below 2^-7 + 2e-3 = 1e-2.  `few` with bf16 weights rounds h to bf16
(2^-9); with 8-bit weights nothing is rounded but the result: 1e-2 covers both.
"""
import pytest
import torch

from paper_2411_02581_b200 import binding as B
from paper_2411_02581_b200 import build as build_mod
from test_fp8 import activations, plain_quantize, value

FP8 = torch.float8_e4m3fn
TOL = 1e-2


def fp8_weights(count, rows, cols, seed):
    from paper_2411_02581_b200 import moe
    g = torch.Generator().manual_seed(seed)
    w = (torch.randn(count, rows, cols, generator=g) * cols ** -0.5)
    parts = [moe.fp8_quantize(m.cuda(), "tiles") for m in w]
    return torch.stack([p[0].contiguous().view(torch.uint8) for p in parts]).view(FP8), torch.stack([p[1] for p in parts])


def bf16_weights(count, rows, cols, seed):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(count, rows, cols, generator=g) * cols ** -0.5).to(torch.bfloat16).cuda()


def held(q, s, i):
    return q[i].cpu().double() if s is None else value(q[i], s[i], "tiles")


def stored(x):
    """x as 8-bit rows hold it, in 64 bits."""
    q, s = plain_quantize(x.float(), "rows")
    return value(q, s, "rows")


def plain_layer(x, ids, w, w13, s13, w2, s2, store):
    """Sum over the chosen experts, in 64 bits; `store` rounds x and h to 8 bits."""
    e, i, d = w13.shape[0], w13.shape[2], w13.shape[3]
    gate = (w13.view(2 * e, i, d), None if s13 is None else s13.view(2 * e, *s13.shape[2:]))
    x, ids, w = x.cpu().double(), ids.cpu().long(), w.cpu().double()
    if store:
        x = stored(x)
    out = torch.zeros_like(x)
    for j in range(e):
        t, slot = (ids == j).nonzero(as_tuple=True)
        if t.numel():
            h = torch.nn.functional.silu(x[t] @ held(*gate, 2 * j).t()) * (x[t] @ held(*gate, 2 * j + 1).t())
            out.index_add_(0, t, (stored(h) if store else h) @ held(w2, s2, j).t() * w[t, slot][:, None])
    return out


def near(got, want):
    got, want = got.cpu().double(), want
    if not want.numel():
        return got.shape == want.shape
    norm = want.norm(dim=1)
    return bool(((got - want).norm(dim=1) <= TOL * norm + 1e-6 * float(norm.max() + 1)).all())


@pytest.mark.gpu
@pytest.mark.parametrize("t,e,k,d,i", [(1, 4, 2, 128, 128), (3, 8, 2, 256, 144), (70, 16, 4, 272, 400), (300, 5, 1, 512, 256), (513, 60, 6, 1024, 80),
                                       (0, 4, 2, 128, 128), (1000, 3, 3, 144, 512)])
def test_experts(t, e, k, d, i):
    from paper_2411_02581_b200 import moe
    g = torch.Generator().manual_seed(t + d)
    x = activations(t, d, t + 1).cuda()
    w13, s13 = fp8_weights(2 * e, i, d, 1)
    w2, s2 = fp8_weights(e, d, i, 2)
    w13, s13 = w13.view(e, 2, i, d), s13.view(e, 2, *s13.shape[1:])
    ids = torch.rand(t, e, generator=g).argsort(1)[:, :k].to(torch.int32)
    ids[torch.rand(t, k, generator=g) < 0.1] = -1
    ids[ids == e - 1] = 0 if e > 3 else -1                 # an expert that nobody chose (and one that may come twice)
    if t > 2:
        ids[1] = -1                                        # a token without experts
    w = torch.rand(t, k, generator=g)
    ids, w = ids.cuda(), w.cuda()
    got = moe.experts(x, ids, w, w13, s13, w2, s2)
    assert near(got, plain_layer(x, ids, w, w13, s13, w2, s2, True))
    if t:
        counts, offsets, rows, pos = moe.order(ids, e)
        y = moe.expert_rows(x[rows.clamp(min=0)], offsets, w13, s13, w2, s2)
        assert torch.equal(moe.combine(y, w, pos), got)
    assert moe.device_status() == 0


FEW = [(1, 4, 1, 128, 128), (1, 64, 2, 1024, 512), (2, 5, 5, 16, 16), (7, 16, 3, 272, 144), (16, 8, 2, 512, 4096), (33, 16, 6, 2048, 784),
       (64, 8, 8, 256, 256), (64, 300, 10, 528, 64), (5, 512, 32, 64, 48), (9, 6, 2, 4112, 96), (40, 4, 2, 96, 5136), (3, 3, 2, 8192, 8192)]


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bf16", "fp8"])
@pytest.mark.parametrize("t,e,k,d,i", FEW)
def test_few(t, e, k, d, i, kind):
    from paper_2411_02581_b200 import moe
    x, router = activations(t, d, t).cuda(), bf16_weights(1, e, d, 3)[0]
    if kind == "fp8":
        w13, s13 = fp8_weights(2 * e, i, d, 1)
        w2, s2 = fp8_weights(e, d, i, 2)
        w13, s13 = w13.view(e, 2, i, d), s13.view(e, 2, *s13.shape[1:])
    else:
        w13, w2, s13, s2 = bf16_weights(2 * e, i, d, 1).view(e, 2, i, d), bf16_weights(e, d, i, 2), None, None
    for scoring, renormalize in (("softmax", True), ("sigmoid", False)):
        ids, w = torch.empty(t, k, dtype=torch.int32, device="cuda"), torch.empty(t, k, device="cuda")
        got = moe.few(x, router, k, w13, w2, s13=s13, s2=s2, scoring=scoring, renormalize=renormalize, scale=1.5, ids=ids, weights=w)
        z = x.cpu().double() @ router.cpu().double().t()
        p = torch.softmax(z, 1) if scoring == "softmax" else torch.sigmoid(z)
        top, order = torch.sort(z, dim=1, descending=True)
        # the choice, wherever 32-bit logits can tell the last chosen from the first not chosen
        clear = torch.ones(t, dtype=torch.bool) if k == e else top[:, k - 1] - top[:, k] > 1e-4 * top.abs().amax(1)
        assert torch.equal(ids.cpu().long().sort(1).values[clear], order[clear, :k].sort(1).values)
        want_w = p.gather(1, ids.cpu().long())
        want_w = 1.5 * (want_w / want_w.sum(1, keepdim=True) if renormalize else want_w)
        assert torch.allclose(w.cpu().double(), want_w, rtol=2e-3, atol=1e-6)   # |dz| <= 2^-22 * sum |x r| ~ 1e-4
        assert near(got, plain_layer(x, ids, w, w13, s13, w2, s2, False))
    assert moe.device_status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bf16", "fp8"])
def test_few_values_that_are_large_small_or_not_finite(kind):
    from paper_2411_02581_b200 import moe
    e, k, d, i = 4, 4, 128, 64
    w13, w2, s13, s2 = bf16_weights(2 * e, i, d, 1).view(e, 2, i, d), bf16_weights(e, d, i, 2), None, None
    if kind == "fp8":
        w13, s13 = fp8_weights(2 * e, i, d, 1)
        w2, s2 = fp8_weights(e, d, i, 2)
        w13, s13 = w13.view(e, 2, i, d), s13.view(e, 2, *s13.shape[1:])
    x = activations(8, d, 5)
    x[1] = 0
    x[2] *= 1e15
    x[3] *= 1e-15
    x[4, 7] = float("nan")
    x[5, 9] = float("inf")
    router = torch.zeros(e, d, dtype=torch.bfloat16, device="cuda")   # every expert at the same logit
    ids, w = torch.empty(8, k, dtype=torch.int32, device="cuda"), torch.empty(8, k, device="cuda")
    got = moe.few(x.cuda(), router, k, w13, w2, s13=s13, s2=s2, renormalize=True, ids=ids, weights=w)
    fine = [0, 1, 2, 3, 6, 7]
    assert torch.equal(ids[fine].cpu(), torch.arange(4, dtype=torch.int32).repeat(6, 1))    # ties go to the lowest
    want = plain_layer(x, ids, w, w13, s13, w2, s2, False)
    for r in fine:                                         # row by row: they differ by thirty orders of magnitude
        assert near(got[r:r + 1], want[r:r + 1]), r
    # a token whose logits are NaN has no expert: its sum is empty
    assert bool((ids[4:6] == -1).all()) and bool((got[4:6] == 0).all())


@pytest.mark.gpu
@pytest.mark.parametrize("power", [118, 121, 122, 126, 127])
def test_few_values_up_to_the_largest_finite_one(power):
    """8-bit weights so small that products with x near the end of its range are ordinary numbers: x is held in two pieces
    whose scale has to follow it to the end."""
    from paper_2411_02581_b200 import moe
    e, k, d, i = 2, 2, 256, 64
    w13, s13 = fp8_weights(2 * e, i, d, 1)
    w2, s2 = fp8_weights(e, d, i, 2)
    s13 = (s13 * 2.0 ** -power).view(e, 2, *s13.shape[1:])
    x = activations(4, d, 5, torch.float32)
    x = (x / x.abs().amax() * 1.99 * 2.0 ** power).to(torch.bfloat16)      # (1.99 rounds to 1.992 in 8 bits: finite at 2^127)
    x[3] *= 2.0 ** -20
    router = torch.zeros(e, d, dtype=torch.bfloat16, device="cuda")
    ids, w = torch.empty(4, k, dtype=torch.int32, device="cuda"), torch.empty(4, k, device="cuda")
    got = moe.few(x.cuda(), router, k, w13.view(e, 2, i, d), w2, s13=s13, s2=s2, renormalize=True, ids=ids, weights=w)
    want = plain_layer(x, ids, w, w13.view(e, 2, i, d), s13, w2, s2, False)
    for r in range(4):
        assert bool(torch.isfinite(got[r]).all()) and near(got[r:r + 1], want[r:r + 1]), r


@pytest.mark.gpu
@pytest.mark.parametrize("small", [2.0 ** -10, 2.0 ** -13, 2.0 ** -16, 2.0 ** -20])
def test_few_small_values_beside_a_large_one(small):
    """8-bit weights: a value of x or h is held to 2^-9 of itself or to 2^-21 of the largest one of its 128, whichever
    is more (x, of bf16, exactly where the first is more).  The large channels have no weight of their own, so the
    result is made of the small ones.

    The bound of an output follows: gate and up sums move by G = sum_k 2^-21 max |x of the block| |w| (and 2^-20 of
    sum |x w| for the 32-bit sums), h by 1.1 G |u| + |silu(g)| U + 1.1 G U (silu rises by 1.1 at most) and by its own
    rounding, y and the weighted sum linearly with them; the result is rounded to bf16 (2^-9)."""
    from paper_2411_02581_b200 import moe
    e, k, d, i, t = 2, 2, 256, 144, 5
    g = torch.Generator().manual_seed(4)
    x = torch.randn(t, d, generator=g) * small
    loud = [3, 200]                                               # one in each block of 128
    x[:, loud] = torch.tensor([1.9, -1.5])
    x = x.to(torch.bfloat16)
    w13, s13 = fp8_weights(2 * e, i, d, 1)
    w13.view(torch.uint8)[:, :, loud] = 0
    w2, s2 = fp8_weights(e, d, i, 2)
    s13 = s13 / small                                             # so that g and u are about one
    w13, s13 = w13.view(e, 2, i, d), s13.view(e, 2, *s13.shape[1:])
    router = torch.zeros(e, d, dtype=torch.bfloat16, device="cuda")
    ids, w = torch.empty(t, k, dtype=torch.int32, device="cuda"), torch.empty(t, k, device="cuda")
    got = moe.few(x.cuda(), router, k, w13, w2, s13=s13, s2=s2, renormalize=True, ids=ids, weights=w).cpu().double()
    X = x.double()
    top = lambda v: torch.nn.functional.pad(v.abs(), (0, -v.shape[1] % 128)).unflatten(1, (-1, 128)).amax(2).repeat_interleave(128, 1)[:, :v.shape[1]]  # noqa: E731
    out, bound = torch.zeros(t, d, dtype=torch.float64), torch.zeros(t, d, dtype=torch.float64)
    for j in range(e):
        wg, wu, wd = value(w13[j, 0], s13[j, 0], "tiles"), value(w13[j, 1], s13[j, 1], "tiles"), value(w2[j], s2[j], "tiles")
        a, b = X @ wg.t(), X @ wu.t()
        A, Bd = [(2.0 ** -21 * top(X) + 2.0 ** -20 * X.abs()) @ m.abs().t() for m in (wg, wu)]
        silu = torch.nn.functional.silu(a)
        h = silu * b
        H = 1.1 * A * b.abs() + silu.abs() * Bd + 1.1 * A * Bd + 2.0 ** -20 * h.abs()
        H = H + torch.maximum(2.0 ** -9 * (h.abs() + H), 2.0 ** -21 * top(h.abs() + H))
        out += 0.5 * (h @ wd.t())
        bound += 0.5 * ((H + 2.0 ** -20 * h.abs()) @ wd.abs().t())
    assert bool(((got - out).abs() <= bound + 2.0 ** -9 * (out.abs() + bound)).all())


@pytest.mark.gpu
def test_few_again_and_again_on_one_workspace():
    """Counters return to zero, sums do not depend on the blocks' order, and sizes may change."""
    from paper_2411_02581_b200 import moe
    e, k, d, i = 8, 2, 512, 256
    w13, w2 = bf16_weights(2 * e, i, d, 1).view(e, 2, i, d), bf16_weights(e, d, i, 2)
    router = bf16_weights(1, e, d, 3)[0]
    ws = moe.few_workspace(64, e, k, d, i)
    xs = [activations(t, d, t).cuda() for t in (1, 64, 5, 17)]
    want = [moe.few(x, router, k, w13, w2) for x in xs]
    for _ in range(10):
        for x, y in zip(xs, want):
            assert torch.equal(moe.few(x, router, k, w13, w2, workspace=ws), y)
    assert moe.few(xs[0][:0], router, k, w13, w2).shape == (0, d)
    wide = torch.zeros(17, d + 3, dtype=torch.bfloat16, device="cuda")
    wide[:, 3:] = xs[3]
    assert torch.equal(moe.few(wide[:, 3:], router, k, w13, w2), want[3])


@pytest.mark.gpu
def test_few_and_experts_on_another_stream_and_in_a_graph():
    from paper_2411_02581_b200 import moe
    e, k, d, i, t = 8, 2, 256, 256, 6
    w13, s13 = fp8_weights(2 * e, i, d, 1)
    w2, s2 = fp8_weights(e, d, i, 2)
    w13, s13 = w13.view(e, 2, i, d), s13.view(e, 2, *s13.shape[1:])
    router, x = bf16_weights(1, e, d, 3)[0], activations(t, d, 1).cuda()
    ids, w = torch.empty(t, k, dtype=torch.int32, device="cuda"), torch.empty(t, k, device="cuda")
    few = lambda **kw: moe.few(x, router, k, w13, w2, s13=s13, s2=s2, ids=ids, weights=w, **kw)  # noqa: E731
    want = few()
    want_many = moe.experts(x, ids, w, w13, s13, w2, s2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got, many = few(stream=side), moe.experts(x, ids, w, w13, s13, w2, s2, stream=side)
    side.synchronize()
    assert torch.equal(got, want) and torch.equal(many, want_many)
    ws = moe.few_workspace(t, e, k, d, i)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a, b = few(workspace=ws), moe.experts(x, ids, w, w13, s13, w2, s2)
    for seed in (2, 3):
        x.copy_(activations(t, d, seed))
        graph.replay()
        assert torch.equal(a, few()) and torch.equal(b, moe.experts(x, ids, w, w13, s13, w2, s2))


def test_layer_refusals():
    """Refused on the host, before any GPU work (pointers are never followed)."""
    build_mod.build()
    L = B.lib()
    n, z = B.ctypes.c_size_t(), B.ctypes.c_size_t()
    size = lambda *a: L.tuna_moe_few_workspace_bytes(*a, B.ctypes.byref(n), B.ctypes.byref(z))  # noqa: E731
    assert size(64, 64, 2, 4096, 2048) == 0 and 0 < z.value < n.value
    assert size(65, 64, 2, 4096, 2048) == -9 and size(1, 513, 2, 64, 64) == -9 and size(1, 64, 33, 64, 64) == -9
    assert size(1, 64, 2, 8208, 64) == -9 and size(1, 64, 2, 64, 8208) == -9
    assert size(1, 64, 2, 72, 64) == -1 and size(1, 64, 2, 64, 8) == -1 and size(1, 2, 3, 64, 64) == -1 and size(-1, 2, 1, 64, 64) == -1
    size(4, 8, 2, 64, 64)

    def few(x=256, ldx=64, t=4, router=256, scoring=0, dt=1, s=256, out=256, ldo=64, ws=256, nb=None):
        return L.tuna_moe_few(x, ldx, t, router, 8, 2, scoring, 0, 1.0, 64, 64, dt, 256, s, 256, s, out, ldo, None, None, ws,
                              n.value if nb is None else nb, None)
    assert few(x=None) == -1 and few(x=264) == -1 and few(ldx=56) == -1 and few(ldx=68) == -1 and few(router=None) == -1
    assert few(scoring=2) == -1 and few(dt=0) == -1 and few(dt=2, s=None) == -1 and few(out=257) == -1 and few(ldo=63) == -1
    assert few(ws=None) == -6 and few(ws=128) == -6 and few(nb=16) == -6 and few(t=0) == 0

    many = lambda *a: L.tuna_moe_experts_workspace_bytes(*a, B.ctypes.byref(n))  # noqa: E731
    assert many(100, 64, 2, 4096, 2048) == 0 and many(100, 64, 0, 64, 64) == -1 and many(-1, 64, 2, 64, 64) == -1
    assert many(100, 64, 2, 72, 64) == -1 and many(100, 513, 2, 64, 64) == -9 and many(1 << 25, 64, 2, 64, 64) == -9
    many(4, 8, 2, 64, 64)

    def experts(x=256, ldx=64, ids=256, w13=256, s=256, out=256, ldo=64, ws=256, nb=None):
        return L.tuna_moe_experts(x, ldx, 4, ids, 256, 2, 8, 64, 64, w13, s, 256, s, out, ldo, ws, n.value if nb is None else nb, None)
    assert experts(x=None) == -1 and experts(ldx=63) == -1 and experts(ids=None) == -1 and experts(w13=264) == -1 and experts(s=None) == -1
    assert experts(out=None) == -1 and experts(ldo=63) == -1 and experts(ws=None) == -6 and experts(nb=1) == -6

    rows = L.tuna_moe_expert_rows
    assert L.tuna_moe_expert_rows_workspace_bytes(10, 64, 64, None) == -1
    assert rows(256, 64, 4, 8, None, 64, 64, 256, 256, 256, 256, 256, 64, 256, 1 << 20, None) == -1     # no offsets
    assert rows(256, 64, 4, 8, 256, 64, 64, 256, 256, 256, 256, 256, 64, 256, 8, None) == -6
    assert rows(None, 64, 0, 8, None, 64, 64, None, None, None, None, None, 64, None, 0, None) == 0


def test_marshalling_is_built_and_refuses_on_the_host():
    """The C++ marshalling loads, binds to the library and raises the Python errors (no GPU needed)."""
    import subprocess
    import sys
    from paper_2411_02581_b200 import moe
    build_mod.build()
    fast = moe._fast()
    with pytest.raises(ValueError, match="CUDA tensor"):
        moe.fp8_quantize(torch.zeros(4, 4))
    with pytest.raises(ValueError, match="layout"):
        moe.fp8_quantize(torch.zeros(4, 4), "diagonal")
    with pytest.raises(ValueError, match="a tensor is wanted"):
        moe.fp8_matmul(None, None, None, None)
    with pytest.raises(ValueError, match="b_blocks"):
        moe.fp8_matmul(None, None, None, None, b_blocks="columns")
    with pytest.raises(TypeError, match="7 arguments"):
        fast.route(1)
    missing = "import os; from paper_2411_02581_b200 import build, moe; build.TORCH_PATH = os.devnull + '/none'; moe._fast()"
    r = subprocess.run([sys.executable, "-c", missing], capture_output=True, text=True, cwd=build_mod.ROOT)
    assert r.returncode != 0 and "is missing: build it" in r.stderr
