"""8-bit quantisation and block-scaled products against plain 64-bit implementations.

Quantisation is defined bit by bit, so it is compared bit by bit.  A product of quantised
operands is compared with the 64-bit one: the sums over a block of 128 are exact to 2^-23 of
their terms' magnitude, the outer sum adds at most one rounding of 2^-24 a block, so the error
stays below (blocks + 8) * 2^-23 of sum |a b| (2e-5 at 130 blocks); bf16 results add half a
unit of 2^-8.
"""
import pytest
import torch

from paper_2411_02581_b200 import binding as B
from paper_2411_02581_b200 import build as build_mod

FP8 = torch.float8_e4m3fn


def plain_quantize(x, layout):
    """On the CPU: (q, scale) of a 32-bit matrix."""
    x = x.float()
    if layout == "columns":
        return plain_quantize(x.t().contiguous(), "rows")
    if layout == "tiles_t":
        return plain_quantize(x.t().contiguous(), "tiles")
    r, c = x.shape
    br = 128 if layout == "tiles" else 1
    p = torch.nn.functional.pad(x, (0, -c % 128, 0, -r % br))
    b = p.view(p.shape[0] // br, br, p.shape[1] // 128, 128)
    amax = b.abs().amax((1, 3))
    amax = torch.where(torch.isfinite(amax), amax, torch.full_like(amax, float("nan")))
    s = torch.clamp(amax, min=2.0 ** -100) / torch.full_like(amax, 448.0)
    q = (b / s[:, None, :, None]).to(FP8).reshape(p.shape)[:r, :c]
    return q, (s if layout == "tiles" else s.t().contiguous())


def value(q, s, blocks):
    q = q.cpu().double()
    s = s.cpu().double()
    n, k = q.shape
    kb = torch.arange(k) // 128
    return q * (s.t()[:, kb] if blocks == "rows" else s[torch.arange(n) // 128][:, kb])


def close(got, a, b, bf16):
    got, want, size = got.cpu().double(), a @ b.t(), a.abs() @ b.abs().t()
    blocks = -(-a.shape[1] // 128)
    tol = (blocks + 8) * 2.0 ** -23 * size + (2.0 ** -8 * want.abs() if bf16 else 0) + 1e-30
    return bool(((got - want).abs() <= tol).all())


def activations(rows, cols, seed, dtype=torch.bfloat16):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g)
    x[:, torch.rand(cols, generator=g) < 0.02] *= 30
    return x.to(dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["rows", "columns", "tiles", "tiles_t"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 128), (3, 16), (128, 128), (130, 520), (257, 1000), (5, 4099), (700, 96)])
def test_quantize_is_the_definition(rows, cols, dtype, layout):
    from paper_2411_02581_b200 import moe
    x = activations(rows, cols, rows + cols, dtype)
    if rows > 3:
        x[1] = 0                                   # a block of zeros
        x[2] *= 1e-30                              # below the floor of the scale
    q, s = moe.fp8_quantize(x.cuda(), layout)
    wq, ws = plain_quantize(x, layout)
    assert torch.equal(s.cpu(), ws)
    assert torch.equal(q.cpu().view(torch.uint8), wq.view(torch.uint8))


@pytest.mark.gpu
def test_quantize_strided_and_misaligned_rows():
    from paper_2411_02581_b200 import moe
    x = activations(200, 300, 3)
    big = torch.zeros(200, 411, dtype=torch.bfloat16, device="cuda")
    big[:, 5:305] = x.cuda()
    for layout in ("rows", "columns", "tiles", "tiles_t"):
        (a, sa), (b, sb) = moe.fp8_quantize(x.cuda(), layout), moe.fp8_quantize(big[:, 5:305], layout)
        assert torch.equal(sa, sb) and torch.equal(a.view(torch.uint8), b.view(torch.uint8))


@pytest.mark.gpu
def test_quantize_keeps_what_is_not_finite():
    from paper_2411_02581_b200 import moe
    x = torch.ones(4, 256)
    x[1, 3], x[2, 200], x[3, 7] = float("nan"), float("inf"), -float("inf")
    for layout, bad in (("rows", [[0, 1, 0, 1], [0, 0, 1, 0]]), ("tiles", [[1, 1]])):
        _, s = moe.fp8_quantize(x.cuda(), layout)
        assert torch.equal(torch.isnan(s.cpu()), torch.tensor(bad, dtype=torch.bool))
    q, s = moe.fp8_quantize(x.cuda())
    w, ws = moe.fp8_quantize(torch.ones(8, 256, device="cuda"), "tiles")
    y = moe.fp8_matmul(q, s, w, ws).cpu()
    assert bool(torch.isnan(y[1:]).all()) and bool(torch.isfinite(y[0]).all())


PRODUCTS = [(1, 1, 1), (1, 128, 128), (1, 4096, 512), (2, 100, 300), (17, 640, 2064), (64, 256, 128), (65, 1000, 1040), (128, 256, 4096),
            (129, 257, 130), (300, 2000, 272), (1000, 96, 1024), (2500, 2304, 256), (20000, 517, 144), (0, 64, 64), (5, 7, 0)]


@pytest.mark.gpu
@pytest.mark.parametrize("out_dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("b_blocks", ["tiles", "rows"])
@pytest.mark.parametrize("m,n,k", PRODUCTS)
def test_product(m, n, k, b_blocks, out_dtype):
    from paper_2411_02581_b200 import moe
    a, b = activations(m, k, m + 1), activations(n, k, n + 2)
    qa, sa = moe.fp8_quantize(a.cuda(), "rows")
    qb, sb = moe.fp8_quantize(b.cuda(), b_blocks)
    got = moe.fp8_matmul(qa, sa, qb, sb, b_blocks=b_blocks, out_dtype=out_dtype)
    assert got.shape == (m, n) and got.dtype == out_dtype
    assert close(got, value(qa, sa, "rows"), value(qb, sb, b_blocks), out_dtype == torch.bfloat16)
    assert moe.device_status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("n,k", [(256, 512), (300, 144), (2048, 1024)])
@pytest.mark.parametrize("sizes", [[5], [0, 3, 0, 200, 128, 1, 0], [129, 127, 64, 1000], [0, 0], [1] * 60])
def test_grouped_product(n, k, sizes):
    from paper_2411_02581_b200 import moe
    g, spare = len(sizes), 9                       # rows behind the last group stay as they are
    offsets = torch.tensor([0] + sizes).cumsum(0)
    m = int(offsets[-1]) + spare
    a, b = activations(m, k, 4), activations(g * n, k, 5)
    qa, sa = moe.fp8_quantize(a.cuda(), "rows")
    parts = [moe.fp8_quantize(b[i * n:(i + 1) * n].cuda(), "tiles") for i in range(g)]
    qb, sb = torch.stack([p[0].view(torch.uint8) for p in parts]).view(FP8), torch.stack([p[1] for p in parts])
    got = moe.fp8_matmul(qa, sa, qb, sb, offsets=offsets.cuda())
    va = value(qa, sa, "rows")
    for i in range(g):
        lo, hi = int(offsets[i]), int(offsets[i + 1])
        assert close(got[lo:hi], va[lo:hi], value(qb[i], sb[i], "tiles"), True), i
    assert moe.device_status() == 0


@pytest.mark.gpu
def test_rows_outside_the_groups_are_left_alone():
    L = B.lib()
    from paper_2411_02581_b200 import moe
    a, w = torch.ones(300, 128, device="cuda"), torch.ones(2 * 64, 128, device="cuda")
    qa, sa = moe.fp8_quantize(a)
    qw, sw = moe.fp8_quantize(w[:64], "tiles")
    qw, sw = torch.cat([qw.view(torch.uint8)] * 2).view(FP8), torch.cat([sw] * 2)
    off = torch.tensor([10, 20, 250], device="cuda")
    out = torch.full((300, 64), 7.0, device="cuda")
    assert L.tuna_fp8_matmul(qa.data_ptr(), sa.data_ptr(), 300, 128, qw.data_ptr(), sw.data_ptr(), 2, 64, 128, 128, 2, off.data_ptr(),
                             out.data_ptr(), 0, 64, None) == 0
    torch.cuda.synchronize()
    want = value(qa, sa, "rows")[10:250], value(qw[:64], sw[:1], "tiles")   # (448 * fl(1 / 448) is not quite 1)
    assert close(out[10:250], *want, False) and bool((out[:10] == 7).all()) and bool((out[250:] == 7).all())


@pytest.mark.gpu
def test_offsets_that_are_no_offsets_are_cut_to_the_operand():
    """Falling, negative and too large ones: no row outside the operand is read or written, and the call ends."""
    from paper_2411_02581_b200 import moe
    m, n, k = 100, 72, 144
    a, w = activations(m, k, 1), activations(5 * n, k, 2)
    qa, sa = moe.fp8_quantize(a.cuda())
    tiles = [moe.fp8_quantize(w[i * n:(i + 1) * n].cuda(), "tiles") for i in range(5)]
    qw, sw = torch.stack([q.view(torch.uint8) for q, _ in tiles]).view(FP8), torch.stack([s for _, s in tiles])
    for offsets, alone in (([50, 20, -5, 1 << 40, 10, 0], 2), ([-(1 << 63), (1 << 63) - 1, 0, -(1 << 63), 0, 0], 0), ([7, 7, 7, 7, 7, 7], None)):
        space = torch.full((m + 64, n), 7.0, dtype=torch.bfloat16, device="cuda")     # canaries on both sides
        assert B.lib().tuna_fp8_matmul(qa.data_ptr(), sa.data_ptr(), m, k, qw.data_ptr(), sw.data_ptr(), 2, n, k, k, 5,
                                       torch.tensor(offsets, device="cuda").data_ptr(), space[32:].data_ptr(), 1, n, None) == 0
        torch.cuda.synchronize()
        assert bool((space[:32] == 7).all()) and bool((space[32 + m:] == 7).all())
        out = space[32:32 + m]
        if alone is None:
            assert bool((out == 7).all())
        else:
            assert close(out, value(qa, sa, "rows"), value(qw[alone], sw[alone], "tiles"), True)
    # all rows in each of the groups: many more tiles than rows, the same results from equal matrices
    same = torch.stack([qw[0].view(torch.uint8)] * 5).view(FP8)
    overlapping = torch.tensor([0, m, 0, m, 0, m], device="cuda")
    got = moe.fp8_matmul(qa, sa, same, torch.stack([sw[0]] * 5), offsets=overlapping)
    assert close(got, value(qa, sa, "rows"), value(qw[0], sw[0], "tiles"), True)
    assert moe.device_status() == 0


@pytest.mark.gpu
def test_layer_gradients_against_the_formula_and_differences():
    """dx and dw of y = x w^T: the formula on the quantised operands, and the change of <y, dy>."""
    from paper_2411_02581_b200 import moe
    m, n, k = 200, 384, 272
    x, w, dy = activations(m, k, 1).cuda(), activations(n, k, 2).cuda(), activations(m, n, 3).cuda()
    wt, swt = moe.fp8_quantize(w, "tiles_t")
    q, s = moe.fp8_quantize(dy, "rows")
    dx = moe.fp8_matmul(q, s, wt, swt)
    assert close(dx, value(q, s, "rows"), value(wt, swt, "tiles"), True)
    qt, st = moe.fp8_quantize(dy, "columns")
    xt, sxt = moe.fp8_quantize(x, "columns")
    dw = moe.fp8_matmul(qt, st, xt, sxt, b_blocks="rows", out_dtype=torch.float32)
    assert close(dw, value(qt, st, "rows"), value(xt, sxt, "rows"), False)

    # A quantised value is within 2^-4 of its value (half a unit of 3 fraction bits), so <step, g> is within
    # 2 * 2^-4 + 2^-8 < 0.14 of the sum of its terms' magnitudes; a random direction is far inside.
    def rise(f, at, step):
        return float((f(at + step) - f(at - step)) / 2)
    X, Wd, G = x.double().cpu(), w.double().cpu(), dy.double().cpu()
    step = torch.randn(m, k, dtype=torch.float64, generator=torch.Generator().manual_seed(7))
    size = float((step.abs() * (G.abs() @ Wd.abs())).sum())
    assert abs(rise(lambda v: (v @ Wd.t() * G).sum(), X, step) - float((dx.cpu().double() * step).sum())) <= 0.14 * size
    step = torch.randn(n, k, dtype=torch.float64, generator=torch.Generator().manual_seed(8))
    size = float((step.abs() * (G.abs().t() @ X.abs())).sum())
    assert abs(rise(lambda v: (X @ v.t() * G).sum(), Wd, step) - float((dw.cpu().double() * step).sum())) <= 0.14 * size


@pytest.mark.gpu
def test_operands_off_16_bytes_and_other_streams():
    from paper_2411_02581_b200 import moe
    x, w = activations(50, 272, 1).cuda(), activations(80, 272, 2).cuda()
    q, s = moe.fp8_quantize(x)
    v, t = moe.fp8_quantize(w, "tiles")
    want = moe.fp8_matmul(q, s, v, t)
    odd = torch.zeros(50, 281, dtype=torch.uint8, device="cuda")
    odd[:, 3:275] = q.view(torch.uint8)
    assert torch.equal(moe.fp8_matmul(odd[:, 3:275].view(FP8), s, v, t), want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    q2, s2 = moe.fp8_quantize(x, stream=side)
    got = moe.fp8_matmul(q2, s2, v, t, stream=side)
    side.synchronize()
    assert torch.equal(got, want)


@pytest.mark.gpu
def test_more_values_than_32_bits_count():
    """2^31 + values: the last rows of the operand and of the result are where they should be."""
    from paper_2411_02581_b200 import moe
    m, k, n = 66000, 32768, 40
    x = torch.empty(m, k, dtype=torch.bfloat16, device="cuda")
    x.view(torch.int16).copy_(torch.arange(k, device="cuda").remainder(251).to(torch.int16)[None, :] + 0x3f00)
    tail = activations(5, k, 1).cuda()
    x[-5:] = tail
    q, s = moe.fp8_quantize(x)
    wq, ws = plain_quantize(tail.cpu(), "rows")
    assert torch.equal(s[:, -5:].cpu(), ws) and torch.equal(q[-5:].cpu().view(torch.uint8), wq.view(torch.uint8))
    v, t = moe.fp8_quantize(activations(n, k, 2).cuda(), "tiles")
    y = moe.fp8_matmul(q, s, v, t)
    assert close(y[-5:], value(wq, ws, "rows"), value(v, t, "tiles"), True)
    assert torch.equal(y[0], y[m - 6])            # equal rows give equal results wherever they are
    del x, q, y
    torch.cuda.empty_cache()


@pytest.mark.gpu
def test_one_answer_however_often():
    from paper_2411_02581_b200 import moe
    q, s = moe.fp8_quantize(activations(7, 4096, 1).cuda())
    v, t = moe.fp8_quantize(activations(1024, 4096, 2).cuda(), "tiles")
    want = moe.fp8_matmul(q, s, v, t, out_dtype=torch.float32)
    for _ in range(20):
        assert torch.equal(moe.fp8_matmul(q, s, v, t, out_dtype=torch.float32), want)


def test_fp8_refusals():
    """Refused on the host, before any GPU work (pointers are never followed)."""
    build_mod.build()
    L = B.lib()

    def quantize(x=256, dtype=1, rows=4, cols=64, ld=64, layout=0, q=256, ldq=64, s=256):
        return L.tuna_fp8_quantize(x, dtype, rows, cols, ld, layout, q, ldq, s, None)
    assert quantize(dtype=2) == -1 and quantize(ld=63) == -1 and quantize(layout=4) == -1 and quantize(layout=-1) == -1
    assert quantize(ldq=48) == -1 and quantize(ldq=72) == -1 and quantize(layout=1, rows=65) == -1
    assert quantize(x=None) == -1 and quantize(x=257) == -1 and quantize(q=264) == -1 and quantize(s=None) == -1
    assert quantize(cols=1 << 25, ld=1 << 25, ldq=1 << 25) == -9
    assert quantize(rows=-1) == -1 and quantize(rows=0) == 0 and quantize(cols=0) == 0

    def product(a=256, sa=256, m=4, lda=64, b=256, sb=256, layout=2, n=8, ldb=64, k=64, groups=1, off=None, out=256, dt=1, ldo=8):
        return L.tuna_fp8_matmul(a, sa, m, lda, b, sb, layout, n, ldb, k, groups, off, out, dt, ldo, None)
    assert product(lda=63) == -1 and product(lda=72) == -1 and product(ldb=40) == -1 and product(ldo=7) == -1
    assert product(layout=1) == -1 and product(layout=3) == -1 and product(groups=2) == -1 and product(layout=0, groups=2, off=256) == -1
    assert product(dt=2) == -1 and product(a=None) == -1 and product(a=264) == -1 and product(b=264) == -1 and product(out=257) == -1
    assert product(groups=513, off=256) == -9 and product(m=0) == 0 and product(n=0, ldo=0) == 0 and product(m=-1) == -1
