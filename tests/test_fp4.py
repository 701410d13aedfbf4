"""4-bit microscaled quantisation and products against plain 64-bit implementations.

Quantisation is defined bit by bit, so it is compared bit by bit.  A product of quantised operands has exact terms; the
tensor cores add 64 of them to the 32-bit sum at a time, off by at most 2^-23 of the magnitude of all terms so far, so
after k / 64 steps the error stays below (k / 64 + 8) * 2^-23 of sum |a b|; bf16 results add half a unit of 2^-8.
"""
import pytest
import torch

from paper_2411_02581_b200 import binding as B
from paper_2411_02581_b200 import build as build_mod
from test_fp8 import activations

FP4, POWER = torch.float4_e2m1fn_x2, torch.float8_e8m0fnu
GRID = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64)
BAD = 255


def plain_quantize(x, layout="rows"):
    """On the CPU, from the definition: codes [rows, cols] (sign in bit 3) and bytes [rows, blocks of 32]."""
    x = x.double()
    if layout == "columns":
        x = x.t().contiguous()
    r, c = x.shape
    b = torch.nn.functional.pad(x, (0, -c % 32)).view(r, -1, 32)
    top = b.abs().amax(2)
    bad = ~torch.isfinite(b).all(2)
    e = torch.frexp(torch.where(bad, torch.ones_like(top), top)).exponent - 1 - 2
    byte = torch.where(top == 0, torch.zeros_like(e), e + 127).clamp(min=0)
    v = (b * torch.exp2(127 - byte.double())[:, :, None]).abs()
    v = torch.where(bad[:, :, None], torch.zeros_like(v), v)
    low = (torch.bucketize(v, GRID, right=True) - 1).clamp(max=6)
    mid = (GRID[low] + GRID[low + 1]) / 2
    code = low + ((v > mid) | ((v == mid) & (low % 2 == 1))).long()
    code = code + 8 * torch.signbit(b).long()
    return code.view(r, -1)[:, :c], torch.where(bad, torch.full_like(byte, BAD), byte)


def plain_value(code, byte):
    v = GRID[code & 7] * torch.where(code > 7, -1.0, 1.0)
    s = torch.exp2(byte.double() - 127)
    s = torch.where(byte == BAD, torch.full_like(s, float("nan")), s)
    return v * s.repeat_interleave(32, 1)[:, :v.shape[1]]


def stored(x):
    return plain_value(*plain_quantize(x))


def codes(q, cols):
    q = q.cpu().contiguous().view(torch.uint8).long()
    return torch.stack([q & 15, q >> 4], -1).flatten(-2)[..., :cols]


def bytes_of(s, rows, blocks, offsets=None):
    """The scales' bytes [rows, blocks] out of their tiles."""
    s = s.cpu().view(torch.uint8).long()
    r, b = torch.arange(rows)[:, None], torch.arange(blocks)[None, :]
    tile, at = r // 128, r % 128
    if offsets is not None:
        g = (torch.bucketize(r, torch.tensor(offsets), right=True) - 1).clamp(0, len(offsets) - 2)
        first = torch.tensor(offsets)[g]
        tile, at = first // 128 + g + (r - first) // 128, (r - first) % 128
    return s[tile, b // 4, at % 32, at // 32, b % 4]


def value(q, s, cols=None):
    """The values of a quantised matrix, in 64 bits."""
    cols = 2 * q.shape[1] if cols is None else cols
    return plain_value(codes(q, cols), bytes_of(s, q.shape[0], -(-cols // 32)))


def close(got, a, b, bf16):
    got, want, size = got.cpu().double(), a @ b.t(), a.abs() @ b.abs().t()
    tol = (a.shape[1] / 64 + 8) * 2.0 ** -23 * size + (2.0 ** -8 * want.abs() if bf16 else 0) + 1e-37
    return bool(((got - want).abs() <= tol).all())


def same(a, b):
    return all(torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8)) for x, y in zip(a, b))


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["rows", "columns"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 32), (3, 33), (31, 64), (128, 128), (130, 520), (257, 1000), (5, 4099), (700, 96), (97, 2)])
def test_quantize_is_the_definition(rows, cols, dtype, layout):
    from paper_2411_02581_b200 import moe
    x = activations(rows, cols, rows + cols, dtype)
    if rows > 3:
        x[1] = 0                                            # a block of zeros
        x[2] = (x[2].double() * 2.0 ** -127).to(dtype)      # below the smallest scale
        x[3] = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0, -0.25, -5.0, 4.0] * (cols // 12 + 1))[:cols].to(dtype)  # halves
    q, s = moe.fp4_quantize(x.cuda(), layout)
    code, byte = plain_quantize(x, layout)
    n, k = code.shape
    assert q.shape == (n, (k + 1) // 2) and q.dtype == FP4 and s.shape == (-(-n // 128), -(-k // 128), 32, 4, 4) and s.dtype == POWER
    assert torch.equal(bytes_of(s, n, byte.shape[1]), byte)
    assert torch.equal(codes(q, k), code)
    assert bool((bytes_of(s, n, 4 * s.shape[1]) != BAD).all())    # nor is a scale behind the last column
    if k % 2:
        assert bool((codes(q, k + 1)[:, k] == 0).all())
    for out in (torch.bfloat16, torch.float32):
        back = moe.fp4_dequantize(q, s, out_dtype=out)
        assert back.dtype == out and torch.equal(back[:, :k].cpu().double(), plain_value(code, byte))


@pytest.mark.gpu
def test_quantize_strided_and_misaligned_rows():
    from paper_2411_02581_b200 import moe
    for dtype in (torch.bfloat16, torch.float32):
        x = activations(200, 300, 3, dtype)
        big = torch.zeros(200, 411, dtype=dtype, device="cuda")
        big[:, 5:305] = x.cuda()
        for layout in ("rows", "columns"):
            a, b = moe.fp4_quantize(x.cuda(), layout), moe.fp4_quantize(big[:, 5:305], layout)
            n, blocks = a[0].shape[0], -(-(a[0].shape[1] * 2) // 32)
            assert same(a[:1], b[:1]) and torch.equal(bytes_of(a[1], n, blocks), bytes_of(b[1], n, blocks))
        q, s = moe.fp4_quantize(x.cuda())
        odd = torch.zeros(200, 211, dtype=torch.uint8, device="cuda")
        odd[:, 3:153] = q.view(torch.uint8)
        assert torch.equal(moe.fp4_dequantize(odd[:, 3:153].view(FP4), s), moe.fp4_dequantize(q, s))


@pytest.mark.gpu
def test_quantize_values_at_the_ends_of_the_range_and_not_finite():
    from paper_2411_02581_b200 import moe
    x = torch.ones(8, 160)
    x[1, 3], x[2, 100], x[3, 159] = float("nan"), float("inf"), -float("inf")
    x[4] = torch.finfo(torch.float32).max
    x[5] = 2.0 ** -149
    x[6, 32:64] = torch.linspace(-1, 1, 32) * 2.0 ** -126
    code, byte = plain_quantize(x)
    for y in (x, x.to(torch.bfloat16)):
        code, byte = plain_quantize(y)
        q, s = moe.fp4_quantize(y.cuda())
        got, fine = bytes_of(s, 8, 5), byte != BAD
        assert torch.equal(got, byte)
        wide = fine.repeat_interleave(32, 1)
        assert torch.equal(codes(q, 160)[wide], code[wide])
        back = moe.fp4_dequantize(q, s, out_dtype=torch.float32).cpu().double()
        assert torch.equal(torch.isnan(back), ~wide) and torch.equal(back[wide], plain_value(code, byte)[wide])
        w = moe.fp4_quantize(torch.ones(8, 160, device="cuda"))
        prod = moe.fp4_matmul(q, s, *w, out_dtype=torch.float32).cpu()
        assert bool(torch.isnan(prod[1:4]).all()) and bool(torch.isfinite(prod[[0, 5, 6, 7]]).all())
        # 160 terms of 6 * 2^125 are over 2^128; as bf16 the value itself is infinite, and its scale NaN
        assert bool((prod[4] == float("inf")).all() if y.dtype == torch.float32 else torch.isnan(prod[4]).all())


GROUPS = [[5], [0, 3, 0, 200, 128, 1, 0], [129, 127, 64, 300], [0, 0], [1] * 60, [128, 256], [3] * 300]


@pytest.mark.gpu
@pytest.mark.parametrize("sizes", GROUPS)
def test_quantize_in_groups(sizes):
    from paper_2411_02581_b200 import moe
    for first, spare in ((0, 0), (7, 9)):                   # rows of no group in front and behind
        bounds = (torch.tensor([0] + sizes).cumsum(0) + first).tolist()
        m, k = bounds[-1] + spare, 200
        if m == 0:
            continue
        x = activations(m, k, 4)
        offsets = torch.tensor(bounds, device="cuda")
        q, s = moe.fp4_quantize(x.cuda(), offsets=offsets)
        assert s.shape == (m // 128 + len(sizes), 2, 32, 4, 4)
        code, byte = plain_quantize(x)
        at = slice(bounds[0], bounds[-1])
        assert torch.equal(codes(q, k)[at], code[at]) and torch.equal(bytes_of(s, m, 7, bounds)[at], byte[at])
        assert torch.equal(moe.fp4_dequantize(q, s, offsets=offsets, out_dtype=torch.float32)[at].cpu().double(), plain_value(code, byte)[at])


PRODUCTS = [(1, 1, 2), (1, 128, 128), (1, 4096, 512), (2, 100, 300), (17, 640, 2064), (64, 256, 128), (65, 1000, 1040), (128, 256, 4096),
            (129, 257, 130), (300, 2000, 272), (1000, 96, 1024), (2500, 2304, 256), (20000, 517, 144), (0, 64, 64), (5, 7, 0), (3, 130, 2895),
            (513, 4000, 2894), (700, 5000, 66), (2049, 1025, 4096), (8201, 3585, 290), (57000, 517, 130)]


@pytest.mark.gpu
@pytest.mark.parametrize("out_dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("m,n,k", PRODUCTS)
def test_product(m, n, k, out_dtype):
    from paper_2411_02581_b200 import moe
    a, b = activations(m, k, m + 1), activations(n, k, n + 2)
    qa, sa = moe.fp4_quantize(a.cuda())
    qb, sb = moe.fp4_quantize(b.cuda())
    got = moe.fp4_matmul(qa, sa, qb, sb, out_dtype=out_dtype)
    assert got.shape == (m, n) and got.dtype == out_dtype
    assert close(got, value(qa, sa), value(qb, sb), out_dtype == torch.bfloat16)
    assert moe.device_status() == 0


@pytest.mark.gpu
def test_product_of_scales_that_differ_in_every_block():
    """Blocks from 2^-60 to 2^60 of each other: every scale meets its own block."""
    from paper_2411_02581_b200 import moe
    g = torch.Generator().manual_seed(2)
    for m, n, k in ((140, 300, 800), (600, 1100, 512)):
        a, b = (torch.randn(r, k, generator=g) * torch.exp2(torch.randint(-60, 61, (r, k // 32), generator=g).float()).repeat_interleave(32, 1) for r in (m, n))
        qa, qb = moe.fp4_quantize(a.cuda()), moe.fp4_quantize(b.cuda())
        assert close(moe.fp4_matmul(*qa, *qb, out_dtype=torch.float32), value(*qa), value(*qb), False)


def grouped(sizes, n, k, first=0, spare=9):
    from paper_2411_02581_b200 import moe
    g = len(sizes)
    bounds = (torch.tensor([0] + sizes).cumsum(0) + first).tolist()
    m = bounds[-1] + spare
    a, b = activations(m, k, 4), activations(g * n, k, 5)
    offsets = torch.tensor(bounds, device="cuda")
    parts = [moe.fp4_quantize(b[i * n:(i + 1) * n].cuda()) for i in range(g)]
    return a, offsets, bounds, torch.stack([p[0].contiguous() for p in parts]), torch.stack([p[1] for p in parts])


@pytest.mark.gpu
@pytest.mark.parametrize("n,k", [(256, 512), (300, 144), (2048, 1024), (2800, 130)])
@pytest.mark.parametrize("sizes", GROUPS[:6] + [[700, 0, 513, 40], [1500, 0, 2561, 700, 1], [5000, 3000, 2600]])
def test_grouped_product(n, k, sizes):
    from paper_2411_02581_b200 import moe
    a, offsets, bounds, qb, sb = grouped(sizes, n, k, first=3)
    qa, sa = moe.fp4_quantize(a.cuda(), offsets=offsets)
    for dtype in (torch.bfloat16, torch.float32):
        got = moe.fp4_matmul(qa, sa, qb, sb, offsets=offsets, out_dtype=dtype)
        va = stored(a)
        for i in range(len(sizes)):
            lo, hi = bounds[i], bounds[i + 1]
            assert close(got[lo:hi], va[lo:hi], value(qb[i], sb[i], k), dtype == torch.bfloat16), i
    assert moe.device_status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [0, 1])
def test_rows_outside_the_groups_are_left_alone(dt):
    from paper_2411_02581_b200 import moe
    a, _, _, qb, sb = grouped([10, 230], 72, 128)
    bounds = [10, 20, 245]
    offsets = torch.tensor(bounds, device="cuda")
    m = a.shape[0]
    q, s = torch.full((m, 64), 0x77, dtype=torch.uint8, device="cuda"), torch.empty(m // 128 + 2, 1, 512, dtype=torch.uint8, device="cuda")
    x = a.cuda()
    assert B.lib().tuna_fp4_quantize(x.data_ptr(), 1, m, 128, 128, 0, 2, offsets.data_ptr(), q.data_ptr(), 64, s.data_ptr(), None) == 0
    out = torch.full((m, 72), 7.0, device="cuda", dtype=(torch.float32, torch.bfloat16)[dt])
    assert B.lib().tuna_fp4_matmul(q.data_ptr(), s.data_ptr(), m, 64, qb.data_ptr(), sb.data_ptr(), 72, 64, 128, 2, offsets.data_ptr(), out.data_ptr(), dt, 72, None) == 0
    back = torch.full((m, 128), 7.0, device="cuda")
    assert B.lib().tuna_fp4_dequantize(q.data_ptr(), 64, s.data_ptr(), m, 128, 2, offsets.data_ptr(), back.data_ptr(), 0, 128, None) == 0
    torch.cuda.synchronize()
    for t, v in ((q, 0x77), (out, 7), (back, 7)):
        assert bool((t[:10] == v).all()) and bool((t[245:] == v).all())
    va = stored(a)
    assert close(out[10:20], va[10:20], value(qb[0], sb[0]), dt == 1) and close(out[20:245], va[20:245], value(qb[1], sb[1]), dt == 1)


@pytest.mark.gpu
def test_offsets_that_are_no_offsets_are_cut_to_the_operand():
    """Falling, negative and too large ones: no row outside the operand is read or written, and the calls end."""
    from paper_2411_02581_b200 import moe
    a, _, _, qb, sb = grouped([20] * 5, 72, 160, spare=0)
    m, n = 100, 72
    va = stored(a)
    for bounds, alone in (([50, 20, -5, 1 << 40, 10, 0], None), ([-(1 << 63), (1 << 63) - 1, 1 << 62, 1 << 62, 1 << 62, 1 << 62], 0), ([7] * 6, -1)):
        offsets = torch.tensor(bounds, device="cuda")
        q, s = moe.fp4_quantize(a.cuda(), offsets=offsets)
        space = torch.full((m + 64, n), 7.0, dtype=torch.bfloat16, device="cuda")     # canaries on both sides
        assert q.stride(0) == qb.stride(1) == 80
        assert B.lib().tuna_fp4_matmul(q.data_ptr(), s.data_ptr(), m, 80, qb.data_ptr(), sb.data_ptr(), n, 80, 160, 5, offsets.data_ptr(), space[32:].data_ptr(), 1, n, None) == 0
        torch.cuda.synchronize()
        got = moe.fp4_matmul(q, s, qb, sb, offsets=offsets)
        moe.fp4_dequantize(q, s, offsets=offsets)
        torch.cuda.synchronize()
        assert bool((space[:32] == 7).all()) and bool((space[32 + m:] == 7).all())
        if alone == 0:
            assert close(got, va, value(qb[0], sb[0]), True)
        if alone == -1:
            assert bool((space == 7).all())
    # all rows in each of the groups: many more tiles than rows (the call ends; results of rows that groups share mean nothing)
    overlapping = torch.tensor([0, m, 0, m, 0, m], device="cuda")
    q, s = moe.fp4_quantize(a.cuda(), offsets=overlapping)
    moe.fp4_matmul(q, s, qb, sb, offsets=overlapping)
    assert moe.device_status() == 0


@pytest.mark.gpu
def test_layer_gradients_against_the_formula_and_differences():
    """dx and dw of y = x w^T: the formula on the quantised operands, and the change of <y, dy>."""
    from paper_2411_02581_b200 import moe
    m, n, k = 200, 384, 272
    x, w, dy = activations(m, k, 1).cuda(), activations(n, k, 2).cuda(), activations(m, n, 3).cuda()
    q, wt = moe.fp4_quantize(dy), moe.fp4_quantize(w, "columns")
    dx = moe.fp4_matmul(*q, *wt)
    assert close(dx, stored(dy.cpu()), stored(w.cpu().t()), True)
    qt, xt = moe.fp4_quantize(dy, "columns"), moe.fp4_quantize(x, "columns")
    dw = moe.fp4_matmul(*qt, *xt, out_dtype=torch.float32)
    assert close(dw, stored(dy.cpu().t()), stored(x.cpu().t()), False)

    # A value v of a block moves by at most a quarter of the scale where |v| < 2 scale, by half of it below 4, by the whole of it
    # up to 6, and by |v| / 4 up to 8; the scale is at most a quarter of the block's largest value: max(|v| / 4, top / 16).
    def moves(v):
        b = torch.nn.functional.pad(v, (0, -v.shape[1] % 32)).view(v.shape[0], -1, 32).abs()
        return torch.maximum(b / 4, b.amax(2, keepdim=True) / 16).flatten(1)[:, :v.shape[1]]

    def rise(f, at, step):
        return float((f(at + step) - f(at - step)) / 2)
    X, Wd, G = x.double().cpu(), w.double().cpu(), dy.double().cpu()

    def bound(step, a, b):  # of <step, stored(a) stored(b)^T> against <step, a b^T>: each side moved
        da, db = moves(a), moves(b)
        return float((step.abs() * (da @ b.abs().t() + a.abs() @ db.t() + da @ db.t() + 2.0 ** -7 * a.abs() @ b.abs().t())).sum())
    step = torch.randn(m, k, dtype=torch.float64, generator=torch.Generator().manual_seed(7))
    assert abs(rise(lambda v: (v @ Wd.t() * G).sum(), X, step) - float((dx.cpu().double() * step).sum())) <= bound(step, G, Wd.t().contiguous())
    step = torch.randn(n, k, dtype=torch.float64, generator=torch.Generator().manual_seed(8))
    assert abs(rise(lambda v: (X @ v.t() * G).sum(), Wd, step) - float((dw.cpu().double() * step).sum())) <= bound(step, G.t().contiguous(), X.t().contiguous())


@pytest.mark.gpu
def test_operands_off_16_bytes_and_results_of_any_pitch():
    from paper_2411_02581_b200 import moe
    x, w = activations(200, 270, 1).cuda(), activations(150, 270, 2).cuda()
    (q, s), (v, t) = moe.fp4_quantize(x), moe.fp4_quantize(w)
    want = moe.fp4_matmul(q, s, v, t)
    odd = torch.zeros(200, 141, dtype=torch.uint8, device="cuda")
    odd[:, 3:138] = q.view(torch.uint8)
    assert torch.equal(moe.fp4_matmul(odd[:, 3:138].view(FP4), s, v, t), want)
    tight = torch.empty(150, 135, dtype=torch.uint8, device="cuda").copy_(v.view(torch.uint8)).view(FP4)
    assert torch.equal(moe.fp4_matmul(q, s, tight, t), want)
    for dt, dtype in ((0, torch.float32), (1, torch.bfloat16)):
        full = moe.fp4_matmul(q, s, v, t, out_dtype=dtype)
        for ldo, at in ((150, 1), (151, 0), (152, 0), (160, 8), (163, 3)):
            out = torch.full((202, ldo), 7.0, dtype=dtype, device="cuda")
            p = out.view(-1)[ldo + at:]
            assert B.lib().tuna_fp4_matmul(q.data_ptr(), s.data_ptr(), 200, q.stride(0), v.data_ptr(), t.data_ptr(), 150, v.stride(0), 270, 0, None,
                                           p.data_ptr(), dt, ldo, None) == 0
            torch.cuda.synchronize()
            got = p[:200 * ldo].view(200, ldo)[:, :150]
            assert torch.equal(got, full)
            p[:200 * ldo].view(200, ldo)[:, :150] = 7
            assert bool((out == 7).all())


@pytest.mark.gpu
@pytest.mark.parametrize("rows,count,pitch,at", [(1, 1, 1, 0), (7, 15, 15, 0), (200, 33, 37, 1), (300, 1448, 1448, 0), (33, 64, 66, 2), (50, 100, 104, 4), (9, 4097, 5000, 3)])
def test_rows_laid_on_16_bytes(rows, count, pitch, at):
    g = torch.Generator().manual_seed(rows)
    src = torch.randint(0, 256, (rows * pitch + at + 16,), dtype=torch.uint8, generator=g).cuda()
    ldo = (count + 15) // 16 * 16 + 16
    out = torch.full((rows, ldo), 7, dtype=torch.uint8, device="cuda")
    assert B.lib().tuna_fp4_align(src[at:].data_ptr(), pitch, rows, count, out.data_ptr(), ldo, None) == 0
    torch.cuda.synchronize()
    assert torch.equal(out[:, :count], src[at:at + rows * pitch].view(rows, pitch)[:, :count]) and bool((out[:, count:] == 7).all())


@pytest.mark.gpu
def test_more_values_than_32_bits_count():
    """2^31 + values: the last rows of the operand and of the result are where they should be."""
    from paper_2411_02581_b200 import moe
    m, k, n = 132000, 32768, 40
    x = torch.empty(m, k, dtype=torch.bfloat16, device="cuda")
    x.view(torch.int16).copy_(torch.arange(k, device="cuda").remainder(251).to(torch.int16)[None, :] + 0x3f00)
    tail = activations(5, k, 1).cuda()
    x[-5:] = tail
    q, s = moe.fp4_quantize(x)
    code, byte = plain_quantize(tail.cpu())
    r = torch.arange(m - 5, m)[:, None]
    got = s.view(torch.uint8)[(r // 128).cuda(), (torch.arange(k // 32)[None, :] // 4).cuda(), (r % 32).cuda(), (r % 128 // 32).cuda(), (torch.arange(k // 32)[None, :] % 4).cuda()]
    assert torch.equal(got.cpu().long(), byte) and torch.equal(codes(q[-5:], k), code)
    w = moe.fp4_quantize(activations(n, k, 2).cuda())
    y = moe.fp4_matmul(q, s, *w)
    assert close(y[-5:], plain_value(code, byte), value(*w), True)
    assert torch.equal(y[0], y[m - 6])                      # equal rows give equal results wherever they are
    back = moe.fp4_dequantize(q, s)
    assert torch.equal(back[-5:].cpu().double(), plain_value(code, byte))
    del back, y
    turned = moe.fp4_quantize(x[:, :64], "columns")         # rows 64 KB apart, 2^32 values in between
    code, byte = plain_quantize(x[-64:, :64].cpu(), "columns")
    assert torch.equal(codes(turned[0], m)[:, -64:], code)
    del x, q, s
    torch.cuda.empty_cache()


@pytest.mark.gpu
def test_one_answer_however_often_captured_or_on_another_stream():
    from paper_2411_02581_b200 import moe
    x, w = activations(7, 4096, 1).cuda(), activations(1024, 4096, 2).cuda()
    big, dense = activations(900, 1024, 3).cuda(), activations(1100, 1024, 4).cuda()

    def call(**kw):
        a, b = moe.fp4_quantize(x, **kw), moe.fp4_quantize(w, **kw)
        c, d = moe.fp4_quantize(big, **kw), moe.fp4_quantize(dense, **kw)
        return [moe.fp4_matmul(*a, *b, out_dtype=torch.float32, **kw), moe.fp4_matmul(*c, *d, **kw), moe.fp4_dequantize(*d, **kw),
                moe.fp4_matmul(*moe.fp4_quantize(dense, "columns", **kw), *moe.fp4_quantize(dense, "columns", **kw), **kw)]
    want = call()
    for _ in range(10):
        assert all(torch.equal(p, q) for p, q in zip(call(), want))
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
        assert all(torch.equal(p, q) for p, q in zip(out, want))
    for held in (side, torch.cuda.current_stream()):
        with torch.cuda.stream(held):
            torch.cuda._sleep(20_000_000)
        got = call(stream=side)
        junk = [torch.full((n,), 0x5a, dtype=torch.uint8, device="cuda") for n in (512 << i for i in range(15)) for _ in range(3)]
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, want))
        del junk


@pytest.mark.gpu
def test_python_refusals():
    from paper_2411_02581_b200 import moe
    x = torch.randn(8, 256, device="cuda")
    q, s = moe.fp4_quantize(x)
    w, t = moe.fp4_quantize(torch.randn(130, 256, device="cuda"))
    off = torch.tensor([0, 8], device="cuda")
    with pytest.raises(ValueError, match="layout: one of rows, columns"):
        moe.fp4_quantize(x, "tiles")
    with pytest.raises(ValueError, match="x: a CUDA matrix of float32 bfloat16"):
        moe.fp4_quantize(x.half())
    with pytest.raises(ValueError, match="offsets go with"):
        moe.fp4_quantize(x, "columns", offsets=off)
    with pytest.raises(ValueError, match="offsets"):
        moe.fp4_quantize(x, offsets=off.int())
    with pytest.raises(ValueError, match="offsets"):
        moe.fp4_quantize(x, offsets=off[:1])
    with pytest.raises(ValueError, match="q: a CUDA matrix of float4"):
        moe.fp4_dequantize(q.view(torch.uint8), s)
    with pytest.raises(ValueError, match="scale"):
        moe.fp4_dequantize(q, s.view(torch.uint8))
    with pytest.raises(ValueError, match="scale"):
        moe.fp4_dequantize(w, s)
    with pytest.raises(ValueError, match="out_dtype"):
        moe.fp4_dequantize(q, s, out_dtype=torch.float16)
    with pytest.raises(ValueError, match="a_scale"):
        moe.fp4_matmul(w, s, w, t)
    with pytest.raises(ValueError, match="b_scale"):
        moe.fp4_matmul(q, s, w, s)
    with pytest.raises(ValueError, match="a has 128 columns, b 256"):
        moe.fp4_matmul(*moe.fp4_quantize(x[:, :128]), w, t.narrow(1, 0, 1).contiguous())
    with pytest.raises(ValueError, match="b: contiguous matrices"):
        moe.fp4_matmul(q, s, w, t, offsets=off)
    with pytest.raises(ValueError, match="a_scale"):                 # quantised without the offsets
        y = torch.zeros(256, 256, device="cuda")
        moe.fp4_matmul(*moe.fp4_quantize(y), w[None].contiguous(), t[None], offsets=torch.tensor([0, 256], device="cuda"))
    with pytest.raises(ValueError, match="out_dtype"):
        moe.fp4_matmul(q, s, w, t, out_dtype=torch.float16)


def test_fp4_refusals():
    """Refused on the host, before any GPU work (pointers are never followed)."""
    build_mod.build()
    L = B.lib()

    def quantize(x=256, dtype=1, rows=4, cols=64, ld=64, layout=0, groups=0, off=None, q=256, ldq=32, s=256):
        return L.tuna_fp4_quantize(x, dtype, rows, cols, ld, layout, groups, off, q, ldq, s, None)
    assert quantize(dtype=2) == -1 and quantize(ld=63) == -1 and quantize(layout=2) == -1 and quantize(layout=-1) == -1
    assert quantize(ldq=16) == -1 and quantize(ldq=40) == -1 and quantize(layout=1, rows=65) == -1 and quantize(groups=2) == -1
    assert quantize(off=256) == -1 and quantize(groups=-1) == -1 and quantize(groups=2, off=256, layout=1) == -1 and quantize(groups=513, off=256) == -9
    assert quantize(x=None) == -1 and quantize(x=257) == -1 and quantize(q=264) == -1 and quantize(s=None) == -1 and quantize(s=264) == -1
    assert quantize(groups=1, off=260) == -1 and quantize(cols=1 << 25, ld=1 << 25, ldq=1 << 24) == -9 and quantize(rows=1 << 31) == -9
    assert quantize(rows=-1) == -1 and quantize(rows=0) == 0 and quantize(cols=0) == 0

    def back(q=256, ldq=32, s=256, rows=4, cols=64, groups=0, off=None, out=256, dt=1, ldo=64):
        return L.tuna_fp4_dequantize(q, ldq, s, rows, cols, groups, off, out, dt, ldo, None)
    assert back(ldq=31) == -1 and back(ldo=63) == -1 and back(dt=2) == -1 and back(groups=1) == -1 and back(s=264) == -1 and back(out=257) == -1
    assert back(q=None) == -1 and back(rows=0) == 0 and back(cols=0) == 0 and back(rows=-1) == -1 and back(groups=600, off=256) == -9

    def align(q=256, ldq=32, rows=4, count=32, out=256, ldo=32):
        return L.tuna_fp4_align(q, ldq, rows, count, out, ldo, None)
    assert align(ldq=31) == -1 and align(ldo=40) == -1 and align(ldo=16) == -1 and align(q=None) == -1 and align(out=264) == -1 and align(rows=-1) == -1
    assert align(rows=0) == 0 and align(count=0) == 0 and align(rows=1 << 32) == -9 and align(count=1 << 25, ldq=1 << 25, ldo=1 << 25) == -9

    def product(a=256, sa=256, m=4, lda=32, b=256, sb=256, n=8, ldb=32, k=64, groups=0, off=None, out=256, dt=1, ldo=8):
        return L.tuna_fp4_matmul(a, sa, m, lda, b, sb, n, ldb, k, groups, off, out, dt, ldo, None)
    assert product(lda=31) == -1 and product(lda=40) == -1 and product(ldb=24) == -1 and product(ldo=7) == -1 and product(k=63) == -1
    assert product(groups=2) == -1 and product(off=256) == -1 and product(dt=2) == -1 and product(a=None) == -1 and product(a=264) == -1
    assert product(b=264) == -1 and product(sa=264) == -1 and product(sb=264) == -1 and product(out=257) == -1 and product(groups=1, off=260) == -1
    assert product(groups=513, off=256) == -9 and product(k=1 << 25, lda=1 << 24, ldb=1 << 24) == -9 and product(m=0) == 0 and product(n=0, ldo=0) == 0 and product(m=-1) == -1
