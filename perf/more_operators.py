"""Benchmark cases of the operators that stand beside the router and the 8-bit products: the balance loss of a router,
microscaled 4-bit values (quantisation, product), and experts with 4-bit weights; in plain torch and through the library.

Sizes follow the token-dispatch workload of this repository (hidden 4096, 64 experts, top-2, 8192 tokens a rank)
and generic ones around it: smaller hidden sizes, more slots, odd token counts, lengths that no block divides.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # the loss of a small batch, as an evaluation step looks at it
        dict(name="balance small", kind="balance", tokens=512, experts=8, k=2, dtype="bf16", scoring="softmax", segments=1, padded=0, backward=False),
        # a training step: 8 sequences of 8192 tokens, a loss and a z loss for each, with the gradient
        dict(name="balance train", kind="balance", tokens=65536, experts=64, k=2, dtype="f32", scoring="softmax", segments=8, padded=0, backward=True),
        # packed sequences of different lengths, some of them empty, padding behind the last one, many experts
        dict(name="balance ragged", kind="balance", tokens=20011, experts=160, k=6, dtype="bf16", scoring="sigmoid", segments=37, padded=100, backward=True),
        # a weight matrix put into 4 bits and read back
        dict(name="quantize weight", kind="quantize", rows=4096, cols=4096, dtype="bf16", layout="rows"),
        # gradients of a ragged batch along the other axis, from 32 bits
        dict(name="quantize ragged columns", kind="quantize", rows=1777, cols=2896, dtype="f32", layout="columns"),
        # one token through a dense layer
        dict(name="linear4 one token", kind="linear", m=1, n=4096, k=4096, backward=False),
        # a ragged batch: no size is a multiple of a block, and the last value of a row has no neighbour
        dict(name="linear4 ragged", kind="linear", m=777, n=2001, k=2895, backward=False),
        # prefill of one rank's tokens
        dict(name="linear4 prefill", kind="linear", m=8192, n=4096, k=4096, backward=False),
        # a training step of a dense layer: output, input gradient, weight gradient, everything quantised on the way
        dict(name="linear4 train", kind="linear", m=4096, n=2048, k=4096, backward=True),
        # one token through its two experts
        dict(name="experts4 one token", kind="experts", tokens=1, experts=64, k=2, hidden=4096, inter=2048),
        # a short prompt of odd length: a handful of rows an expert
        dict(name="experts4 short prompt", kind="experts", tokens=501, experts=64, k=2, hidden=2048, inter=1408),
        # one rank's tokens of the dispatch workload
        dict(name="experts4 prefill", kind="experts", tokens=8192, experts=64, k=2, hidden=4096, inter=2048),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    kind = rng.choice(["balance", "quantize", "linear", "experts"])
    if kind == "balance":
        experts = rng.choice([8, 16, 60, 64, 128, 160, 256])
        tokens = _log(rng, 64, 65536 * 64 // max(experts, 64))
        return dict(kind=kind, tokens=tokens, experts=experts, k=rng.choice([1, 2, 4, 6, 8]), dtype=rng.choice(["bf16", "f32"]),
                    scoring=rng.choice(["softmax", "sigmoid"]), segments=rng.choice([1, _log(rng, 1, 64)]), padded=rng.choice([0, 0, tokens // 9]),
                    backward=rng.random() < 0.6)
    if kind == "quantize":
        return dict(kind=kind, rows=_log(rng, 1, 8192), cols=_log(rng, 32, 8192), dtype=rng.choice(["bf16", "f32"]), layout=rng.choice(["rows", "columns"]))
    if kind == "linear":
        backward = rng.random() < 0.3
        return dict(kind=kind, m=_log(rng, 128 if backward else 1, 4096 if backward else 8192), n=16 * rng.randint(16, 128 if backward else 256) - rng.choice([0, 0, 5]),
                    k=16 * rng.choice([rng.randint(32, 180), rng.choice([64, 128, 256])]) - rng.choice([0, 0, 7]), backward=backward)
    hidden = rng.choice([1024, 2048, 4096])
    return dict(kind=kind, tokens=_log(rng, 1, 8192), experts=rng.choice([8, 16, 60, 64]), k=rng.choice([1, 2, 4] if hidden < 4096 else [1, 2]),
                hidden=hidden, inter=32 * rng.randint(12, 64))


# ---- inputs ------------------------------------------------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _activations(g, rows, cols, dtype=torch.bfloat16):
    """Normal values with a few strong channels, as hidden states have them."""
    x = torch.randn(rows, cols, generator=g, device="cuda")
    strong = 1.0 + 15.0 * (torch.rand(cols, generator=g, device="cuda") < 0.01)
    return (x * strong).to(dtype)


def _held_weights(g, count, rows, cols):
    """`count` matrices of normal weights in 4 bits, as a checkpoint holds them: (q [count, rows, cols / 2], scale [count, tiles, blocks, 32, 4, 4])."""
    q = torch.empty(count, rows, (cols + 1) // 2, dtype=torch.uint8, device="cuda")
    s = torch.empty(count, -(-rows // 128), -(-cols // 128), 32, 4, 4, dtype=torch.uint8, device="cuda")
    for i in range(count):
        code, byte = _codes(torch.randn(rows, cols, generator=g, device="cuda") * (cols ** -0.5))
        q[i], s[i] = _packed(code), _tiled(byte)
    return q.view(torch.float4_e2m1fn_x2), s.view(torch.float8_e8m0fnu)


def prepare(case, seed):
    g = _generator(seed)
    c = dict(case)
    if c["kind"] == "balance":
        t, e, segments = c["tokens"], c["experts"], c["segments"]
        z = 1.5 * torch.randn(t, e, generator=g, device="cuda") + 0.5 * torch.randn(e, generator=g, device="cuda")
        z = z.to(DTYPES[c["dtype"]])
        z[t - c["padded"]:] = -math.inf                       # padding: nothing of the row is left
        c["logits"] = z
        ids = torch.sort(z.float(), dim=1, descending=True, stable=True).indices[:, :c["k"]].to(torch.int32)
        ids[t - c["padded"]:] = -1
        c["ids"] = ids
        cuts = torch.rand(segments - 1, generator=g, device="cuda").sort().values * t
        if segments > 2:
            cuts[1] = cuts[0]                                 # a sequence without tokens
        if segments == 8:
            cuts = torch.arange(1, 8, device="cuda") * (t / 8)
        c["offsets"] = torch.cat([cuts.new_zeros(1), cuts, cuts.new_full((1,), t)]).long() if segments > 1 else None
        c["dloss"] = 0.01 * (0.5 + torch.rand(segments, generator=g, device="cuda"))
        c["dz"] = 0.001 * (0.5 + torch.rand(segments, generator=g, device="cuda"))
    elif c["kind"] == "quantize":
        c["x"] = _activations(g, c["rows"], c["cols"], DTYPES[c["dtype"]])
    elif c["kind"] == "linear":
        c["x"] = _activations(g, c["m"], c["k"])
        if c["backward"]:
            c["w"] = (torch.randn(c["n"], c["k"], generator=g, device="cuda") * c["k"] ** -0.5).to(torch.bfloat16)
            c["dy"] = torch.randn(c["m"], c["n"], generator=g, device="cuda").to(torch.bfloat16)
        else:
            q, s = _held_weights(g, 1, c["n"], c["k"])
            c["w"], c["ws"] = q[0], s[0]
    else:
        e, d, i = c["experts"], c["hidden"], c["inter"]
        c["x"] = _activations(g, c["tokens"], d)
        q, s = _held_weights(g, 2 * e, i, d)
        c["w13"], c["s13"] = q.view(e, 2, i, d // 2), s.view(e, 2, *s.shape[1:])
        c["w2"], c["s2"] = _held_weights(g, e, d, i)
        z = torch.randn(c["tokens"], e, generator=g, device="cuda") + 0.5 * torch.randn(e, generator=g, device="cuda")
        z, ids = torch.topk(z, c["k"], dim=1)                 # distinct experts for every token, some liked more than others
        c["ids"], c["weights"] = ids.to(torch.int32), torch.softmax(z, 1)
        c["most"] = int(torch.bincount(ids.reshape(-1), minlength=e).max())  # rows of the fullest expert
    return c


# ---- plain forms -------------------------------------------------------------------------------------------------

def _blocks_of_32(x):
    x = x.float()
    return torch.nn.functional.pad(x, (0, -x.shape[-1] % 32)).unflatten(-1, (-1, 32))


def _power(byte):
    """2^(byte - 127) as the 32-bit value with those bits."""
    return torch.where(byte > 0, byte << 23, torch.full_like(byte, 1 << 22)).view(torch.float32)


def _rounded(x):
    """The values of blocks of 32 along a matrix's rows over their scales, rounded to the 4-bit ones, and the scales' bytes."""
    b = _blocks_of_32(x)
    byte = ((b.abs().amax(-1).view(torch.int32) >> 23) - 2).clamp(min=0)  # the exponent of the largest magnitude is 2, that of 6
    v = b * _power(254 - byte).unsqueeze(-1)
    a = v.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    return torch.clamp(torch.round(v / step) * step, -6.0, 6.0), byte


def _stand(x):
    """What a matrix is when its rows are held in 4 bits."""
    v, byte = _rounded(x)
    return (v * _power(byte).unsqueeze(-1)).flatten(-2)[..., :x.shape[-1]]


def _codes(x):
    """(codes 0 .. 15 [rows, whole blocks of 32], bytes [rows, blocks]) of a matrix."""
    v, byte = _rounded(x)
    a = v.abs()
    code = torch.where(a <= 2, a * 2, torch.where(a <= 4, a + 2, torch.full_like(a, 7))).to(torch.uint8)
    return (code + 8 * (v < 0).to(torch.uint8)).flatten(-2)[:, :x.shape[1]], byte


def _packed(code):
    code = torch.nn.functional.pad(code, (0, code.shape[1] % 2))
    return code[:, 0::2] + 16 * code[:, 1::2]


def _tiled(byte):
    """[rows, blocks] -> [tiles of 128 rows, runs of 4 blocks, 32, 4, 4]: row 32 j + i of a tile at [i, j]."""
    r, b = byte.shape
    p = torch.nn.functional.pad(byte, (0, -b % 4, 0, -r % 128))
    return p.view(p.shape[0] // 128, 4, 32, p.shape[1] // 4, 4).permute(0, 3, 2, 1, 4).to(torch.uint8)


def _held(q, s):
    """The values of matrices [..., rows, cols / 2] held in 4 bits."""
    q, s = q.view(torch.uint8), s.view(torch.uint8)
    code = torch.stack([q & 15, q >> 4], -1).flatten(-2)
    a = (code & 7).float()
    a = torch.where(a < 4, a / 2, torch.where(a < 6, a - 2, 2 * a - 8))
    byte = s.movedim((-5, -2, -3, -4, -1), (-5, -4, -3, -2, -1)).flatten(-2).flatten(-4, -2)[..., :q.shape[-2], :].int()  # [rows, blocks]
    return torch.where(code > 7, -a, a) * _power(byte).repeat_interleave(32, -1)[..., :code.shape[-1]]


def _segment_of(c):
    """The segment of each token."""
    t = torch.arange(c["tokens"], device="cuda")
    return torch.zeros_like(t) if c["offsets"] is None else (t[:, None] >= c["offsets"][None, 1:-1]).sum(1)


def _balance(c):
    z = c["logits"].float()
    e, k, segments = c["experts"], c["k"], c["segments"]
    live = (z > -math.inf).any(1)
    zl = torch.where(live[:, None], z, torch.zeros_like(z))
    top = zl.amax(1, keepdim=True)
    x = torch.exp(zl - top)
    total = x.sum(1, keepdim=True)
    soft, lse = x / total, (top + torch.log(total))[:, 0]
    p, s = soft, None
    if c["scoring"] == "sigmoid":
        s = 1 / (1 + torch.exp(-zl))
        p = s / s.sum(1, keepdim=True)
    at, keep = _segment_of(c), live[:, None]
    n = torch.zeros(segments, dtype=torch.int64, device="cuda").index_add_(0, at, live.long())
    mass = torch.zeros(segments, e, dtype=torch.float64, device="cuda").index_add_(0, at, (p * keep).double())
    squares = torch.zeros(segments, dtype=torch.float64, device="cuda").index_add_(0, at, (lse * lse * live).double())
    ids = c["ids"].long()
    there = (ids >= 0).long()
    counts = torch.zeros(segments * e, dtype=torch.int64, device="cuda").scatter_add_(
        0, (at[:, None] * e + ids.clamp(min=0)).reshape(-1), there.reshape(-1)).view(segments, e)
    per = torch.where(n > 0, e / (k * (n * n).double().clamp(min=1)), 0.0)
    out = dict(loss=(per * (counts.double() * mass).sum(1)).float(), z=(squares / n.clamp(min=1)).float(), counts=counts, mass=mass.float(), tokens=n)
    if c["backward"]:
        g = ((c["dloss"].double() * per)[:, None] * counts.double()).float()[at]
        d = p * (g - (p * g).sum(1, keepdim=True))
        if s is not None:
            d = d * (1 - s)
        d = d + (c["dz"] * 2 / n.clamp(min=1))[at][:, None] * lse[:, None] * soft
        out["dlogits"] = torch.where(keep, d, torch.zeros_like(d)).to(c["logits"].dtype)
    return out


def _quantize(c):
    x = c["x"] if c["layout"] == "rows" else c["x"].t()
    return _stand(x).to(c["x"].dtype)


def _linear(c):
    x = _stand(c["x"])
    if not c["backward"]:
        return (x @ _held(c["w"], c["ws"])[:, :c["k"]].t()).to(torch.bfloat16)
    y = x @ _stand(c["w"]).t()
    dx = _stand(c["dy"]) @ _stand(c["w"].t()).t()
    dw = _stand(c["dy"].t()) @ _stand(c["x"].t()).t()
    return dict(y=y.to(torch.bfloat16), dx=dx.to(torch.bfloat16), dw=dw.to(torch.bfloat16))


def _experts(c):
    e, k, most = c["experts"], c["k"], c["most"]
    ids = c["ids"].reshape(-1).long()
    at = torch.sort(ids, stable=True).indices
    count = torch.zeros(e, dtype=torch.int64, device="cuda").scatter_add_(0, ids, torch.ones_like(ids))
    first = count.cumsum(0) - count
    place = ids[at] * most + torch.arange(at.numel(), device="cuda") - first[ids[at]]
    x = _stand(c["x"])
    rows = x.new_zeros(e * most, x.shape[1])
    rows[place] = x[at // k]
    rows = rows.view(e, most, -1)
    gate, up = rows @ _held(c["w13"][:, 0], c["s13"][:, 0]).transpose(1, 2), rows @ _held(c["w13"][:, 1], c["s13"][:, 1]).transpose(1, 2)
    h = _stand(gate / (1 + torch.exp(-gate)) * up)
    y = (h @ _held(c["w2"], c["s2"]).transpose(1, 2)).view(e * most, -1)[place]
    out = torch.empty_like(y)
    out[at] = y * c["weights"].reshape(-1)[at][:, None]
    return out.view(c["tokens"], k, -1).sum(1).to(torch.bfloat16)


# ---- through the library -----------------------------------------------------------------------------------------

def _balance_own(c):
    from paper_2411_02581_b200 import moe
    b = moe.balance(c["logits"], c["ids"], scoring=c["scoring"], offsets=c["offsets"])
    out = dict(loss=b.loss, z=b.z, counts=b.counts, mass=b.mass, tokens=b.tokens)
    if c["backward"]:
        out["dlogits"] = moe.balance_backward(c["logits"], b.counts, b.tokens, c["k"], c["dloss"], c["dz"], scoring=c["scoring"], offsets=c["offsets"])
    return out


def _quantize_own(c):
    from paper_2411_02581_b200 import moe
    q, s = moe.fp4_quantize(c["x"], c["layout"])
    return moe.fp4_dequantize(q, s, out_dtype=c["x"].dtype)[:, :c["x"].shape[1 if c["layout"] == "rows" else 0]]


def _linear_own(c):
    from paper_2411_02581_b200 import moe
    x, xs = moe.fp4_quantize(c["x"])
    if not c["backward"]:
        return moe.fp4_matmul(x, xs, c["w"], c["ws"])
    w, ws = moe.fp4_quantize(c["w"])
    wt, wts = moe.fp4_quantize(c["w"], "columns")
    dy, dys = moe.fp4_quantize(c["dy"])
    dyt, dyts = moe.fp4_quantize(c["dy"], "columns")
    xt, xts = moe.fp4_quantize(c["x"], "columns")
    return dict(y=moe.fp4_matmul(x, xs, w, ws), dx=moe.fp4_matmul(dy, dys, wt, wts), dw=moe.fp4_matmul(dyt, dyts, xt, xts))


def _experts_own(c):
    from paper_2411_02581_b200 import moe
    return moe.fp4_experts(c["x"], c["ids"], c["weights"], c["w13"], c["s13"], c["w2"], c["s2"])


PLAIN = {"balance": _balance, "quantize": _quantize, "linear": _linear, "experts": _experts}
OWN = {"balance": _balance_own, "quantize": _quantize_own, "linear": _linear_own, "experts": _experts_own}


def run(state):
    return (OWN if own else PLAIN)[state["kind"]](state)


# ---- work and 64-bit values --------------------------------------------------------------------------------------

def _bytes4(rows, cols):
    """A matrix in 4 bits with its scales."""
    return rows * (-(-cols // 2) + -(-cols // 32))


def work(case):
    c = case
    if c["kind"] == "balance":
        t, e, k, s, size = c["tokens"], c["experts"], c["k"], c["segments"], 2 if c["dtype"] == "bf16" else 4
        moved = t * e * size + t * k * 4 + s * e * 12 + s * 16
        return {"bytes": moved + (t * e * size if c["backward"] else 0), "flops": t * e * (12 if c["backward"] else 5)}
    if c["kind"] == "quantize":
        n, size = c["rows"] * c["cols"], 2 if c["dtype"] == "bf16" else 4
        return {"bytes": 2 * n * size, "flops": 4 * n}
    if c["kind"] == "linear":
        m, n, k = c["m"], c["n"], c["k"]
        if c["backward"]:
            return {"bytes": 2 * (2 * m * k + 2 * n * k + 2 * m * n), "flops": 6.0 * m * n * k}
        return {"bytes": 2 * m * k + _bytes4(n, k) + 2 * m * n, "flops": 2.0 * m * n * k}
    t, e, k, d, i = c["tokens"], c["experts"], c["k"], c["hidden"], c["inter"]
    met = min(e, max(k, e * (1 - (1 - 1 / e) ** (t * k))))  # experts that so many evenly spread choices are expected to reach
    return {"bytes": met * (2 * _bytes4(i, d) + _bytes4(d, i)) + 4 * t * d + 8 * t * k, "flops": 6.0 * t * k * d * i}


def _exact_stand(x):
    """What remains of a matrix whose rows are held in 4 bits with a power of two for each 32 values, from the definition."""
    k = x.shape[1]
    b = torch.nn.functional.pad(x.double(), (0, -k % 32)).view(x.shape[0], -1, 32)
    top = b.abs().amax(2, keepdim=True)
    e = torch.frexp(top).exponent - 1                        # floor of the logarithm
    scale = torch.ldexp(torch.ones_like(top), (e - 2).clamp(min=-127))
    scale = torch.where(top > 0, scale, torch.ones_like(scale))
    v = b / scale
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device=x.device)
    low = (torch.bucketize(v.abs(), grid, right=True) - 1).clamp(max=6)
    a, z = grid[low], grid[low + 1]
    middle = (a + z) / 2
    up = (v.abs() > middle) | ((v.abs() == middle) & (low % 2 == 1))
    return (torch.where(up, z, a) * v.sign() * scale).flatten(1)[:, :k]


def _exact_held(q, s):
    """A matrix that a checkpoint holds in 4 bits, in 64."""
    q, s = q.view(torch.uint8).long(), s.view(torch.uint8)
    table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device=q.device)
    table = torch.cat([table, -table])
    r = torch.arange(q.shape[0], device=q.device)[:, None]
    c = torch.arange(q.shape[1] * 2, device=q.device)[None, :]
    code = torch.where(c % 2 == 0, q.repeat_interleave(2, 1) % 16, q.repeat_interleave(2, 1) // 16)
    byte = s[r // 128, c // 128, r % 32, r % 128 // 32, c % 128 // 32]
    return table[code] * torch.exp2(byte.double() - 127)


def exact(case, seed):
    c = prepare(case, seed)
    if c["kind"] == "balance":
        z, k, e = c["logits"].double(), c["k"], c["experts"]
        bounds = [0, c["tokens"]] if c["offsets"] is None else c["offsets"].tolist()
        loss, zs, mass, d = [], [], [], torch.zeros_like(z)
        for g in range(c["segments"]):
            at = torch.arange(bounds[g], bounds[g + 1], device="cuda")
            at = at[torch.isfinite(z[at]).any(1)]
            n = at.numel()
            if n == 0:
                loss.append(z.new_zeros(())), zs.append(z.new_zeros(())), mass.append(z.new_zeros(e))
                continue
            rows = z[at].clone().requires_grad_(True)
            if c["scoring"] == "sigmoid":
                p = torch.sigmoid(rows)
                p = p / p.sum(1, keepdim=True)
            else:
                p = torch.softmax(rows, 1)
            f = torch.bincount(c["ids"][at].reshape(-1).long(), minlength=e).double()
            loss.append(e * (f / (k * n) * p.mean(0)).sum())
            zs.append(torch.logsumexp(rows, 1).square().mean())
            mass.append(p.sum(0).detach())
            if c["backward"]:
                d[at], = torch.autograd.grad(c["dloss"][g].double() * loss[-1] + c["dz"][g].double() * zs[-1], rows)
        out = dict(loss=torch.stack(loss).detach(), z=torch.stack(zs).detach(), counts=None, mass=torch.stack(mass), tokens=None)
        if c["backward"]:
            out["dlogits"] = d
        return out
    if c["kind"] == "quantize":
        return _exact_stand(c["x"] if c["layout"] == "rows" else c["x"].t())
    if c["kind"] == "linear":
        if not c["backward"]:
            return _exact_stand(c["x"]) @ _exact_held(c["w"], c["ws"])[:, :c["k"]].t()
        x, w, dy = c["x"], c["w"], c["dy"]
        return dict(y=_exact_stand(x) @ _exact_stand(w).t(), dx=_exact_stand(dy) @ _exact_stand(w.t()).t(),
                    dw=_exact_stand(dy.t()) @ _exact_stand(x.t()).t())
    x, ids = _exact_stand(c["x"]), c["ids"].long()
    out = torch.zeros_like(x)
    for j in range(c["experts"]):
        t, slot = (ids == j).nonzero(as_tuple=True)
        if t.numel():
            g, u = _exact_held(c["w13"][j, 0], c["s13"][j, 0]), _exact_held(c["w13"][j, 1], c["s13"][j, 1])
            h = _exact_stand(torch.nn.functional.silu(x[t] @ g.t()) * (x[t] @ u.t()))
            out.index_add_(0, t, (h @ _exact_held(c["w2"][j], c["s2"][j]).t()) * c["weights"][t, slot].double()[:, None])
    return out
