"""Mixture-of-experts operators over torch tensors: router, 8-bit block-scaled products,
experts, few-token layer.

A thin layer over the C ABI in ``include/tuna.h``, like :mod:`binding`: arguments are
checked and marshalled, outputs and workspaces come from torch's allocator, every
computation runs in the CUDA library (there is no CPU fallback).  Work is enqueued on
``stream`` (default: torch's current one).  A tensor that was made on another stream is
the caller's to order, as with any torch operation.
"""
from __future__ import annotations

import ctypes
import functools
from typing import NamedTuple

import torch

from . import binding as B

SOFTMAX, SIGMOID = 0, 1
SCORING = {"softmax": SOFTMAX, "sigmoid": SIGMOID}
DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float8_e4m3fn: 2}
LAYOUTS = {"rows": 0, "columns": 1, "tiles": 2, "tiles_t": 3}
FLOATS = (torch.float32, torch.bfloat16)


class Routing(NamedTuple):
    """What :func:`route` returns; see ``tuna_moe_route`` for each."""
    ids: torch.Tensor      # int32 [tokens, k]
    weights: torch.Tensor  # float32 [tokens, k]
    counts: torch.Tensor   # int64 [ranks, experts]
    offsets: torch.Tensor  # int64 [ranks * experts + 1]
    rows: torch.Tensor     # int64 [tokens * k]
    pos: torch.Tensor      # int64 [tokens, k]


def _stream(stream, device):
    """The raw stream: torch's current one of the tensors' device, or the caller's."""
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(device.index)
    return B._stream(stream)


def _check(rc, what):
    if rc != 0:
        raise B.TunaError(rc, what, B.lib().tuna_ops_cuda_error() if rc == -7 else 0)


def _matrix(t, name, dtypes):
    """A CUDA matrix whose rows are contiguous; returns its row pitch."""
    if not isinstance(t, torch.Tensor) or t.dim() != 2 or t.dtype not in dtypes or not t.is_cuda:
        raise ValueError(f"{name}: a CUDA matrix of {', '.join(str(d) for d in dtypes)} is wanted")
    rows, cols = t.shape
    ld, step = t.stride()
    if cols > 1 and step != 1 or rows > 1 and ld < cols:
        raise ValueError(f"{name}: rows must be contiguous and must not overlap (strides {t.stride()})")
    return ld if rows > 1 else max(cols, 1)


def _dense(t, name, dtype, shape):
    if not isinstance(t, torch.Tensor) or t.dtype != dtype or t.shape != shape or not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{name}: a contiguous CUDA tensor of {dtype}, shape {tuple(shape)}, is wanted")
    return t


def _scoring(name):
    if name not in SCORING:
        raise ValueError(f"scoring: one of {', '.join(SCORING)}, got {name!r}")
    return SCORING[name]


@functools.lru_cache(maxsize=4096)
def _bytes(function, *sizes):
    """A workspace size, asked of the library once for each set of sizes."""
    n = ctypes.c_size_t()
    _check(getattr(B.lib(), function)(*sizes, ctypes.byref(n)), function)
    return n.value


def _order_workspace(tokens, experts, k, ranks, device):
    return torch.empty(max(_bytes("tuna_moe_order_workspace_bytes", tokens, experts, k, ranks), 256), dtype=torch.uint8, device=device)


def _order_outputs(tokens, experts, k, ranks, device):
    new = torch.empty
    return (new(ranks, experts, dtype=torch.int64, device=device), new(ranks * experts + 1, dtype=torch.int64, device=device),
            new(tokens * k, dtype=torch.int64, device=device), new(tokens, k, dtype=torch.int64, device=device))


def route(logits, k, *, scoring="softmax", renormalize=False, scale=1.0, ranks=1, stream=None) -> Routing:
    """The ``k`` best experts of every token, their weights and the rows' order (``tuna_moe_route``)."""
    ld = _matrix(logits, "logits", FLOATS)
    t, e = logits.shape
    if ranks < 1 or t % ranks:
        raise ValueError(f"{t} tokens do not divide over {ranks} ranks")
    device, empty, long = logits.device, torch.empty, torch.int64
    need = _bytes("tuna_moe_route_workspace_bytes", t, e, k, ranks)
    ws = empty(need, dtype=torch.uint8, device=device) if need else None
    ids = empty(t, k, dtype=torch.int32, device=device)
    weights = empty(t, k, dtype=torch.float32, device=device)
    counts = empty(ranks, e, dtype=long, device=device)
    offsets = empty(ranks * e + 1, dtype=long, device=device)
    rows = empty(t * k, dtype=long, device=device)
    pos = empty(t, k, dtype=long, device=device)
    rc = B.lib().tuna_moe_route(logits.data_ptr(), DTYPES[logits.dtype], t, e, ld, k, ranks, _scoring(scoring), renormalize, scale,
                                ids.data_ptr(), weights.data_ptr(), counts.data_ptr(), offsets.data_ptr(), rows.data_ptr(),
                                pos.data_ptr(), ws.data_ptr() if need else None, need, _stream(stream, device))
    if rc:
        _check(rc, "tuna_moe_route")
    return Routing(ids, weights, counts, offsets, rows, pos)


def order(ids, experts, *, ranks=1, stream=None):
    """(counts, offsets, rows, pos) of choices made elsewhere (``tuna_moe_order``)."""
    if ids.dim() != 2:
        raise ValueError("ids: [tokens, k] is wanted")
    t, k = ids.shape
    _dense(ids, "ids", torch.int32, (t, k))
    if ranks < 1 or t % ranks:
        raise ValueError(f"{t} tokens do not divide over {ranks} ranks")
    ws = _order_workspace(t, experts, k, ranks, ids.device)
    out = _order_outputs(t, experts, k, ranks, ids.device)
    _check(B.lib().tuna_moe_order(ids.data_ptr(), t, experts, k, ranks, *[o.data_ptr() for o in out], ws.data_ptr(), ws.numel(),
                                  _stream(stream, ids.device)), "tuna_moe_order")
    return out


def route_backward(logits, ids, dweights, *, scoring="softmax", renormalize=False, scale=1.0, stream=None):
    """Gradient of :func:`route`'s weights with respect to the logits (``tuna_moe_route_backward``)."""
    ld = _matrix(logits, "logits", FLOATS)
    t, e = logits.shape
    k = ids.shape[1]
    _dense(ids, "ids", torch.int32, (t, k))
    _dense(dweights, "dweights", torch.float32, (t, k))
    d = torch.empty(t, e, dtype=logits.dtype, device=logits.device)
    _check(B.lib().tuna_moe_route_backward(logits.data_ptr(), DTYPES[logits.dtype], t, e, ld, k, _scoring(scoring), int(renormalize),
                                           scale, ids.data_ptr(), dweights.data_ptr(), d.data_ptr(), e, _stream(stream, logits.device)),
           "tuna_moe_route_backward")
    return d


def combine(y, weights, pos, *, out_dtype=torch.bfloat16, stream=None):
    """out[t] = sum over s of weights[t, s] * y[pos[t, s]] (``tuna_moe_combine``)."""
    ld = _matrix(y, "y", FLOATS)
    t, k = weights.shape
    _dense(weights, "weights", torch.float32, (t, k))
    _dense(pos, "pos", torch.int64, (t, k))
    if out_dtype not in FLOATS:
        raise ValueError(f"out_dtype: one of {FLOATS}")
    out = torch.empty(t, y.shape[1], dtype=out_dtype, device=y.device)
    _check(B.lib().tuna_moe_combine(y.data_ptr(), DTYPES[y.dtype], y.shape[0], y.shape[1], ld, weights.data_ptr(), pos.data_ptr(), t, k,
                                    out.data_ptr(), DTYPES[out_dtype], y.shape[1], _stream(stream, y.device)), "tuna_moe_combine")
    return out


def combine_backward(dout, y, weights, pos, *, stream=None):
    """(dy, dweights) of :func:`combine`; rows of y that no slot names get a zero gradient."""
    ldg, ldy = _matrix(dout, "dout", FLOATS), _matrix(y, "y", FLOATS)
    t, k = weights.shape
    _dense(weights, "weights", torch.float32, (t, k))
    _dense(pos, "pos", torch.int64, (t, k))
    if tuple(dout.shape) != (t, y.shape[1]):
        raise ValueError(f"dout: shape {tuple(dout.shape)}, wanted {(t, y.shape[1])}")
    dy = torch.zeros(y.shape, dtype=y.dtype, device=y.device)
    dw = torch.zeros_like(weights)
    _check(B.lib().tuna_moe_combine_backward(dout.data_ptr(), DTYPES[dout.dtype], ldg, y.data_ptr(), DTYPES[y.dtype], y.shape[0],
                                             y.shape[1], ldy, weights.data_ptr(), pos.data_ptr(), t, k, dy.data_ptr(), y.shape[1],
                                             dw.data_ptr(), _stream(stream, y.device)), "tuna_moe_combine_backward")
    return dy, dw


def _blocks(n):
    return -(-n // 128)


def fp8_quantize(x, layout="rows", *, stream=None):
    """(q, scale): ``x`` in 8 bits with a scale for each block (``tuna_fp8_quantize``).

    ``q`` of the layouts "columns" and "tiles_t" is that of the transposed matrix."""
    ld = _matrix(x, "x", FLOATS)
    which = LAYOUTS.get(layout)
    if which is None:
        raise ValueError(f"layout: one of {', '.join(LAYOUTS)}, got {layout!r}")
    rows, cols = x.shape
    out_rows, out_cols = (cols, rows) if which & 1 else (rows, cols)
    pitch = (out_cols + 15) & ~15
    device = x.device
    q = torch.empty(out_rows, pitch, dtype=torch.float8_e4m3fn, device=device)
    blocks = (out_cols + 127) >> 7
    if which < 2:
        scale = torch.empty(blocks, out_rows, dtype=torch.float32, device=device)
    else:
        scale = torch.empty((out_rows + 127) >> 7, blocks, dtype=torch.float32, device=device)
    rc = B.lib().tuna_fp8_quantize(x.data_ptr(), DTYPES[x.dtype], rows, cols, ld, which, q.data_ptr(), pitch or 16, scale.data_ptr(),
                                   _stream(stream, device))
    if rc:
        _check(rc, "tuna_fp8_quantize")
    return q if pitch == out_cols else q[:, :out_cols], scale


def _fp8_matrix(q, name):
    """(operand, pitch, rows, columns) of an e4m3 matrix; copies one whose rows do not start on 16-byte boundaries."""
    ld = _matrix(q, name, (torch.float8_e4m3fn,))
    rows, cols = q.shape
    if rows <= 1:
        ld = (cols + 15) & ~15   # the pitch of a single row is free
    if ld & 15 or q.data_ptr() & 15:
        p = torch.zeros(rows, (cols + 15) & ~15, dtype=torch.uint8, device=q.device)
        p[:, :cols] = q.view(torch.uint8)
        q, ld = p, p.shape[1]
    return q, ld or 16, rows, cols


def fp8_matmul(a, a_scale, b, b_scale, *, offsets=None, b_blocks="tiles", out_dtype=torch.bfloat16, stream=None):
    """a b^T with a scale for each block of 128 (``tuna_fp8_matmul``).

    ``a`` [m, k] with "rows" scales.  ``b`` [n, k] with "tiles" scales, or "rows" scales
    (``b_blocks="rows"``); or [groups, n, k] with ``offsets`` (int64 [groups + 1]): rows
    offsets[g] .. offsets[g + 1] of ``a`` meet ``b[g]``."""
    a, lda, m, k = _fp8_matrix(a, "a")
    if out_dtype not in FLOATS:
        raise ValueError(f"out_dtype: one of {FLOATS}")
    blocks = (k + 127) >> 7
    groups, at = 1, None
    if offsets is not None:
        if b.dim() != 3 or not b.is_contiguous() or b_blocks != "tiles":
            raise ValueError("b: contiguous matrices [groups, n, k] with tile scales go with offsets")
        groups, n, kb = b.shape
        at = _dense(offsets, "offsets", torch.int64, (groups + 1,)).data_ptr()
        b, ldb, _, _ = _fp8_matrix(b.view(groups * n, kb), "b")
        _dense(b_scale, "b_scale", torch.float32, (groups, (n + 127) >> 7, blocks))
    else:
        b, ldb, n, kb = _fp8_matrix(b, "b")
        if b_blocks == "tiles":
            _dense(b_scale, "b_scale", torch.float32, ((n + 127) >> 7, blocks))
        elif b_blocks == "rows":
            _dense(b_scale, "b_scale", torch.float32, (blocks, n))
        else:
            raise ValueError(f"b_blocks: tiles or rows, got {b_blocks!r}")
    if kb != k:
        raise ValueError(f"a has {k} columns, b {kb}")
    _dense(a_scale, "a_scale", torch.float32, (blocks, m))
    device = a.device
    out = torch.empty(m, n, dtype=out_dtype, device=device)
    rc = B.lib().tuna_fp8_matmul(a.data_ptr(), a_scale.data_ptr(), m, lda, b.data_ptr(), b_scale.data_ptr(), LAYOUTS[b_blocks], n, ldb, k,
                                 groups, at, out.data_ptr(), DTYPES[out_dtype], n or 1, _stream(stream, device))
    if rc:
        _check(rc, "tuna_fp8_matmul")
    return out


def _experts_weights(w13, s13, w2, s2, hidden):
    """Checked shapes of 8-bit expert weights: (experts, inter)."""
    if w13.dim() != 4 or w13.shape[1] != 2 or w13.shape[3] != hidden:
        raise ValueError(f"w13: [experts, 2, inter, {hidden}] is wanted, got {tuple(w13.shape)}")
    e, _, i, d = w13.shape
    _dense(w13, "w13", torch.float8_e4m3fn, (e, 2, i, d))
    _dense(s13, "s13", torch.float32, (e, 2, _blocks(i), _blocks(d)))
    _dense(w2, "w2", torch.float8_e4m3fn, (e, d, i))
    _dense(s2, "s2", torch.float32, (e, _blocks(d), _blocks(i)))
    return e, i


def _space(need, workspace, device):
    if workspace is None:
        return torch.empty(max(need, 256), dtype=torch.uint8, device=device)
    return workspace


def expert_rows(x, offsets, w13, s13, w2, s2, *, workspace=None, stream=None):
    """Rows in expert order through their experts (``tuna_moe_expert_rows``); a row of the result that no expert has is undefined."""
    ldx = _matrix(x, "x", (torch.bfloat16,))
    rows, d = x.shape
    e, i = _experts_weights(w13, s13, w2, s2, d)
    _dense(offsets, "offsets", torch.int64, (e + 1,))
    ws = _space(_bytes("tuna_moe_expert_rows_workspace_bytes", rows, d, i), workspace, x.device)
    y = torch.empty(rows, d, dtype=torch.bfloat16, device=x.device)
    _check(B.lib().tuna_moe_expert_rows(x.data_ptr(), ldx, rows, e, offsets.data_ptr(), d, i, w13.data_ptr(), s13.data_ptr(), w2.data_ptr(),
                                        s2.data_ptr(), y.data_ptr(), d, ws.data_ptr(), ws.numel(), _stream(stream, x.device)), "tuna_moe_expert_rows")
    return y


def experts(x, ids, weights, w13, s13, w2, s2, *, workspace=None, stream=None):
    """The experts of many tokens in 8 bits (``tuna_moe_experts``): ids and weights as :func:`route` makes them."""
    ldx = _matrix(x, "x", (torch.bfloat16,))
    t, d = x.shape
    e, i = _experts_weights(w13, s13, w2, s2, d)
    k = ids.shape[-1]
    _dense(ids, "ids", torch.int32, (t, k))
    _dense(weights, "weights", torch.float32, (t, k))
    ws = _space(_bytes("tuna_moe_experts_workspace_bytes", t, e, k, d, i), workspace, x.device)
    out = torch.empty(t, d, dtype=torch.bfloat16, device=x.device)
    _check(B.lib().tuna_moe_experts(x.data_ptr(), ldx, t, ids.data_ptr(), weights.data_ptr(), k, e, d, i, w13.data_ptr(), s13.data_ptr(),
                                    w2.data_ptr(), s2.data_ptr(), out.data_ptr(), d, ws.data_ptr(), ws.numel(), _stream(stream, x.device)),
           "tuna_moe_experts")
    return out


@functools.lru_cache(maxsize=4096)
def _few_bytes(*sizes):
    n, z = ctypes.c_size_t(), ctypes.c_size_t()
    _check(B.lib().tuna_moe_few_workspace_bytes(*sizes, ctypes.byref(n), ctypes.byref(z)), "tuna_moe_few_workspace_bytes")
    return max(n.value, 256), z.value


def few_workspace(tokens, experts, k, hidden, inter, device="cuda"):
    """A workspace of :func:`few`, ready for use by one stream."""
    need, zeroed = _few_bytes(tokens, experts, k, hidden, inter)
    ws = torch.empty(need, dtype=torch.uint8, device=device)
    ws[:zeroed].zero_()
    return ws


_few_spaces = {}  # (device, stream) -> workspaces that few() keeps: the last one serves, older ones may be held by graphs


def few(x, router, k, w13, w2, *, s13=None, s2=None, scoring="softmax", renormalize=False, scale=1.0, ids=None, weights=None,
        workspace=None, stream=None):
    """A whole layer for at most 64 tokens in one launch (``tuna_moe_few``).

    ``w13`` [experts, 2, inter, hidden] and ``w2`` [experts, hidden, inter] in bf16, or in
    e4m3 with ``s13`` and ``s2``.  ``ids`` / ``weights``: optional outputs [tokens, k].
    ``workspace``: from :func:`few_workspace`; without one the module keeps one a stream."""
    ldx = _matrix(x, "x", (torch.bfloat16,))
    t, d = x.shape
    if ldx % 8 or x.data_ptr() % 16:
        x, ldx = x.clone(memory_format=torch.contiguous_format), d
    e = router.shape[0]
    _dense(router, "router", torch.bfloat16, (e, d))
    if w13.dim() != 4:
        raise ValueError(f"w13: [experts, 2, inter, hidden] is wanted, got {tuple(w13.shape)}")
    i = w13.shape[2]
    if w13.dtype == torch.float8_e4m3fn:
        if s13 is None or s2 is None:
            raise ValueError("8-bit weights need s13 and s2")
        if _experts_weights(w13, s13, w2, s2, d) != (e, i):
            raise ValueError(f"w13: {e} experts are wanted, got {w13.shape[0]}")
    else:
        _dense(w13, "w13", torch.bfloat16, (e, 2, i, d))
        _dense(w2, "w2", torch.bfloat16, (e, d, i))
    if ids is not None:
        _dense(ids, "ids", torch.int32, (t, k))
    if weights is not None:
        _dense(weights, "weights", torch.float32, (t, k))
    s = _stream(stream, x.device)
    if workspace is None:
        kept = _few_spaces.setdefault((x.device.index, s), [])
        if not kept or kept[-1].numel() < _few_bytes(t, e, k, d, i)[0]:
            if torch.cuda.is_current_stream_capturing():
                raise RuntimeError("few: pass a workspace (few_workspace) when the first call of this size is captured")
            with torch.cuda.stream(torch.cuda.ExternalStream(s, device=x.device)):
                kept.append(few_workspace(t, e, k, d, i, x.device))
        workspace = kept[-1]
    out = torch.empty(t, d, dtype=torch.bfloat16, device=x.device)
    _check(B.lib().tuna_moe_few(x.data_ptr(), ldx, t, router.data_ptr(), e, k, _scoring(scoring), int(renormalize), scale, d, i,
                                DTYPES[w13.dtype], w13.data_ptr(), None if s13 is None else s13.data_ptr(), w2.data_ptr(),
                                None if s2 is None else s2.data_ptr(), out.data_ptr(), d, None if ids is None else ids.data_ptr(),
                                None if weights is None else weights.data_ptr(), workspace.data_ptr(), workspace.numel(), s),
           "tuna_moe_few")
    return out


def device_status() -> int:
    """0, or 1 if a kernel of these operators gave up a bounded wait (synchronises the device)."""
    n = ctypes.c_int()
    _check(B.lib().tuna_ops_device_status(ctypes.byref(n)), "tuna_ops_device_status")
    return n.value
