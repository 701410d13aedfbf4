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
from typing import NamedTuple

import torch

from . import binding as B

SOFTMAX, SIGMOID = 0, 1
SCORING = {"softmax": SOFTMAX, "sigmoid": SIGMOID}
DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float8_e4m3fn: 2}
FLOATS = (torch.float32, torch.bfloat16)


class Routing(NamedTuple):
    """What :func:`route` returns; see ``tuna_moe_route`` for each."""
    ids: torch.Tensor      # int32 [tokens, k]
    weights: torch.Tensor  # float32 [tokens, k]
    counts: torch.Tensor   # int64 [ranks, experts]
    offsets: torch.Tensor  # int64 [ranks * experts + 1]
    rows: torch.Tensor     # int64 [tokens * k]
    pos: torch.Tensor      # int64 [tokens, k]


def _check(rc, what):
    if rc != 0:
        raise B.TunaError(rc, what, B.lib().tuna_ops_cuda_error() if rc == -7 else 0)


def _matrix(t, name, dtypes, rows=None, cols=None):
    """A CUDA matrix whose rows are contiguous; returns its row pitch."""
    if not isinstance(t, torch.Tensor) or t.dim() != 2 or t.dtype not in dtypes or not t.is_cuda:
        raise ValueError(f"{name}: a CUDA matrix of {', '.join(str(d) for d in dtypes)} is wanted")
    if rows is not None and t.shape[0] != rows or cols is not None and t.shape[1] != cols:
        raise ValueError(f"{name}: shape {tuple(t.shape)}, wanted ({rows if rows is not None else 'any'}, "
                         f"{cols if cols is not None else 'any'})")
    if t.shape[1] > 1 and t.stride(1) != 1 or t.shape[0] > 1 and t.stride(0) < t.shape[1]:
        raise ValueError(f"{name}: rows must be contiguous and must not overlap (strides {t.stride()})")
    return t.stride(0) if t.shape[0] > 1 else max(t.shape[1], 1)


def _dense(t, name, dtype, shape):
    if not isinstance(t, torch.Tensor) or t.dtype != dtype or tuple(t.shape) != tuple(shape) or not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{name}: a contiguous CUDA tensor of {dtype}, shape {tuple(shape)}, is wanted")
    return t


def _scoring(name):
    if name not in SCORING:
        raise ValueError(f"scoring: one of {', '.join(SCORING)}, got {name!r}")
    return SCORING[name]


def _order_workspace(tokens, experts, k, ranks, device):
    n = ctypes.c_size_t()
    _check(B.lib().tuna_moe_order_workspace_bytes(tokens, experts, k, ranks, ctypes.byref(n)), "tuna_moe_order_workspace_bytes")
    return torch.empty(max(n.value, 256), dtype=torch.uint8, device=device)


def _order_outputs(tokens, experts, k, ranks, device):
    new = lambda *shape: torch.empty(*shape, dtype=torch.int64, device=device)  # noqa: E731
    return new(ranks, experts), new(ranks * experts + 1), new(tokens * k), new(tokens, k)


def route(logits, k, *, scoring="softmax", renormalize=False, scale=1.0, ranks=1, stream=None) -> Routing:
    """The ``k`` best experts of every token, their weights and the rows' order (``tuna_moe_route``)."""
    ld = _matrix(logits, "logits", FLOATS)
    t, e = logits.shape
    if ranks < 1 or t % ranks:
        raise ValueError(f"{t} tokens do not divide over {ranks} ranks")
    ws = _order_workspace(t, e, k, ranks, logits.device)
    ids = torch.empty(t, k, dtype=torch.int32, device=logits.device)
    weights = torch.empty(t, k, dtype=torch.float32, device=logits.device)
    counts, offsets, rows, pos = _order_outputs(t, e, k, ranks, logits.device)
    _check(B.lib().tuna_moe_route(logits.data_ptr(), DTYPES[logits.dtype], t, e, ld, k, ranks, _scoring(scoring), int(renormalize), scale,
                                  ids.data_ptr(), weights.data_ptr(), counts.data_ptr(), offsets.data_ptr(), rows.data_ptr(),
                                  pos.data_ptr(), ws.data_ptr(), ws.numel(), B._stream(stream)), "tuna_moe_route")
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
                                  B._stream(stream)), "tuna_moe_order")
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
                                           scale, ids.data_ptr(), dweights.data_ptr(), d.data_ptr(), e, B._stream(stream)),
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
                                    out.data_ptr(), DTYPES[out_dtype], y.shape[1], B._stream(stream)), "tuna_moe_combine")
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
                                             dw.data_ptr(), B._stream(stream)), "tuna_moe_combine_backward")
    return dy, dw


def device_status() -> int:
    """0, or 1 if a kernel of these operators gave up a bounded wait (synchronises the device)."""
    n = ctypes.c_int()
    _check(B.lib().tuna_ops_device_status(ctypes.byref(n)), "tuna_ops_device_status")
    return n.value
