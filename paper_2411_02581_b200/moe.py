"""Mixture-of-experts operators over torch tensors: router and its balance loss, 8-bit block-scaled and
4-bit microscaled products, experts, few-token layer.

A thin layer over the C ABI in ``include/tuna.h``, like :mod:`binding`: arguments are
checked and marshalled, outputs and workspaces come from torch's allocator, every
computation runs in the CUDA library (there is no CPU fallback).  The calls of a decode
step are marshalled in C++ (``csrc/tuna_torch.cpp``), where ctypes and the interpreter
would take longer than their kernels.  Work is enqueued on ``stream`` (default: torch's
current one), which is torch's current stream until the call returns: outputs, workspaces
and copies are its own.  An input that was made on another stream is the caller's to
order, as with any torch operation, and so is an output before another stream reads it.

Nothing here is recorded by autograd: outputs carry no gradient, whatever the inputs require.
Gradients are calls of their own (:func:`route_backward`, :func:`balance_backward`,
:func:`combine_backward`, and :func:`fp8_matmul` or :func:`fp4_matmul` on operands quantised along the
other axis), which a ``torch.autograd.Function`` of the caller's may make; :func:`experts`,
:func:`expert_rows`, their 4-bit forms and :func:`few` have none.
"""
from __future__ import annotations

import contextlib
import ctypes
import functools
import importlib.util
import os
from typing import NamedTuple

import torch

from . import binding as B
from . import build as _build

SOFTMAX, SIGMOID = 0, 1
SCORING = {"softmax": SOFTMAX, "sigmoid": SIGMOID}
DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float8_e4m3fn: 2}
# two values a byte; the scale of 32 values (None: a torch without them, which has the other operators)
FP4, POWER = getattr(torch, "float4_e2m1fn_x2", None), getattr(torch, "float8_e8m0fnu", None)
FP4_LAYOUTS = {"rows": 0, "columns": 1}
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


class Balance(NamedTuple):
    """What :func:`balance` returns; see ``tuna_moe_balance`` for each."""
    loss: torch.Tensor     # float32 [segments]
    z: torch.Tensor        # float32 [segments]
    counts: torch.Tensor   # int64 [segments, experts]
    mass: torch.Tensor     # float32 [segments, experts]
    tokens: torch.Tensor   # int64 [segments]: live tokens


def _same(*tensors):
    return tensors if len(tensors) > 1 else tensors[0]


def _on(stream, device):
    """Makes ``device`` the current one and ``stream`` torch's current stream for a whole call, so that
    what is allocated and filled on the way belongs to it.  Yields the raw stream and what outputs leave
    through: the caller may use and free them on the stream that was current before."""
    if stream is None and device.index == torch.cuda.current_device():
        return contextlib.nullcontext((torch._C._cuda_getCurrentRawStream(device.index), _same))
    return _on_another(stream, device)


@contextlib.contextmanager
def _on_another(stream, device):
    with torch.cuda.device(device.index):
        before = torch._C._cuda_getCurrentRawStream(device.index)
        at = before if stream is None else B._stream(stream)
        at = 0 if at == 1 else at  # cudaStreamLegacy: torch's name of the same stream is 0
        if at == before:
            yield at, _same
            return
        was = torch.cuda.current_stream(device)

        def out(*tensors):
            for t in tensors:
                t.record_stream(was)
            return _same(*tensors)
        with torch.cuda.stream(stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(at, device=device)):
            yield at, out


def _check(rc, what):
    if rc != 0:
        raise B.TunaError(rc, what, B.lib().tuna_ops_cuda_error() if rc == -7 else 0)


_marshal = None


def _fast():
    """The C++ marshalling, bound to the loaded library; raises if it has not been built."""
    global _marshal
    if _marshal is None:
        if not os.path.exists(_build.TORCH_PATH):
            raise RuntimeError(f"{_build.TORCH_PATH} is missing: build it with `python -m paper_2411_02581_b200.build`")
        spec = importlib.util.spec_from_file_location("tuna_torch", _build.TORCH_PATH)
        module = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(module)
        module.bind(B.lib()._handle, _check)
        _marshal = module
    return _marshal


def _beside(t, name, device):
    if t.device != device:
        raise ValueError(f"{name}: on {t.device}, its fellows are on {device}")


def _matrix(t, name, dtypes, device=None):
    """A CUDA matrix whose rows are contiguous, on ``device``; returns its row pitch."""
    if not isinstance(t, torch.Tensor) or t.dim() != 2 or t.dtype not in dtypes or not t.is_cuda:
        raise ValueError(f"{name}: a CUDA matrix of {', '.join(str(d) for d in dtypes)} is wanted")
    rows, cols = t.shape
    ld, step = t.stride()
    if cols > 1 and step != 1 or rows > 1 and ld < cols:
        raise ValueError(f"{name}: rows must be contiguous and must not overlap (strides {t.stride()})")
    _beside(t, name, device or t.device)
    return ld if rows > 1 else max(cols, 1)


def _dense(t, name, dtype, shape, device=None):
    if not isinstance(t, torch.Tensor) or t.dtype != dtype or t.shape != shape or not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{name}: a contiguous CUDA tensor of {dtype}, shape {tuple(shape)}, is wanted")
    _beside(t, name, device or t.device)
    return t


def _scoring(name):
    which = SCORING.get(name)
    if which is None:
        raise ValueError(f"scoring: one of {', '.join(SCORING)}, got {name!r}")
    return which


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
    return Routing(*(_marshal or _fast()).route(logits, k, _scoring(scoring), renormalize, scale, ranks, stream))


def order(ids, experts, *, ranks=1, stream=None):
    """(counts, offsets, rows, pos) of choices made elsewhere (``tuna_moe_order``)."""
    if ids.dim() != 2:
        raise ValueError("ids: [tokens, k] is wanted")
    t, k = ids.shape
    _dense(ids, "ids", torch.int32, (t, k))
    if ranks < 1 or t % ranks:
        raise ValueError(f"{t} tokens do not divide over {ranks} ranks")
    with _on(stream, ids.device) as (at, out):
        ws = _order_workspace(t, experts, k, ranks, ids.device)
        made = _order_outputs(t, experts, k, ranks, ids.device)
        _check(B.lib().tuna_moe_order(ids.data_ptr(), t, experts, k, ranks, *[o.data_ptr() for o in made], ws.data_ptr(), ws.numel(), at),
               "tuna_moe_order")
        return out(*made)


def route_backward(logits, ids, dweights, *, scoring="softmax", renormalize=False, scale=1.0, stream=None):
    """Gradient of :func:`route`'s weights with respect to the logits (``tuna_moe_route_backward``)."""
    return (_marshal or _fast()).route_backward(logits, ids, dweights, _scoring(scoring), renormalize, scale, stream)


def balance(logits, ids, *, scoring="softmax", offsets=None, stream=None) -> Balance:
    """The balance loss of every segment of the tokens, the mean square of the logits' log-sum-exp, and what they are
    made of (``tuna_moe_balance``).  ``ids`` as :func:`route` makes them (-1 for a row without live logits: other ids
    of such a row are counted); ``offsets`` (int64 [segments + 1]): the segments'
    bounds, None for one segment."""
    return Balance(*(_marshal or _fast()).balance(logits, ids, _scoring(scoring), offsets, stream))


def balance_backward(logits, counts, tokens, k, dloss, dz=None, *, scoring="softmax", offsets=None, stream=None):
    """Gradient of sum(dloss * loss + dz * z) of :func:`balance` with respect to the logits (``tuna_moe_balance_backward``);
    ``k``: slots a token.  A row takes part if it has a logit that is not masked."""
    return (_marshal or _fast()).balance_backward(logits, counts, tokens, k, dloss, dz, _scoring(scoring), offsets, stream)


def combine(y, weights, pos, *, out_dtype=torch.bfloat16, stream=None):
    """out[t] = sum over s of weights[t, s] * y[pos[t, s]] (``tuna_moe_combine``)."""
    ld = _matrix(y, "y", FLOATS)
    t, k = weights.shape
    _dense(weights, "weights", torch.float32, (t, k), y.device)
    _dense(pos, "pos", torch.int64, (t, k), y.device)
    if out_dtype not in FLOATS:
        raise ValueError(f"out_dtype: one of {FLOATS}")
    with _on(stream, y.device) as (at, out):
        o = torch.empty(t, y.shape[1], dtype=out_dtype, device=y.device)
        _check(B.lib().tuna_moe_combine(y.data_ptr(), DTYPES[y.dtype], y.shape[0], y.shape[1], ld, weights.data_ptr(), pos.data_ptr(), t, k,
                                        o.data_ptr(), DTYPES[out_dtype], y.shape[1], at), "tuna_moe_combine")
        return out(o)


def combine_backward(dout, y, weights, pos, *, stream=None):
    """(dy, dweights) of :func:`combine`; rows of y that no slot names get a zero gradient."""
    ldg, ldy = _matrix(dout, "dout", FLOATS), _matrix(y, "y", FLOATS, dout.device)
    t, k = weights.shape
    _dense(weights, "weights", torch.float32, (t, k), y.device)
    _dense(pos, "pos", torch.int64, (t, k), y.device)
    if tuple(dout.shape) != (t, y.shape[1]):
        raise ValueError(f"dout: shape {tuple(dout.shape)}, wanted {(t, y.shape[1])}")
    with _on(stream, y.device) as (at, out):
        dy = torch.zeros(y.shape, dtype=y.dtype, device=y.device)
        dw = torch.zeros_like(weights)
        _check(B.lib().tuna_moe_combine_backward(dout.data_ptr(), DTYPES[dout.dtype], ldg, y.data_ptr(), DTYPES[y.dtype], y.shape[0],
                                                 y.shape[1], ldy, weights.data_ptr(), pos.data_ptr(), t, k, dy.data_ptr(), y.shape[1],
                                                 dw.data_ptr(), at), "tuna_moe_combine_backward")
        return out(dy, dw)


def _blocks(n):
    return -(-n // 128)


def fp8_quantize(x, layout="rows", *, stream=None):
    """(q, scale): ``x`` in 8 bits with a scale for each block (``tuna_fp8_quantize``).

    ``q`` of the layouts "columns" and "tiles_t" is that of the transposed matrix."""
    which = LAYOUTS.get(layout)
    if which is None:
        raise ValueError(f"layout: one of {', '.join(LAYOUTS)}, got {layout!r}")
    return (_marshal or _fast()).fp8_quantize(x, which, stream)


def fp8_matmul(a, a_scale, b, b_scale, *, offsets=None, b_blocks="tiles", out_dtype=torch.bfloat16, stream=None):
    """a b^T with a scale for each block of 128 (``tuna_fp8_matmul``).

    ``a`` [m, k] with "rows" scales.  ``b`` [n, k] with "tiles" scales, or "rows" scales
    (``b_blocks="rows"``); or [groups, n, k] with ``offsets`` (int64 [groups + 1]): rows
    offsets[g] .. offsets[g + 1] of ``a`` meet ``b[g]``."""
    if b_blocks != "tiles" and b_blocks != "rows":
        raise ValueError(f"b_blocks: tiles or rows, got {b_blocks!r}")
    if out_dtype not in FLOATS:
        raise ValueError(f"out_dtype: one of {FLOATS}")
    return (_marshal or _fast()).fp8_matmul(a, a_scale, b, b_scale, offsets, LAYOUTS[b_blocks], DTYPES[out_dtype], stream)


def fp4_quantize(x, layout="rows", *, offsets=None, stream=None):
    """(q, scale): ``x`` in 4 bits with a power of two for every 32 values along the row (``tuna_fp4_quantize``).

    ``q`` (float4_e2m1fn_x2: two values an element, the first in its low half) is [rows, (cols + 1) // 2], of the layout "columns"
    that of the transposed matrix.  ``scale`` (float8_e8m0fnu) is [row tiles, runs of 128 columns, 32, 4, 4]: that of row r and
    block j of a run is at [r // 128, run, r % 32, r % 128 // 32, j].  With ``offsets`` (int64 [groups + 1]) the row tiles
    are of rows of one group each, as :func:`fp4_matmul` with these offsets takes them."""
    which = FP4_LAYOUTS.get(layout)
    if which is None:
        raise ValueError(f"layout: one of {', '.join(FP4_LAYOUTS)}, got {layout!r}")
    return (_marshal or _fast()).fp4_quantize(x, which, offsets, stream)


def fp4_dequantize(q, scale, *, offsets=None, out_dtype=torch.bfloat16, stream=None):
    """The values that ``q`` stands for, [rows, 2 * q.shape[1]] (``tuna_fp4_dequantize``); a row outside every group is undefined."""
    if out_dtype not in FLOATS:
        raise ValueError(f"out_dtype: one of {FLOATS}")
    return (_marshal or _fast()).fp4_dequantize(q, scale, offsets, DTYPES[out_dtype], stream)


def fp4_matmul(a, a_scale, b, b_scale, *, offsets=None, out_dtype=torch.bfloat16, stream=None):
    """a b^T of operands that :func:`fp4_quantize` made along the contracted axis (``tuna_fp4_matmul``).

    ``b`` [n, k / 2], or [groups, n, k / 2] with ``offsets`` (int64 [groups + 1]): rows offsets[g] .. offsets[g + 1] of
    ``a``, which was quantised with these offsets, meet ``b[g]``; a row of the result that is outside every group is undefined.
    Operands lie as :func:`fp4_quantize` returns them, each row on a 16-byte boundary; others (a contiguous copy of rows
    whose bytes are no multiple of 16) are laid so in every call."""
    if out_dtype not in FLOATS:
        raise ValueError(f"out_dtype: one of {FLOATS}")
    return (_marshal or _fast()).fp4_matmul(a, a_scale, b, b_scale, offsets, DTYPES[out_dtype], stream)


def fp4_expert_rows(x, offsets, w13, s13, w2, s2, *, workspace=None, stream=None):
    """:func:`expert_rows` with weights, x and h in 4 bits (``tuna_fp4_expert_rows``).

    ``w13`` [experts, 2, inter, hidden / 2] and ``w2`` [experts, hidden, inter / 2] with ``s13`` and ``s2`` of every matrix
    as :func:`fp4_quantize` makes them; hidden and inter are multiples of 32."""
    return (_marshal or _fast()).fp4_expert_rows(x, offsets, w13, s13, w2, s2, workspace, stream)


def fp4_experts(x, ids, weights, w13, s13, w2, s2, *, workspace=None, stream=None):
    """:func:`experts` with weights, x and h in 4 bits (``tuna_fp4_experts``); weights as in :func:`fp4_expert_rows`."""
    return (_marshal or _fast()).fp4_experts(x, ids, weights, w13, s13, w2, s2, workspace, stream)


def _experts_weights(w13, s13, w2, s2, hidden, device):
    """Checked shapes of 8-bit expert weights: (experts, inter)."""
    if w13.dim() != 4 or w13.shape[1] != 2 or w13.shape[3] != hidden:
        raise ValueError(f"w13: [experts, 2, inter, {hidden}] is wanted, got {tuple(w13.shape)}")
    e, _, i, d = w13.shape
    _dense(w13, "w13", torch.float8_e4m3fn, (e, 2, i, d), device)
    _dense(s13, "s13", torch.float32, (e, 2, _blocks(i), _blocks(d)), device)
    _dense(w2, "w2", torch.float8_e4m3fn, (e, d, i), device)
    _dense(s2, "s2", torch.float32, (e, _blocks(d), _blocks(i)), device)
    return e, i


def _own_space(workspace, device):
    """Checks a workspace that the caller brought."""
    if workspace is None:
        return
    if not isinstance(workspace, torch.Tensor) or not workspace.is_cuda or not workspace.is_contiguous():
        raise ValueError("workspace: a contiguous CUDA tensor is wanted")
    _beside(workspace, "workspace", device)


def _space(need, workspace, device):
    return torch.empty(max(need, 256), dtype=torch.uint8, device=device) if workspace is None else workspace


def expert_rows(x, offsets, w13, s13, w2, s2, *, workspace=None, stream=None):
    """Rows in expert order through their experts (``tuna_moe_expert_rows``); a row of the result that no expert has is undefined."""
    ldx = _matrix(x, "x", (torch.bfloat16,))
    rows, d = x.shape
    e, i = _experts_weights(w13, s13, w2, s2, d, x.device)
    _dense(offsets, "offsets", torch.int64, (e + 1,), x.device)
    _own_space(workspace, x.device)
    with _on(stream, x.device) as (at, out):
        ws = _space(_bytes("tuna_moe_expert_rows_workspace_bytes", rows, d, i), workspace, x.device)
        y = torch.empty(rows, d, dtype=torch.bfloat16, device=x.device)
        _check(B.lib().tuna_moe_expert_rows(x.data_ptr(), ldx, rows, e, offsets.data_ptr(), d, i, w13.data_ptr(), s13.data_ptr(), w2.data_ptr(),
                                            s2.data_ptr(), y.data_ptr(), d, ws.data_ptr(), ws.nbytes, at), "tuna_moe_expert_rows")
        return out(y)


def experts(x, ids, weights, w13, s13, w2, s2, *, workspace=None, stream=None):
    """The experts of many tokens in 8 bits (``tuna_moe_experts``): ids and weights as :func:`route` makes them."""
    ldx = _matrix(x, "x", (torch.bfloat16,))
    t, d = x.shape
    e, i = _experts_weights(w13, s13, w2, s2, d, x.device)
    k = ids.shape[-1]
    _dense(ids, "ids", torch.int32, (t, k), x.device)
    _dense(weights, "weights", torch.float32, (t, k), x.device)
    _own_space(workspace, x.device)
    with _on(stream, x.device) as (at, out):
        ws = _space(_bytes("tuna_moe_experts_workspace_bytes", t, e, k, d, i), workspace, x.device)
        o = torch.empty(t, d, dtype=torch.bfloat16, device=x.device)
        _check(B.lib().tuna_moe_experts(x.data_ptr(), ldx, t, ids.data_ptr(), weights.data_ptr(), k, e, d, i, w13.data_ptr(), s13.data_ptr(),
                                        w2.data_ptr(), s2.data_ptr(), o.data_ptr(), d, ws.data_ptr(), ws.nbytes, at), "tuna_moe_experts")
        return out(o)


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


_few_spaces = {}  # (device, stream) -> the workspace that eager calls of few() share there, one after the other


def _few_space(x, router, k, w13, at):
    """The workspace of a call on the stream ``at``, which is torch's current one.  A captured call gets one
    of its own out of the graph's memory, zeroed at each replay: a graph may be replayed on any stream, beside
    other graphs and eager calls."""
    t, d = x.shape
    sizes = t, router.shape[0], k, d, w13.shape[2]
    if torch.cuda.is_current_stream_capturing():
        return few_workspace(*sizes, x.device)
    place = x.get_device(), at
    kept = _few_spaces.get(place)
    if kept is None or kept.numel() < _few_bytes(*sizes)[0]:
        kept = _few_spaces[place] = few_workspace(*sizes, x.device)
    return kept


def few(x, router, k, w13, w2, *, s13=None, s2=None, scoring="softmax", renormalize=False, scale=1.0, ids=None, weights=None,
        workspace=None, stream=None):
    """A whole layer for at most 64 tokens in one launch (``tuna_moe_few``).

    ``w13`` [experts, 2, inter, hidden] and ``w2`` [experts, hidden, inter] in bf16, or in
    e4m3 with ``s13`` and ``s2``.  ``ids`` / ``weights``: optional outputs [tokens, k].
    ``workspace``: from :func:`few_workspace`, of one call at a time.  Without one, the calls on a stream
    share one that the module keeps, as large as the largest of them needed, and each call that
    ``torch.cuda.graph`` captures has its own; who captures by other means passes one."""
    if workspace is None:
        if not x.is_cuda:
            raise ValueError("x: a CUDA matrix of torch.bfloat16 is wanted")
        if stream is None and x.get_device() == torch.cuda.current_device():  # (a decode step's call: no context to enter)
            workspace = _few_space(x, router, k, w13, torch._C._cuda_getCurrentRawStream(x.get_device()))
        else:
            with _on(stream, x.device) as (at, _):
                workspace = _few_space(x, router, k, w13, at)
    return (_marshal or _fast()).few(x, router, k, w13, w2, s13, s2, _scoring(scoring), renormalize, scale, ids, weights, workspace, stream)


def device_status() -> int:
    """0, or 1 if a kernel of these operators gave up a bounded wait since the last such call: what it made is
    incomplete, what comes later is not affected (synchronises the device)."""
    n = ctypes.c_int()
    _check(B.lib().tuna_ops_device_status(ctypes.byref(n)), "tuna_ops_device_status")
    return n.value
