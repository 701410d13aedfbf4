"""The operators on a stream that is not torch's current one.

Each call runs on a side stream that is held back, while the current stream allocates and
fills memory of the sizes that the calls use, or on a free side stream while the current one
is held back.  What the call needs of its own (workspaces, copies, zeros) has to be ordered
with its kernels, so the results are those of the same call without a stream, bit for bit.
"""
import pytest
import torch

from test_fp8 import activations
from test_moe_layer import bf16_weights, fp8_weights

pytestmark = pytest.mark.gpu
HOLD = 20_000_000  # cycles: some 10 ms


def fp8(x, layout="rows"):
    from paper_2411_02581_b200 import moe
    return moe.fp8_quantize(x, layout)


def calls():
    """name -> a call that takes a stream; inputs are ready."""
    from paper_2411_02581_b200 import moe
    g = torch.Generator().manual_seed(1)
    e, k, d, i, t = 16, 3, 272, 144, 700
    x = activations(t, d, 2).cuda()
    z = torch.randn(t, e, generator=g).cuda()
    w13, s13 = fp8_weights(2 * e, i, d, 1)
    w2, s2 = fp8_weights(e, d, i, 2)
    w13, s13 = w13.view(e, 2, i, d), s13.view(e, 2, *s13.shape[1:])
    r = moe.route(z, k)
    dw = torch.randn(t, k, generator=g).cuda()
    y, dout = activations(t * k, d, 3).cuda(), activations(t, d, 4).cuda()
    q, s = fp8(x)
    v, u = fp8(activations(96, d, 5).cuda(), "tiles")
    odd = torch.zeros(t, d + 9, dtype=torch.uint8, device="cuda")
    odd[:, 3:3 + d] = q.view(torch.uint8)
    odd = odd[:, 3:3 + d].view(torch.float8_e4m3fn)               # off 16 bytes: the call pads a copy
    router, b13, b2 = bf16_weights(1, e, d, 6)[0], bf16_weights(2 * e, i, d, 7).view(e, 2, i, d), bf16_weights(e, d, i, 8)
    wide = torch.zeros(33, d + 3, dtype=torch.bfloat16, device="cuda")
    wide[:, 3:] = x[:33]                                          # off 16 bytes: the call clones it
    sent, offsets = x[r.rows[:t]], r.offsets.clamp(max=t)
    return {
        "route": lambda **kw: moe.route(z, k, **kw),
        "route_backward": lambda **kw: moe.route_backward(z, r.ids, dw, **kw),
        "order": lambda **kw: moe.order(r.ids, e, **kw),
        "combine": lambda **kw: moe.combine(y, r.weights, r.pos, **kw),
        "combine_backward": lambda **kw: moe.combine_backward(dout, y, r.weights, r.pos, **kw),
        "fp8_quantize": lambda **kw: [p.view(torch.uint8) for p in moe.fp8_quantize(x, "columns", **kw)],
        "fp8_matmul, padded operand": lambda **kw: moe.fp8_matmul(odd, s, v, u, **kw),
        "expert_rows": lambda **kw: moe.expert_rows(sent, offsets, w13, s13, w2, s2, **kw),
        "experts": lambda **kw: moe.experts(x, r.ids, r.weights, w13, s13, w2, s2, **kw),
        "few, cloned x": lambda **kw: moe.few(wide[:, 3:], router, k, b13, b2, **kw),
    }


def parts(out):
    return [out] if isinstance(out, torch.Tensor) else list(out)


def churn():
    """Takes and fills what the allocator of the current stream has to give, in sizes from 512 bytes to 8 MB."""
    return [torch.full((n,), 0x5a, dtype=torch.uint8, device="cuda") for n in (512 << i for i in range(15)) for _ in range(4)]


@pytest.mark.parametrize("raw", [False, True])
@pytest.mark.parametrize("held", ["side", "current"])
def test_given_stream_orders_all_that_a_call_does(held, raw):
    for name, call in calls().items():
        want = parts(call())
        side = torch.cuda.Stream()
        torch.cuda.synchronize()
        with torch.cuda.stream(side if held == "side" else torch.cuda.current_stream()):
            torch.cuda._sleep(HOLD)
        got = parts(call(stream=side.cuda_stream if raw else side))
        junk = churn()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b), name
        del junk


def test_outputs_may_be_freed_on_the_stream_that_was_current():
    """The caller waits for the side stream, reads an output on the current one and lets go of it: the side stream
    must not be given its memory before that read is done."""
    from paper_2411_02581_b200 import moe
    y, w = activations(4096, 1024, 1).cuda(), torch.ones(4096, 1, device="cuda")
    pos = torch.arange(4096, device="cuda")[:, None]
    zeros = torch.zeros_like(y)
    side, here = torch.cuda.Stream(), torch.cuda.current_stream()
    torch.cuda.synchronize()
    for call in (lambda v: moe.combine(v, w, pos, stream=side), lambda v: moe.fp8_quantize(v, stream=side)[0].view(torch.uint8)):
        out = call(y)
        here.wait_stream(side)
        torch.cuda._sleep(10 * HOLD)
        kept = out.clone()
        want_at = out.data_ptr()
        del out
        again = [call(zeros) for _ in range(3)]
        read = here.query()             # (memory that has been read may be given out again)
        assert read or all(a.data_ptr() != want_at for a in again)
        want = call(y)
        torch.cuda.synchronize()
        assert torch.equal(kept, want)


def test_stream_arguments_that_are_none():
    from paper_2411_02581_b200 import moe
    z = torch.randn(300, 64, device="cuda")
    with pytest.raises(AttributeError):
        moe.route(z, 2, stream="side")
    with pytest.raises(OverflowError):
        moe.route(z, 2, stream=1 << 80)
    want = moe.route(z, 2)
    for stream in (0, 1, torch.cuda.default_stream()):   # 1: the CUDA runtime's name of the default stream
        for a, b in zip(want, moe.route(z, 2, stream=stream)):
            assert torch.equal(a, b)
        assert torch.equal(moe.combine(z, want.weights, want.pos.clamp(max=299), stream=stream), moe.combine(z, want.weights, want.pos.clamp(max=299)))


@pytest.mark.parametrize("how", ["current", "given"])
def test_captured_few_has_a_workspace_of_its_own(how):
    """A graph may be replayed on any stream, so it must not count on the workspace that eager calls on the stream
    of its capture share: its replays leave that one alone, whether the capturing stream is the current or a given one."""
    from paper_2411_02581_b200 import moe
    e, k, d, i = 16, 2, 256, 128
    router, w13, w2 = bf16_weights(1, e, d, 6)[0], bf16_weights(2 * e, i, d, 7).view(e, 2, i, d), bf16_weights(e, d, i, 8)
    xs = [activations(t, d, t).cuda() for t in (5, 40)]
    want = [moe.few(x, router, k, w13, w2) for x in xs]
    side, other = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    moe.few(xs[1], router, k, w13, w2, stream=side)               # an eager call on the stream that will capture
    kept = moe._few_spaces[torch.cuda.current_device(), side.cuda_stream]
    torch.cuda.synchronize()
    graphs, outs = [torch.cuda.CUDAGraph() for _ in xs], []
    for graph, x in zip(graphs, xs):
        with torch.cuda.graph(graph, stream=side):
            if how == "current":
                outs.append(moe.few(x, router, k, w13, w2))
            else:
                with torch.cuda.stream(other):
                    outs.append(moe.few(x, router, k, w13, w2, stream=side))
    was = kept.clone()
    for out in outs:
        out.zero_()
    torch.cuda.synchronize()
    for _ in range(3):
        for graph, on in zip(graphs, (side, other)):
            with torch.cuda.stream(on):
                graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(kept, was)
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
    again = moe.few(xs[0], router, k, w13, w2, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(again, want[0])
    assert moe.device_status() == 0


def test_few_keeps_one_workspace_a_stream():
    from paper_2411_02581_b200 import moe
    e, k, d, i = 16, 2, 256, 128
    router, w13, w2 = bf16_weights(1, e, d, 6)[0], bf16_weights(2 * e, i, d, 7).view(e, 2, i, d), bf16_weights(e, d, i, 8)
    want = moe.few(activations(1, d, 1).cuda(), router, k, w13, w2)
    sizes = []
    for t in (64, 3, 64, 1):
        x = activations(t, d, t).cuda()
        got = moe.few(x, router, k, w13, w2)
        sizes.append(moe._few_spaces[torch.cuda.current_device(), torch.cuda.current_stream().cuda_stream])
    assert all(s is sizes[0] for s in sizes) and torch.equal(got, want)
