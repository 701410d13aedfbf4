"""What the C++ marshalling of the operator calls refuses on a GPU, before anything is launched."""
import pytest
import torch

from paper_2411_02581_b200 import binding as B

pytestmark = pytest.mark.gpu


def test_shapes_types_and_strides():
    from paper_2411_02581_b200 import moe
    z = torch.randn(8, 16, device="cuda")
    with pytest.raises(ValueError, match="logits: rows must be contiguous"):
        moe.route(z.t(), 2)
    with pytest.raises(ValueError, match="logits: a CUDA matrix of float32 bfloat16"):
        moe.route(z.half(), 2)
    with pytest.raises(ValueError, match="8 tokens do not divide over 3 ranks"):
        moe.route(z, 2, ranks=3)
    with pytest.raises(B.TunaError, match="TUNA_ERR_INVALID_ARG"):
        moe.route(z, 17)                                   # more slots than experts
    with pytest.raises(B.TunaError, match="TUNA_ERR_RANGE"):
        moe.route(torch.zeros(2, 600, device="cuda"), 2)
    r = moe.route(z, 2)
    with pytest.raises(ValueError, match="dweights"):
        moe.route_backward(z, r.ids, r.weights.double())
    with pytest.raises(ValueError, match="ids"):
        moe.route_backward(z, r.ids.long(), r.weights)
    q, s = moe.fp8_quantize(torch.randn(8, 256, device="cuda"))
    w, t = moe.fp8_quantize(torch.randn(130, 256, device="cuda"), "tiles")
    with pytest.raises(ValueError, match="a has 128 columns, b 256"):
        moe.fp8_matmul(q[:, :128], s, w, t)
    with pytest.raises(ValueError, match="a_scale"):
        moe.fp8_matmul(q, s.t(), w, t)
    with pytest.raises(ValueError, match="b_scale"):
        moe.fp8_matmul(q, s, w, t[:1])
    with pytest.raises(ValueError, match="offsets"):
        moe.fp8_matmul(q, s, w, t, offsets=torch.zeros(2, dtype=torch.int64, device="cuda"))
    with pytest.raises(ValueError, match="out_dtype"):
        moe.fp8_matmul(q, s, w, t, out_dtype=torch.float16)
    x = torch.zeros(2, 64, dtype=torch.bfloat16, device="cuda")
    router, w13, w2 = (torch.zeros(*n, dtype=torch.bfloat16, device="cuda") for n in ((4, 64), (4, 2, 32, 64), (4, 64, 32)))
    with pytest.raises(ValueError, match="w2"):
        moe.few(x, router, 2, w13, w2[:3])
    with pytest.raises(ValueError, match="8-bit weights need"):
        moe.few(x, router, 2, w13.to(torch.float8_e4m3fn), w2.to(torch.float8_e4m3fn))
    with pytest.raises(B.TunaError, match="TUNA_ERR_RANGE"):
        moe.few(torch.zeros(65, 64, dtype=torch.bfloat16, device="cuda"), router, 2, w13, w2,
                workspace=torch.zeros(1 << 20, dtype=torch.uint8, device="cuda"))
    with pytest.raises(B.TunaError, match="TUNA_ERR_WORKSPACE"):
        moe.few(x, router, 2, w13, w2, workspace=torch.zeros(256, dtype=torch.uint8, device="cuda"))


def test_stream_arguments():
    """None, a torch stream and a raw handle are taken alike."""
    from paper_2411_02581_b200 import moe
    z = torch.randn(300, 64, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    want = moe.route(z, 2)
    for stream in (side, side.cuda_stream):
        got = moe.route(z, 2, stream=stream)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, got))
    with torch.cuda.stream(side):
        got = moe.route(z, 2)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
