"""Arguments that are not where their fellows are, refused before any pointer is followed.  No GPU needed:
the tensors only say that they are on one."""
import pytest
import torch

FP8, BF16, F32 = torch.float8_e4m3fn, torch.bfloat16, torch.float32


class Claimed(torch.Tensor):
    """A CPU tensor that says it is on a GPU."""
    is_cuda = True

    @property
    def device(self):
        return torch.device("cuda", self.gpu)


def claimed(shape, dtype, gpu=0):
    t = torch.zeros(shape, dtype=torch.uint8 if dtype == FP8 else dtype)
    t = (t.view(FP8) if dtype == FP8 else t).as_subclass(Claimed)
    t.gpu = gpu
    return t


def args(**elsewhere):
    e, i, d, t, k = 4, 32, 64, 6, 2
    shapes = dict(x=((t, d), BF16), ids=((t, k), torch.int32), weights=((t, k), F32), offsets=((e + 1,), torch.int64),
                  w13=((e, 2, i, d), FP8), s13=((e, 2, 1, 1), F32), w2=((e, d, i), FP8), s2=((e, 1, 1), F32),
                  y=((t * k, d), BF16), dout=((t, d), BF16), pos=((t, k), torch.int64))
    return {n: claimed(*s, gpu=elsewhere.get(n, 0)) for n, s in shapes.items()}


ROWS = ("x", "offsets", "w13", "s13", "w2", "s2")
MANY = ("x", "ids", "weights", "w13", "s13", "w2", "s2")


@pytest.mark.parametrize("call,names", [("expert_rows", ROWS), ("experts", MANY), ("combine", ("y", "weights", "pos")),
                                        ("combine_backward", ("dout", "y", "weights", "pos"))])
def test_tensors_of_another_gpu(call, names):
    from paper_2411_02581_b200 import moe
    for name in names[1:]:
        a = args(**{name: 1})
        with pytest.raises(ValueError, match=f"{name}: on cuda:1, its fellows are on cuda:0"):
            getattr(moe, call)(*[a[n] for n in names])


@pytest.mark.parametrize("call,names", [("expert_rows", ROWS), ("experts", MANY)])
def test_workspaces_that_a_kernel_could_not_use(call, names):
    from paper_2411_02581_b200 import moe
    a = args()
    for ws, why in ((torch.empty(1 << 20, dtype=torch.uint8), "a contiguous CUDA tensor"), (claimed((1024, 1024), F32).t()[::2], "a contiguous CUDA tensor"),
                    (1 << 20, "a contiguous CUDA tensor"), (claimed((1 << 20,), F32, gpu=1), "workspace: on cuda:1")):
        with pytest.raises(ValueError, match=why):
            getattr(moe, call)(*[a[n] for n in names], workspace=ws)


def test_few_of_a_host_tensor():
    from paper_2411_02581_b200 import moe
    with pytest.raises(ValueError, match="x: a CUDA matrix"):
        moe.few(torch.zeros(2, 64, dtype=BF16), torch.zeros(4, 64, dtype=BF16), 2, torch.zeros(4, 2, 32, 64, dtype=BF16), torch.zeros(4, 64, 32, dtype=BF16))
