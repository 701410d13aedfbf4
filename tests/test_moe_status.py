"""The report of a wait that a kernel gave up."""
import ctypes

import pytest
import torch

from paper_2411_02581_b200 import binding as B


@pytest.mark.gpu
def test_a_report_is_of_the_calls_since_the_last_one():
    """The word that a kernel raises is raised here from the host: it is reported once, and a later call starts clean."""
    from paper_2411_02581_b200 import moe
    moe.route(torch.randn(4, 8, device="cuda"), 2)
    assert moe.device_status() == 0
    word = B.lib()._ZN8tuna_ops10error_wordEv         # where the kernels' flag is (int *tuna_ops::error_word())
    word.restype, word.argtypes = ctypes.c_void_p, []
    cudart = ctypes.CDLL("libcudart.so.12")
    cudart.cudaMemcpy.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int]
    one = ctypes.c_int(1)
    assert cudart.cudaMemcpy(word(), ctypes.byref(one), 4, 1) == 0
    assert moe.device_status() == 1
    assert moe.device_status() == 0


@pytest.mark.gpu
def test_the_meeting_counter_after_any_call_is_where_the_next_one_expects_it():
    """Every block arrives three times a call, with units of work or without: the count is a multiple of the grid's size."""
    from paper_2411_02581_b200 import moe
    e, k, d, i = 8, 2, 256, 128
    g = torch.Generator(device="cuda").manual_seed(1)
    new = lambda *n: torch.randn(*n, generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    router, w13, w2 = new(e, d), new(e, 2, i, d), new(e, d, i)
    ws = moe.few_workspace(64, e, k, d, i)
    grid = torch.cuda.get_device_properties(0).multi_processor_count
    none = torch.full((3, d), float("nan"), dtype=torch.bfloat16, device="cuda")     # no token has an expert: no units
    for calls, x in enumerate((new(1, d), none, new(64, d), none, new(17, d)), 1):
        moe.few(x, router, k, w13, w2, workspace=ws)
        assert int(ws[:8].view(torch.int64)) == 3 * grid * calls
    assert moe.device_status() == 0
