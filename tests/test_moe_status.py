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
