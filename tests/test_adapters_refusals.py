"""What moe_adapter_forward and moe_adapter_backward refuse beyond test_adapters.py, on the CPU."""

import ctypes

import pytest
import torch  # before the library is loaded: both then share one HIP runtime

from paper_2304_11414_amd import binding as B
from tests.test_adapters import GOOD, lib  # noqa: F401  (lib: a fixture of the module)

MB = 1 << 20


def calls(cfg):
    lib, c = B.load_library(), ctypes.byref(cfg)
    return ((lib.moe_adapter_forward, lib.moe_adapter_workspace_bytes(c), 11, (8, 9, 10)),
            (lib.moe_adapter_backward, lib.moe_adapter_backward_workspace_bytes(c), 14, (10, 11, 12, 13)))


def test_outputs_that_begin_inside_the_adapter_numbers_are_refused():
    """Without perm there is one number per row: 100 of them, 400 bytes."""
    cfg = B.make_adapter_config(**GOOD)
    for call, need, n, written in calls(cfg):
        for w in written:
            a = [(i + 1) * 1024 * MB for i in range(n)]
            a[7] = None
            a[w] = a[6] + 384
            assert call(ctypes.byref(cfg), *(None if p is None else ctypes.c_void_p(p) for p in a), need, None) == -7, (n, w)


MOST_ROWS = (1 << 28) - 256


@pytest.mark.parametrize("K,N,rank", [(8, 8, 8), (1 << 20, 8, 128), (8, 1 << 20, 8), (1 << 20, 1 << 20, 64)])
def test_rows_beyond_a_grid_are_refused_and_fewer_have_a_workspace(K, N, rank):
    lib = B.load_library()
    for rows, good in ((MOST_ROWS, True), (MOST_ROWS + 1, False), ((1 << 31) - 1, False)):
        cfg = B.make_adapter_config(rows, K, N, 1, 1, rank)
        c = ctypes.byref(cfg)
        for size in (lib.moe_adapter_workspace_bytes(c), lib.moe_adapter_backward_workspace_bytes(c)):
            assert (size >= rows * rank * 4) if good else size == 0
        if not good:
            p = [ctypes.c_void_p(i << 44) for i in range(1, 15)]
            assert lib.moe_adapter_forward(c, *p[:11], 1 << 43, None) == -2
            assert lib.moe_adapter_backward(c, *p, 1 << 43, None) == -2
