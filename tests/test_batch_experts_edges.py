"""What the batch experts' entry points take and refuse where a description has two readings, before anything touches a device."""
import ctypes

import pytest
import torch


@pytest.fixture()
def lib():
    if torch.cuda.is_available():
        pytest.skip("host-only: with a device a call that is not refused would run on made-up addresses")
    from paper_2607_24434_b200 import binding
    blank = ctypes.create_string_buffer(4096)
    return binding, binding.load(), ctypes.addressof(blank), blank


A, B, C, D, F, G = (1 << 30, 1 << 32, 1 << 34, 1 << 36, 1 << 38, 1 << 40)      # addresses far from each other


def test_rows_of_dy_that_pairs_in_order_need(lib):
    """100 pairs without a list of them, ``div`` to a token: a row of dy for every token."""
    binding, L, ctx, _ = lib
    desc = ctypes.byref(binding.GroupedDesc(4, 100, 64, 32, 32, 64 * 32))

    def back(dy_rows, div, gather=None, n_pairs=100):
        return L.moe_grouped_swiglu_backward(ctx, desc, A, dy_rows, 64, B, C, 64, 64, n_pairs, 64, gather, div, D, 64, F, 32, 64, G,
                                             1 << 20, None)

    assert back(100, 1) == 3 and back(25, 4) == 3 and back(15, 7) == 3 and back(1, 100) == 3 and back(1, 1 << 30) == 3
    assert back(99, 1) == 2 and back(24, 4) == 2 and back(14, 7) == 2 and back(0, 100) == 2
    assert back(25, 4, n_pairs=99) == 2 and back(1, 4, gather=64, n_pairs=1) == 3
