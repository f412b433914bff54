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


def test_workspace_of_the_loss(lib):
    """What is kept and what is not, by size: short hidden rows keep their logits (fp32) up to 64 MB (of up to 32768 rows), long
    ones up to 2 GB; beside them the packed rows, a piece of dz of up to 256 MB (in bf16, whole blocks of 256 words), shares of dh
    or one sum of it, halves of tiles (of 128 words or more)."""
    _, L, ctx, _ = lib
    least, best = ctypes.c_size_t(0), ctypes.c_size_t(0)
    for N in (1, 16, 128, 129, 1000, 4096, 40000, 1 << 20):
        for V in (1, 257, 32768, 102400):
            words = (V + 255) // 256 * 256
            for H in (64, 1024, 1280, 2048, 8192):
                assert L.spec_head_loss_workspace(ctx, N, V, H, 1, ctypes.byref(least), ctypes.byref(best)) == 0
                fixed = N * H * 2 + 16 * N + 16 * ((V + 127) // 128) * (N + 32) + 4096
                piece = max(256 << 20, 512 * N)
                few = 4 * N * words <= 64 << 20 and N <= 32768
                logits = 4 * N * words if few or (H >= 1280 and 4 * N * words <= 2 << 30) else 0
                shares = 4 * N * H * (32 if N <= 32768 else 1)
                assert N * H * 2 < least.value <= fixed + 512 * N + 4 * N * H + 512
                assert least.value <= best.value <= max(least.value, fixed + logits + min(piece, 2 * N * words) + shares + 2048)
                assert best.value >= logits + 2 * N * H
                loss = ctypes.c_size_t(0)
                assert L.spec_head_loss_workspace(ctx, N, V, H, 0, ctypes.byref(loss), ctypes.byref(best)) == 0
                assert loss.value == best.value <= fixed


def test_workspace_refuses_what_the_loss_refuses(lib):
    _, L, ctx, _ = lib
    a, b = ctypes.c_size_t(7), ctypes.c_size_t(7)
    ask = lambda N, V, H: L.spec_head_loss_workspace(ctx, N, V, H, 1, ctypes.byref(a), ctypes.byref(b))  # noqa: E731
    top = 2 ** 31 - 1
    assert ask(top, 100, 64) == 8 and ask(top - 2047, 100, 64) == 8 and ask(10, top, 64) == 8 and ask(1 << 30, 1 << 30, 64) == 8
    assert ask(1 << 24, 100, 64) == 0 and a.value > (1 << 24) * 128 and ask(10, 1 << 24, 64) == 0
    call = lambda N, V: L.spec_head_loss(ctx, A, N, 64, B, V, 64, 64, 64, None, 64, None, 64, None, 64, G, 1 << 62, None)  # noqa: E731
    assert call(top, 100) == 8 and call(top - 2047, 100) == 8 and call(10, top) == 8 and call(1 << 29, 1 << 29) == 8 and call(10, 100) == 3
