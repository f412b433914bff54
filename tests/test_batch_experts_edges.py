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


def test_sizes_that_32_bits_do_not_count(lib):
    """Rows, columns and tokens that reach 2^31 with the step of a grid or a tile behind them: refused, not counted past it."""
    binding, L, ctx, _ = lib
    top = 2 ** 31 - 8
    desc = lambda rows=100, n=64, k=32: ctypes.byref(binding.GroupedDesc(1, rows, n, k, k, n * k))  # noqa: E731
    far = 1 << 45

    def mm(d, x_rows=100, ldx=32, y_rows=100, ldy=64, t=0):
        return L.moe_grouped_mm(ctx, d, A, x_rows, ldx, far, t, 64, None, 1, None, 2 * far, 1, y_rows, ldy, None)

    assert mm(desc(n=top, k=8), ldx=8, ldy=top, y_rows=1, x_rows=100) in (2, 8)
    assert mm(desc(rows=1, n=top, k=8), ldx=8, ldy=top) == 8 and mm(desc(rows=1, n=8, k=top), ldx=top, ldy=8, x_rows=1) == 8
    assert mm(desc(rows=top, n=8, k=8), x_rows=top, ldx=8, y_rows=top, ldy=8) == 8
    assert mm(desc(rows=1 << 30, n=8, k=8), x_rows=1 << 30, ldx=8, y_rows=1 << 30, ldy=8) == 3
    dw = lambda d, rows, n, k: L.moe_grouped_mm_dw(ctx, d, A, rows, n, None, 1, far, rows, k, None, 1, 64, 2 * far, 0, None)  # noqa: E731
    assert dw(desc(top, 8, 8), top, 8, 8) == 8 and dw(desc(1, top, 8), 1, top, 8) == 8 and dw(desc(1, 8, top), 1, 8, top) == 8
    assert dw(desc(1 << 30, 8, 8), 1 << 30, 8, 8) == 3
    combine = lambda N, k, H: L.moe_combine_tokens(ctx, A, 1, H, None, N, k, H, far, 1, H, None)  # noqa: E731
    back = lambda N, k, H: L.moe_combine_tokens_backward(ctx, A, H, far, H, 1, None, N, k, H, 2 * far, H, None, None)  # noqa: E731
    for call in (combine, back):
        assert call(2 ** 31 - 1, 1, 8) == 8 and call(2 ** 28, 8, 8) == 8 and call(1, 1, top) == 8 and call(1 << 30, 1, 8) == 3
    a, b = ctypes.c_size_t(0), ctypes.c_size_t(0)
    assert L.spec_head_loss_workspace(ctx, 1, 100, top, 1, ctypes.byref(a), ctypes.byref(b)) == 8
    assert L.spec_head_loss(ctx, A, 1, top, far, 1, top, top, 64, None, 64, None, top, None, top, G, 1 << 62, None) == 8
