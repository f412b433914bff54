"""What the entry points of the experts' products, their combination and the loss refuse, before anything touches a device."""
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


def desc(binding, E=4, rows=100, n=64, k=32, ld=None, stride=None):
    ld = k if ld is None else ld
    return ctypes.byref(binding.GroupedDesc(E, rows, n, k, ld, n * ld if stride is None else stride))


def test_grouped_mm_refusals(lib):
    binding, L, ctx, _ = lib

    def call(d=None, ctx=ctx, x=A, x_rows=100, ldx=32, w=B, t=0, off=64, gather=None, div=1, scatter=None, y=C, dt=1, y_rows=100,
             ldy=64, **kw):
        return L.moe_grouped_mm(ctx, desc(binding, **kw) if d is None else d, x, x_rows, ldx, w, t, off, gather, div, scatter, y,
                                dt, y_rows, ldy, None)

    assert call(ctx=None) == 1 and call(d=ctypes.POINTER(binding.GroupedDesc)()) == 1
    assert call(t=2) == 1 and call(dt=2) == 1 and call(div=0) == 1 and call(off=None) == 1
    assert call(w=None) == 1 and call(w=B + 8) == 1 and call(x=None) == 1 and call(x=A + 2) == 1 and call(y=C + 4) == 1
    assert call(E=0) == 2 and call(rows=-1) == 2 and call(n=0) == 2 and call(k=0) == 2 and call(ld=24) == 2
    assert call(E=257) == 8 and call(n=60, ldy=60) == 8 and call(k=36, ldx=36) == 8 and call(ld=36) == 8 and call(stride=64 * 32 + 4) == 8
    assert call(stride=32) == 2 and call(ldx=24) == 2 and call(ldx=36) == 8 and call(ldy=56) == 2 and call(ldy=68) == 8
    assert call(x_rows=99) == 2 and call(y_rows=99) == 2 and call(gather=64, x_rows=0, x=None) == 2
    assert call(t=1, ldx=32) == 2                                           # (transposed: rows of x have n elements)
    assert call(y=A) == 1 and call(y=A + 100 * 64 - 16) == 1 and call(y=B + 64) == 1 and call(y=A - 16) == 1
    assert call(E=256, n=1 << 30, k=8, ldx=8, ldy=1 << 30, ld=8) == 8          # more tiles than 32 bits number
    assert call(rows=0, x=None, x_rows=0, y=None, y_rows=0, off=None) == 0
    assert call() == 3                                                       # (nothing to refuse: no device here)


def test_grouped_dw_refusals(lib):
    binding, L, ctx, _ = lib

    def call(ctx=ctx, dy=A, dy_rows=100, ld_dy=64, gdy=None, ddiv=1, x=B, x_rows=100, ldx=32, gx=None, xdiv=1, off=64, dw=C, dt=0, **kw):
        return L.moe_grouped_mm_dw(ctx, desc(binding, **kw), dy, dy_rows, ld_dy, gdy, ddiv, x, x_rows, ldx, gx, xdiv, off, dw, dt, None)

    assert call(ctx=None) == 1 and call(dt=3) == 1 and call(ddiv=0) == 1 and call(xdiv=-1) == 1 and call(off=None) == 1
    assert call(dw=None) == 1 and call(dy=None) == 1 and call(x=B + 8) == 1 and call(dw=C + 8) == 1
    assert call(ld_dy=56) == 2 and call(ldx=36) == 8 and call(dy_rows=99) == 2 and call(x_rows=7) == 2
    assert call(dw=A) == 1 and call(dw=B + 1600) == 1 and call(E=257) == 8
    assert call() == 3


def test_swiglu_refusals(lib):
    binding, L, ctx, _ = lib

    def call(ctx=ctx, x=A, x_rows=100, ldx=32, w=B, off=64, gather=None, div=1, act=C, ld_act=32, gu=None, ld_gu=64, **kw):
        return L.moe_grouped_swiglu(ctx, desc(binding, **kw), x, x_rows, ldx, w, off, gather, div, act, ld_act, gu, ld_gu, None)

    assert call(ctx=None) == 1 and call(div=0) == 1 and call(off=None) == 1 and call(act=None) == 1 and call(w=None) == 1
    assert call(n=72) == 8 and call(n=63) == 8 and call(ld_act=24) == 2 and call(gu=D, ld_gu=56) == 2 and call(gu=D + 8) == 1
    assert call(x_rows=50) == 2 and call(gu=C) == 1 and call(act=A) == 1 and call(gu=B) == 1
    assert call(rows=0, x=None, x_rows=0, act=None, off=None) == 0
    assert call() == 3 and call(gu=D) == 3

    def back(ctx=ctx, dy=A, rows_=100, ld=64, wd=B, gu=C, ld_gu=64, pw=64, n_pairs=100, off=64, gather=None, div=1, d=D, ld_d=64,
             act=F, ld_act=32, dpw=64, ws=G, size=1 << 20, **kw):
        return L.moe_grouped_swiglu_backward(ctx, desc(binding, **kw), dy, rows_, ld, wd, gu, ld_gu, pw, n_pairs, off, gather, div, d,
                                             ld_d, act, ld_act, dpw, ws, size, None)

    assert back(ctx=None) == 1 and back(div=0) == 1 and back(off=None) == 1 and back(gu=None) == 1 and back(d=None) == 1
    assert back(ld_gu=56) == 2 and back(ld_d=68) == 8 and back(ld_act=24) == 2 and back(rows_=99) == 2 and back(n_pairs=99) == 2
    need = ctypes.c_size_t(0)
    assert L.moe_grouped_swiglu_backward_workspace(desc(binding), ctypes.byref(need)) == 0 and need.value == 8 * 100 * 4
    assert back(ws=None) == 1 and back(size=need.value - 1) == 1 and back(ws=G + 4) == 1
    assert back(d=C) == 1 and back(act=D + 64) == 1 and back(act=A) == 1 and back(d=B) == 1
    assert back() == 3 and back(dpw=None, ws=None, size=0) == 3 and back(size=need.value) == 3
    assert L.moe_grouped_swiglu_backward_workspace(None, ctypes.byref(need)) == 1
    assert L.moe_grouped_swiglu_backward_workspace(desc(binding), None) == 1


def test_combine_refusals(lib):
    _, L, ctx, _ = lib

    def call(ctx=ctx, z=A, zdt=1, ldz=64, w=64, N=10, k=4, H=64, y=B, ydt=0, ldy=64):
        return L.moe_combine_tokens(ctx, z, zdt, ldz, w, N, k, H, y, ydt, ldy, None)

    assert call(ctx=None) == 1 and call(zdt=2) == 1 and call(ydt=-1) == 1 and call(z=None) == 1 and call(y=B + 8) == 1
    assert call(N=-1) == 2 and call(k=0) == 2 and call(H=0) == 2 and call(k=9) == 8 and call(H=60) == 8 and call(ldz=56) == 2
    assert call(N=1 << 29, k=8) == 8 and call(y=A) == 1 and call(y=A + 39 * 128 + 64) == 1
    assert call(N=0, z=None, y=None) == 0 and call() == 3 and call(w=None) == 3

    def back(ctx=ctx, dy=A, ld_dy=64, z=B, ldz=64, dt=1, w=64, N=10, k=4, H=64, dz=C, ld_dz=64, dw=64):
        return L.moe_combine_tokens_backward(ctx, dy, ld_dy, z, ldz, dt, w, N, k, H, dz, ld_dz, dw, None)

    assert back(ctx=None) == 1 and back(dt=2) == 1 and back(dy=None) == 1 and back(z=None) == 1 and back(dz=C + 8) == 1
    assert back(dz=None, dw=None) == 1 and back(dz=A) == 1 and back(dz=B) == 1 and back(ldz=36) == 2 and back(k=9) == 8
    assert back() == 3 and back(z=None, dw=None) == 3 and back(dz=None) == 3


def test_head_loss_refusals(lib):
    _, L, ctx, _ = lib
    least, best = ctypes.c_size_t(0), ctypes.c_size_t(0)
    ask = lambda *a, c=ctx: L.spec_head_loss_workspace(c, *a, ctypes.byref(least), ctypes.byref(best))  # noqa: E731
    assert ask(10, 100, 64, 1, c=None) == 1 and ask(-1, 100, 64, 1) == 2 and ask(10, 0, 64, 1) == 2 and ask(10, 100, 0, 1) == 2
    assert ask(0, 100, 64, 1) == 0 and least.value == 0 == best.value
    for N in (1, 10, 128, 129, 1000, 40000):
        for V in (1, 257, 102400):
            for grad in (0, 1):
                assert ask(N, V, 64, grad) == 0 and 0 < least.value <= best.value
                # logits in fp32 would take N V 4 bytes: the workspace stays below what a bounded piece needs
                assert best.value <= (600 << 20) + N * (64 * 2 + 64 * 4 * 33 + 20) + 16 * ((V + 255) // 256) * (N + 32) * 2
    assert ask(10, 100, 64, 1) == 0
    need = least.value

    def call(ctx=ctx, h=A, N=10, ldh=64, W=B, V=100, ldw=64, H=64, t=64, w=None, loss=64, dh=C, ld_dh=64, dW=D, ld_dW=64, ws=G,
             size=need):
        return L.spec_head_loss(ctx, h, N, ldh, W, V, ldw, H, t, w, loss, dh, ld_dh, dW, ld_dW, ws, size, None)

    assert call(ctx=None) == 1 and call(h=None) == 1 and call(W=None) == 1 and call(t=None) == 1 and call(ws=None) == 1
    assert call(h=A + 8) == 1 and call(dh=C + 2) == 1 and call(ws=G + 128) == 1 and call(size=need - 1) == 1
    assert call(N=-1) == 2 and call(V=0) == 2 and call(H=60, ldh=60, ldw=60) == 8 and call(ldw=56) == 2 and call(ld_dW=68) == 8
    assert call(loss=None, dh=None, dW=None) == 1 and call(dh=A) == 1 and call(dW=B) == 1 and call(dW=C) == 1
    assert call() == 3 and call(loss=None) == 3 and call(dh=None, dW=None) == 3
