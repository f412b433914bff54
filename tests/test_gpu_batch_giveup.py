"""The give-up path of the batch products' bounded waits: with a limit of a single poll the waits for copies, products and tiles
run out while others are on their way.  Every form of the kernel -- CTAs by themselves and in pairs, operands by tensor map and
gathered, boxes of gate and up -- records DX_DEV_WAIT_EXPIRED, waits (bounded) for what is in flight and returns; with the
default limit restored the same call gives the same bits as before, again and again."""
import pytest
import torch

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
WAIT_EXPIRED = 2      # DX_DEV_WAIT_EXPIRED


def rng(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def draw(g, *shape, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(BF16)


def grouped(binding, ctx, g, rows, transposed, gathered, dtype):
    E, n, k = 24, 2048, 2048
    P = E * rows
    off = torch.arange(E + 1, dtype=torch.int32, device="cuda") * rows
    w, x = draw(g, E, n, k), draw(g, P, k)
    index = torch.randperm(P, generator=g, device="cuda").to(torch.int32) if gathered else None
    return lambda: [binding.moe_grouped_mm(ctx, x, w, off, transposed=transposed, gather=index, out_dtype=dtype)]


def gradient(binding, ctx, g, rows, k, gathered):
    E, n = 4, 1024
    off = torch.arange(E + 1, dtype=torch.int32, device="cuda") * rows
    dy, x = draw(g, E * rows, n), draw(g, E * rows, k)
    index = torch.randperm(E * rows, generator=g, device="cuda").to(torch.int32) if gathered else None
    return lambda: [binding.moe_grouped_mm_dw(ctx, dy, x, off, gather_x=index, out_dtype=F32)]


def swiglu(binding, ctx, g, rows, backward, gathered):
    E, H, I = 24, 2048, 1024
    P = E * rows
    off = torch.arange(E + 1, dtype=torch.int32, device="cuda") * rows
    index = torch.randperm(P, generator=g, device="cuda").to(torch.int32) if gathered else None
    if backward:
        dy, wd, gate_up = draw(g, P, H), draw(g, E, H, I), draw(g, P, 2 * I)
        topk_w = torch.rand((P,), generator=g, device="cuda") + 0.1
        return lambda: list(binding.moe_grouped_swiglu_backward(ctx, dy, wd, gate_up, topk_w, off, gather=index).values())
    x, w = draw(g, P, H), draw(g, E, 2 * I, H)
    return lambda: list(binding.moe_grouped_swiglu(ctx, x, w, off, gather=index, save=True).values())


def head(binding, ctx, g, rows, H):
    h, W = draw(g, rows, H), draw(g, 30011, H, scale=H ** -0.5)
    t = torch.randint(0, 30011, (rows,), generator=g, device="cuda").to(torch.int32)
    return lambda: list(binding.spec_head_loss(ctx, h, W, t, grad_weight=True).values())


CALLS = {
    "pairs": (grouped, 300, False, False, BF16), "pairs_gathered": (grouped, 300, False, True, F32),
    "pairs_transposed": (grouped, 300, True, True, BF16), "few": (grouped, 2, False, False, F32),
    "few_gathered": (grouped, 20, True, True, BF16), "some": (grouped, 50, True, False, BF16),
    "dw": (gradient, 1000, 1024, False), "dw_gathered": (gradient, 1000, 1024, True), "dw_single": (gradient, 60, 640, True),
    "dw_long": (gradient, 13000, 1024, False), "dw_long_gathered": (gradient, 13000, 1024, True),
    "swiglu": (swiglu, 300, False, False), "swiglu_few": (swiglu, 4, False, True),
    "swiglu_grad": (swiglu, 300, True, False), "swiglu_grad_gathered": (swiglu, 300, True, True),
    "swiglu_grad_some": (swiglu, 50, True, True), "swiglu_grad_few": (swiglu, 8, True, False),
    "head_few": (head, 16, 2048), "head": (head, 600, 2048), "head_recomputed": (head, 600, 1024),
}


@pytest.mark.parametrize("name", CALLS)
def test_waits_cut_short(name):
    from paper_2607_24434_b200 import binding
    ctx = binding.Context(0)
    make, *args = CALLS[name]
    call = make(binding, ctx, rng(len(name)), *args)
    want = [t.clone() for t in call()]
    torch.cuda.synchronize()
    assert ctx.device_status() == 0
    expired = 0
    for polls in (1, 1, 2, 8, 32):
        ctx.set_wait_limit(polls)
        call()                                       # (what it leaves in its outputs is undefined)
        torch.cuda.synchronize()
        status = ctx.device_status()
        assert status == WAIT_EXPIRED or (status == 0 and polls > 1)
        expired += status == WAIT_EXPIRED
        assert ctx.device_status() == 0              # reading clears the word
        ctx.set_wait_limit(0)
        for _ in range(2):
            assert all(torch.equal(a, b) for a, b in zip(call(), want))
        assert ctx.device_status() == 0
    assert expired >= 2
    ctx.close()
