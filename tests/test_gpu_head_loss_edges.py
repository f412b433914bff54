"""Calls of the loss of hidden rows that its own tests leave out."""
import pytest
import torch

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16
NAN = float("nan")
BAD_TOKEN = 5      # DX_DEV_BAD_TOKEN


@pytest.fixture()
def dx():
    from paper_2607_24434_b200 import binding
    ctx = binding.Context(0)
    ctx.set_wait_limit(1 << 18)
    yield binding, ctx
    assert ctx.device_status() == 0
    ctx.close()


@pytest.mark.parametrize("N", [9, 250, 400])
def test_rows_of_weight_zero_may_have_any_target(dx, N):
    """A padded batch whose padding holds what another framework ignores: the weight says that the rows do not count.  The same
    bits as with targets of -1, nothing reported; with a weight such a target is."""
    binding, ctx = dx
    g = torch.Generator(device="cuda").manual_seed(N)
    h = torch.randn((N, 64), generator=g, device="cuda").to(BF16)
    W = (torch.randn((300, 64), generator=g, device="cuda") * 0.2).to(BF16)
    t = torch.randint(0, 300, (N,), generator=g, device="cuda").to(torch.int32)
    w = torch.rand((N,), generator=g, device="cuda") + 0.5
    pad = torch.arange(N, device="cuda") % 3 == 1
    w[pad] = 0.0
    h[pad] = NAN
    ids = torch.tensor([-100, 300, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device="cuda").repeat(N)[:N]
    want = binding.spec_head_loss(ctx, h, W, torch.where(pad, -1, t), row_weight=w, grad_weight=True)
    got = binding.spec_head_loss(ctx, h, W, torch.where(pad, ids, t), row_weight=w, grad_weight=True)
    assert ctx.device_status() == 0
    assert not got["loss"][pad].any() and not got["dh"][pad].any()
    assert all(torch.equal(got[key], want[key]) for key in want)
    w[4] = 0.25
    got = binding.spec_head_loss(ctx, h, W, torch.where(pad, ids, t), row_weight=w, grad_weight=True)
    assert ctx.device_status() == BAD_TOKEN and ctx.device_status() == 0
    assert got["loss"].isnan().nonzero().tolist() == [[4]] and not got["dh"][4].any() and torch.equal(got["dW"], want["dW"])
