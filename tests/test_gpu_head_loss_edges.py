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


@pytest.mark.parametrize("N", [3, 200])
@pytest.mark.parametrize("H", [4104, 65536])
def test_logits_of_long_hidden_rows(dx, N, H):
    """Targets whose logits are sums of positive terms only, all other logits 0: loss = log(1 + (V - 1) exp(-z)).  Sections of 4096
    terms bound what the tensor cores' truncating additions take off z: (2 * 4096 / 16 + 2) 2^-23 of it and 2^-24 for every section;
    the loss changes by (1 - p) times that, and is good to 2^-16 otherwise (as the other tests allow)."""
    binding, ctx = dx
    V = 300
    g = torch.Generator(device="cuda").manual_seed(N)
    W = torch.zeros((V, H), dtype=BF16, device="cuda")
    W[7] = ((torch.rand((H,), generator=g, device="cuda") + 0.5) * 8 / H).to(BF16)
    h = (torch.rand((N, H), generator=g, device="cuda") + 0.5).to(BF16)
    t = torch.full((N,), 7, dtype=torch.int32, device="cuda")
    z = h.double() @ W[7].double()
    rest = (V - 1) * torch.exp(-z)
    want = torch.log1p(rest)
    off = ((2 * 4096 / 16 + 2) * 2.0 ** -23 + (H // 4096 + 1) * 2.0 ** -24) * z * rest / (1 + rest)
    kept = binding.spec_head_loss(ctx, h, W, t)
    assert bool(((kept["loss"].double() - want).abs() <= off + 2.0 ** -16 * want).all())
    least, _ = binding.spec_head_loss_workspace(ctx, N, V, H)
    again = binding.spec_head_loss(ctx, h, W, t, workspace=torch.empty(least, dtype=torch.uint8, device="cuda"))
    assert torch.equal(again["loss"], kept["loss"]) and torch.equal(again["dh"], kept["dh"])
