"""Waits cut short where a ring's copy thread never waits itself: so few tiles per CTA that all of them are asked for at once.  The
consumers give up while the copies are on their way; the copy thread stays until they have landed, the call returns, and with the
default limit the same call gives the tokens it gave before."""
import pytest
import torch

from paper_2607_24434_b200 import synth

pytestmark = pytest.mark.gpu

WAIT_EXPIRED = 2      # DX_DEV_WAIT_EXPIRED


@pytest.mark.parametrize("V", [16, 148 * 16, 148 * 16 * 2 + 5])
def test_accept_ring_with_all_tiles_on_their_way(V):
    from paper_2607_24434_b200 import binding
    ctx = binding.Context(0)
    M, K, H = 5, 4, 2048
    W = synth.lm_head(V, H, 72, torch.bfloat16, "cuda")
    h = synth.hidden_block(M, H, 73, 0.5, "cuda")
    draft = torch.zeros((K,), dtype=torch.int32, device="cuda")
    want = binding.spec_accept(ctx, h, W, draft, rms_norm=True)["target"].clone()
    torch.cuda.synchronize()
    assert ctx.device_status() == 0
    for polls in (1, 1, 1, 2, 4):
        ctx.set_wait_limit(polls)
        for _ in range(4):
            binding.spec_accept(ctx, h, W, draft, rms_norm=True)
        torch.cuda.synchronize()
        assert ctx.device_status() in (0, WAIT_EXPIRED) and ctx.device_status() == 0
        ctx.set_wait_limit(0)
        assert torch.equal(binding.spec_accept(ctx, h, W, draft, rms_norm=True)["target"], want)
        assert ctx.device_status() == 0
    ctx.close()
