"""The batch operators at the edges of their documented ranges: values, precision and rows that `test_gpu_batch_ops.py`
does not reach.  References are 64-bit torch on the GPU."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DTYPES = [torch.float32, torch.bfloat16]
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
NAN, INF = float("nan"), float("inf")


@pytest.fixture()
def dx():
    from paper_2607_24434_b200 import binding
    ctx = binding.Context(0)
    yield binding, ctx
    assert ctx.device_status() == 0
    ctx.close()


@pytest.mark.parametrize("dtype", DTYPES)
def test_distill_lists_outside_the_range_of_exp(dx, dtype):
    """A renormalised list is the same teacher whatever constant its log probabilities carry.  The constants are
    ones that the sums hold exactly, so loss and gradient are the same bit for bit."""
    binding, ctx = dx
    N, V, k = 9, 704, 40
    g = torch.Generator(device="cuda").manual_seed(50)
    z = (torch.randn((1, V), generator=g, device="cuda") * 2).to(dtype).expand(N, V).contiguous()
    ids = torch.randperm(V, generator=g, device="cuda")[:k].to(torch.int32).expand(N, k).contiguous()
    base = -torch.randint(0, 160, (k,), generator=g, device="cuda").float() / 16
    shift = torch.tensor([0.0, -512.0, -720.0, -744.0, -1024.0, -65536.0, 720.0, 1024.0, 65536.0], device="cuda")
    lp = (base + shift[:, None]).contiguous()
    assert torch.equal(lp - shift[:, None], base.expand(N, k))
    for grad in (True, False):
        got = binding.spec_distill_topk(ctx, z, ids, lp, grad=grad)
        assert torch.isfinite(got["loss"]).all() and (got["loss"] == got["loss"][0]).all()
        if grad:
            assert torch.isfinite(got["dlogits"]).all() and (got["dlogits"] == got["dlogits"][0]).all()
    p = torch.softmax(base.double(), 0)
    logq = torch.log_softmax(z[0].double(), 0)
    want = (p * (p.log() - logq[ids[0].long()])).sum()
    # log S: an exponential 2^-22, the two roundings of its argument at most 2^-23 of a |u| whose mean is below 10, some
    # fifteen additions 2^-24 each -- below 2^-18 together; the result half a step of fp32
    assert abs(float(got["loss"][0].double() - want)) <= 2.0 ** -18 + 2.0 ** -24 * abs(float(want))
    # entries of -inf beside such ones carry no mass; a list of nothing else has loss 0 and gradient 0
    lp[:, ::2] = -INF
    lp[1] = -INF
    got = binding.spec_distill_topk(ctx, z, ids, lp)
    live = torch.arange(N, device="cuda") != 1
    assert (got["loss"][live] == got["loss"][0]).all() and float(got["loss"][1]) == 0
    assert torch.isfinite(got["dlogits"]).all() and not got["dlogits"][1].any()
