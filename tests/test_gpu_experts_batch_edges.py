"""Calls of the batch experts' operators that their own tests leave out: rows outside every group, rows that name a pair twice or
none at all, indexes that are not given."""
import pytest
import torch

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
NAN = float("nan")
BAD_ROW = 7      # DX_DEV_BAD_ROW


@pytest.fixture()
def dx():
    from paper_2607_24434_b200 import binding
    ctx = binding.Context(0)
    ctx.set_wait_limit(1 << 18)
    yield binding, ctx
    assert ctx.device_status() == 0
    ctx.close()


def rng(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def draw(g, *shape, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(BF16)


def ints(*values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def poison():
    """Memory that the allocator hands out next holds NaN: small blocks and large ones."""
    held = [torch.full((256,), NAN, device="cuda") for _ in range(8192)]
    held += [torch.full((1 << 20,), NAN, device="cuda") for _ in range(8)]
    del held


@pytest.mark.parametrize("first,each,index", [(40, 10, "all"), (0, 31, "all"), (256, 0, "all"), (0, 32, "twice"), (0, 32, "bad")])
def test_gates_without_a_row_have_gradient_zero(dx, first, each, index):
    """As many sorted rows as pairs, but some pairs without a row that counts: rows in front of the first group and behind the
    last (the experts of one rank, out of the permutation of all), a pair named twice, so that another is not, an index that is
    reported.  The others get what they get where every row counts, bit for bit."""
    binding, ctx = dx
    g = rng(3)
    N, k, E, H, I = 64, 4, 8, 64, 40
    P = N * k
    perm = torch.randperm(P, generator=g, device="cuda").to(torch.int32)
    dy, wd, gate_up = draw(g, N, H), draw(g, E, H, I), draw(g, P, 2 * I)
    topk_w = torch.rand((N, k), generator=g, device="cuda") + 0.1
    off = [min(P, first + each * e) for e in range(E + 1)]
    has_row = torch.zeros(P, dtype=torch.bool, device="cuda")
    rows = slice(off[0], off[-1])
    has_row[perm[rows].long()] = True
    alone = has_row.clone()
    gone = perm[200].item()
    if index == "twice":
        alone[perm[100].item()] = False      # (which of its two rows it gets is not said)
        perm[200] = perm[100]
    elif index == "bad":
        perm[200] = P
    if index != "all":
        has_row[gone] = alone[gone] = False
    every = torch.zeros(P, dtype=torch.float64, device="cuda")
    a = torch.zeros((P, I), dtype=torch.float64, device="cuda")
    src = perm.long().clamp(max=P - 1)
    for e in range(E):
        here = slice(off[e], off[e + 1])
        a[here] = dy[src[here] // k].double() @ wd[e].double()
    gate, up = gate_up.double().chunk(2, dim=1)
    named = perm < P
    every[src[named]] = (a * gate / (1 + torch.exp(-gate)) * up).sum(1)[named]
    off = ints(*off)
    poison()
    got = binding.moe_grouped_swiglu_backward(ctx, dy, wd, gate_up, topk_w, off, gather=perm, gather_div=k)["d_topk_w"]
    assert ctx.device_status() == (BAD_ROW if index == "bad" else 0)
    got = got.reshape(-1)
    assert not bool(got.isnan().any()) and not bool(got[~has_row].any())
    # (sums of H I products of order one: 1e-4 of their size is far above what fp32 leaves and far below any of them)
    assert bool(((got.double() - every).abs()[alone] <= 1e-4 * every.abs().max()).all())
    kept = torch.full_like(topk_w, 7.0)
    out = {"d_gate_up": torch.empty_like(gate_up), "act_w": torch.empty((P, I), dtype=BF16, device="cuda"), "d_topk_w": kept}
    binding.moe_grouped_swiglu_backward(ctx, dy, wd, gate_up, topk_w, off, gather=perm, gather_div=k, out=out)
    assert ctx.device_status() == (BAD_ROW if index == "bad" else 0)
    kept = kept.reshape(-1)
    assert bool((kept[~has_row] == 7.0).all()) and torch.equal(kept[alone], got[alone])


@pytest.mark.parametrize("counts", [[1, 0, 3], [17, 40, 0, 83], [300, 0, 500]])
@pytest.mark.parametrize("k", [1, 2, 6])
def test_pairs_in_order_take_their_tokens_gradient(dx, counts, k):
    """Without ``gather`` sorted row r is pair r and takes row r // gather_div of dy: what the indexes 0, 1, 2, ... give."""
    binding, ctx = dx
    g = rng(k)
    P = (sum(counts) + k - 1) // k * k
    N, E, H, I = P // k, len(counts), 264, 136
    off = [0]
    for c in counts:
        off.append(off[-1] + c)
    off = ints(*off)
    dy, wd, gate_up = draw(g, N, H), draw(g, E, H, I, scale=0.1), draw(g, P, 2 * I)
    topk_w = torch.rand((N, k), generator=g, device="cuda") + 0.1
    order = torch.arange(P, dtype=torch.int32, device="cuda")
    rows = slice(0, sum(counts))
    for w in (topk_w, None):
        plain = binding.moe_grouped_swiglu_backward(ctx, dy, wd, gate_up, w, off, gather_div=k)
        named = binding.moe_grouped_swiglu_backward(ctx, dy, wd, gate_up, w, off, gather=order, gather_div=k)
        assert plain.keys() == named.keys() and all(torch.equal(plain[n][rows], named[n][rows]) for n in ("d_gate_up", "act_w"))
        assert w is None or torch.equal(plain["d_topk_w"], named["d_topk_w"])
    with pytest.raises(ValueError):
        binding.moe_grouped_swiglu_backward(ctx, dy, wd, gate_up[:-1], topk_w, off, gather_div=k)
    # the forward products' rows are their own: gather_div belongs to gather there
    x, w = draw(g, P, H), draw(g, E, 2 * I, H, scale=0.1)
    assert torch.equal(binding.moe_grouped_mm(ctx, x, w, off, gather_div=k)[rows], binding.moe_grouped_mm(ctx, x, w, off)[rows])
    assert torch.equal(binding.moe_grouped_swiglu(ctx, x, w, off, gather_div=k)["act"][rows],
                       binding.moe_grouped_swiglu(ctx, x, w, off)["act"][rows])
