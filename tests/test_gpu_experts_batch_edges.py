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


# ---- long contractions ----------------------------------------------------------------------------------------------------
# The tensor cores' additions truncate, so a contraction goes in sections of 4096 terms (results in fp32) or 32768 (in bf16) whose
# sums are added up rounded to nearest.  A section's error is that of the other tests, (2 n / 16 + 2) 2^-23 of the sum of absolute
# values for n terms, and each of S additions is off by at most half a step, 2^-24 of it.
def long_bound(terms, section):
    n = min(terms, section)
    return (2 * n / 16 + 2) * 2.0 ** -23 + -(-terms // section) * 2.0 ** -24


def whole(g, *shape, some=1.0):
    """-2, -1, 1, 2, and zeros for all but ``some`` of the elements: sums of their products are exact in fp32 below 2^24."""
    x = torch.randint(1, 3, shape, generator=g, device="cuda") * (1 - 2 * torch.randint(0, 2, shape, generator=g, device="cuda"))
    return (x * (torch.rand(shape, generator=g, device="cuda") < some)).to(BF16)


LENGTHS = [[4096, 4097, 0, 8191, 8192, 8193, 5], [12345, 1, 0, 64, 20000], [63, 4159, 4160, 4161, 300, 16389, 0, 0, 700, 4096, 9000, 30]]


@pytest.mark.parametrize("counts", LENGTHS)
@pytest.mark.parametrize("n,k", [(264, 136), (40, 520), (776, 1288)])
def test_gradients_of_long_groups_are_exact_where_their_sums_are(dx, counts, n, k):
    """Long and short groups, empty ones between them, on few and on many tiles: every term is there once."""
    binding, ctx = dx
    g = rng(n + sum(counts))
    P, E = sum(counts), len(counts)
    off = [0]
    for c in counts:
        off.append(off[-1] + c)
    dy, x = whole(g, P, n), whole(g, P, k)
    want = torch.stack([dy[a:b].double().t() @ x[a:b].double() for a, b in zip(off, off[1:])])
    off = ints(*off)
    assert torch.equal(binding.moe_grouped_mm_dw(ctx, dy, x, off, out_dtype=F32).double(), want)
    order = torch.randperm(P, generator=g, device="cuda")
    put = lambda t: torch.empty_like(t).index_copy_(0, order, t)  # noqa: E731
    named = order.to(torch.int32)
    assert torch.equal(binding.moe_grouped_mm_dw(ctx, put(dy), put(x), off, gather_dy=named, gather_x=named, out_dtype=F32).double(), want)


def test_gradients_of_long_groups_in_bf16(dx):
    """Sums of at most 256, which bf16 holds; sections of 32768 rows."""
    binding, ctx = dx
    g = rng(8)
    counts = [32768, 40000, 7, 0, 98310, 32769]
    off = [0]
    for c in counts:
        off.append(off[-1] + c)
    dy, x = whole(g, off[-1], 136, some=0.02), whole(g, off[-1], 264, some=0.02)
    want = torch.stack([dy[a:b].double().t() @ x[a:b].double() for a, b in zip(off, off[1:])])
    assert float(want.abs().max()) <= 256
    assert torch.equal(binding.moe_grouped_mm_dw(ctx, dy, x, ints(*off)).double(), want)


@pytest.mark.parametrize("counts", [[3, 0, 1], [40, 50, 0, 33], [300, 5, 513, 0, 700]])
@pytest.mark.parametrize("K", [4096, 4104, 8192, 8256, 12296])
@pytest.mark.parametrize("transposed", [False, True])
def test_products_of_long_rows_are_exact_where_their_sums_are(dx, counts, K, transposed):
    binding, ctx = dx
    g = rng(K)
    P, E, n = sum(counts), len(counts), 520
    off = [0]
    for c in counts:
        off.append(off[-1] + c)
    w = whole(g, E, K, n) if transposed else whole(g, E, n, K)
    x = whole(g, P, K)
    want = torch.cat([x[a:b].double() @ (w[e].double() if transposed else w[e].double().t()) for e, (a, b) in enumerate(zip(off, off[1:]))])
    off = ints(*off)
    assert torch.equal(binding.moe_grouped_mm(ctx, x, w, off, transposed=transposed, out_dtype=F32).double(), want)
    order = torch.randperm(P, generator=g, device="cuda").to(torch.int32)
    to = torch.randperm(P, generator=g, device="cuda").to(torch.int32)
    y = binding.moe_grouped_mm(ctx, torch.empty_like(x).index_copy_(0, order.long(), x), w, off, transposed=transposed, gather=order,
                               scatter=to, out_dtype=F32)
    assert torch.equal(y[to.long()].double(), want)


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("rows", [3, 40, 300])
def test_products_of_very_long_rows_in_bf16(dx, transposed, rows):
    binding, ctx = dx
    g = rng(rows)
    K = 65544
    w = whole(g, 2, K, 136, some=0.03) if transposed else whole(g, 2, 136, K, some=0.03)
    x = whole(g, 2 * rows, K, some=0.03)
    want = torch.cat([x[e * rows:(e + 1) * rows].double() @ (w[e].double() if transposed else w[e].double().t()) for e in range(2)])
    assert float(want.abs().max()) <= 256
    assert torch.equal(binding.moe_grouped_mm(ctx, x, w, ints(0, rows, 2 * rows), transposed=transposed).double(), want)


def test_one_tile_of_two_million_rows(dx):
    """As long as the other tests' longest, with a limit on waits that is a fraction of the products' time; every one of the terms
    shows in a sum that is exact."""
    binding, ctx = dx
    ctx.set_wait_limit(1 << 15)
    g, P = rng(5), (1 << 21) + 5
    dy, x = whole(g, P, 8), whole(g, P, 16)
    got = binding.moe_grouped_mm_dw(ctx, dy, x, ints(0, P), out_dtype=F32)
    assert ctx.device_status() == 0
    assert torch.equal(got[0].double(), dy.double().t() @ x.double())


@pytest.mark.parametrize("dtype,P", [(F32, 98309), (F32, 400000), (BF16, 1 << 20)])
def test_sums_of_one_sign_do_not_drift(dx, dtype, P):
    """A weight gradient over one long group whose terms are all positive: what truncation takes away does not grow with the rows."""
    binding, ctx = dx
    g = rng(9)
    dy, x = draw(g, P, 64).abs() + 1, draw(g, P, 72).abs() + 1
    want = dy.double().t() @ x.double()
    got = binding.moe_grouped_mm_dw(ctx, dy, x, ints(0, P), out_dtype=dtype)[0].double()
    bound = long_bound(P, 4096) if dtype is F32 else long_bound(P, 32768) + 2.0 ** -8
    assert float(((got - want).abs() / want).max()) <= bound


@pytest.mark.parametrize("transposed", [False, True])
def test_products_of_one_sign_do_not_drift(dx, transposed):
    binding, ctx = dx
    g, K = rng(10), 65536
    x = draw(g, 90, K).abs() + 1
    w = draw(g, 1, *((K, 64) if transposed else (64, K))).abs() + 1
    want = x.double() @ (w[0].double() if transposed else w[0].double().t())
    got = binding.moe_grouped_mm(ctx, x, w, ints(0, 90), transposed=transposed, out_dtype=F32).double()
    assert float(((got - want).abs() / want).max()) <= long_bound(K, 4096)


@pytest.mark.parametrize("rows", [4, 60, 300])
def test_gates_gradients_through_long_rows(dx, rows):
    """d_topk_w = <W^T dy, act> with all terms positive: what the products are off by, what 32-bit sums over I are, and 2^-18 for the
    sigmoid and the activation (as the other tests of it allow)."""
    binding, ctx = dx
    g, H, I = rng(rows), 65536, 40
    dy, wd = draw(g, rows, H).abs() + 1, draw(g, 1, H, I).abs() + 1
    gate_up = draw(g, rows, 2 * I).abs() + 1
    topk_w = torch.rand((rows,), generator=g, device="cuda") + 0.5
    got = binding.moe_grouped_swiglu_backward(ctx, dy, wd, gate_up, topk_w, ints(0, rows))
    gate, up = gate_up.double().chunk(2, dim=1)
    a, s = dy.double() @ wd[0].double(), torch.sigmoid(gate)
    want = (a * gate * s * up).sum(1)
    bound = long_bound(H, 4096) + I * 2.0 ** -23 + 2.0 ** -18
    assert float(((got["d_topk_w"].double() - want).abs() / want).max()) <= bound
    d_up = topk_w.double()[:, None] * a * gate * s
    assert float(((got["d_gate_up"][:, I:].double() - d_up).abs() / d_up).max()) <= bound + 2.0 ** -8


def test_long_contractions_repeat_themselves(dx):
    """Random operands, long and short groups: the same bits in every call, in place and gathered, alone and beside other work."""
    binding, ctx = dx
    g = rng(21)
    off = ints(0, 9000, 9001, 9001, 22000, 22300, 31000)
    P = 31000
    dy, x = draw(g, P, 520), draw(g, P, 776)
    order = torch.randperm(P, generator=g, device="cuda")
    put = lambda t: torch.empty_like(t).index_copy_(0, order, t)  # noqa: E731
    dy2, x2, named = put(dy), put(x), order.to(torch.int32)
    want = binding.moe_grouped_mm_dw(ctx, dy, x, off, out_dtype=F32).clone()
    ref = torch.stack([dy[a:b].double().t() @ x[a:b].double() for a, b in zip(off.tolist(), off.tolist()[1:])])
    # (root mean square of the errors: running sums are no larger than the final ones in the mean)
    for e in range(6):
        if ref[e].any():
            assert float((want[e].double() - ref[e]).pow(2).mean().sqrt()) <= long_bound(P, 4096) * float(ref[e].pow(2).mean().sqrt())
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(5):
        with torch.cuda.stream(side):
            busy = binding.moe_grouped_mm_dw(ctx, x2, dy2, off, gather_dy=named, gather_x=named, out_dtype=F32)
        assert torch.equal(binding.moe_grouped_mm_dw(ctx, dy, x, off, out_dtype=F32), want)
        assert torch.equal(binding.moe_grouped_mm_dw(ctx, dy2, x2, off, gather_dy=named, gather_x=named, out_dtype=F32), want)
    torch.cuda.synchronize()
    assert float((busy.transpose(1, 2) - want).abs().max()) <= 1e-4 * float(want.abs().max())      # (the transposed product)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = binding.moe_grouped_mm_dw(ctx, dy, x, off, out_dtype=F32)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(held, want)
    del graph


# ---- weights of exactly 0 --------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N,k,H", [(5, 3, 64), (40, 8, 1000), (2500, 2, 264)])
def test_gradient_of_a_weight_of_zero(dx, dtype, N, k, H):
    """y is linear in the weights: the slope is <z, dy> at 0 as anywhere (sums of H products in fp32, each addition half a step).  A
    row that was taken out and holds NaN or infinities has slope 0, and so has its dz."""
    binding, ctx = dx
    g = rng(N)
    z = torch.randn((N * k, H), generator=g, device="cuda").to(dtype)
    dy = torch.randn((N, H), generator=g, device="cuda").to(dtype)
    w = torch.randn((N, k), generator=g, device="cuda")
    zero = torch.rand((N, k), generator=g, device="cuda") < 0.4
    w[zero] = 0.0
    w[0, 0] = -0.0
    zero[0, 0] = True
    want = (z.double().view(N, k, H) * dy.double()[:, None]).sum(2)
    size = (z.double().view(N, k, H) * dy.double()[:, None]).abs().sum(2)
    back = binding.moe_combine_tokens_backward(ctx, dy, z, w)
    assert bool(((back["d_topk_w"].double() - want).abs() <= (H / 8 + 16) * 2.0 ** -24 * size).all())
    assert not back["dz"][zero.reshape(-1)].any()
    out = torch.where(zero.reshape(-1, 1), float("inf"), z.float()).to(dtype)
    out[::2] = torch.where(zero.reshape(-1, 1)[::2], NAN, out[::2].float()).to(dtype)
    gone = binding.moe_combine_tokens_backward(ctx, dy, out, w)
    assert not gone["d_topk_w"][zero].any() and torch.equal(gone["d_topk_w"][~zero], back["d_topk_w"][~zero])
    assert torch.equal(gone["dz"], back["dz"])
    # a row that counts and holds NaN shows it
    out[k - 1] = NAN
    w[0, k - 1] = 0.5
    assert bool(binding.moe_combine_tokens_backward(ctx, dy, out, w)["d_topk_w"][0, k - 1].isnan())


@pytest.mark.parametrize("rows", [3, 50, 300])
def test_gradient_of_a_gate_of_zero(dx, rows):
    """d_topk_w does not depend on the gate: a gate of 0 gets what it gets with any other, bit for bit, and 0 where its row holds
    NaN or infinities; d_gate_up and act_w are zeros either way."""
    binding, ctx = dx
    g = rng(rows)
    E, k, H, I = 3, 2, 264, 136
    P = E * rows // k * k
    off = ints(0, rows, 2 * rows, P)
    perm = torch.randperm(P, generator=g, device="cuda").to(torch.int32)
    dy, wd, gate_up = draw(g, P // k, H), draw(g, E, H, I, scale=0.1), draw(g, P, 2 * I)
    w = torch.rand((P // k, k), generator=g, device="cuda") + 0.1
    call = lambda gu, w: binding.moe_grouped_swiglu_backward(ctx, dy, wd, gu, w, off, gather=perm, gather_div=k)  # noqa: E731
    full = call(gate_up, w)
    zero = torch.rand((P // k, k), generator=g, device="cuda") < 0.4
    zero[0, 0] = True
    of_row = zero.reshape(-1)[perm.long()]
    some = call(gate_up, w.masked_fill(zero, 0.0))
    assert bool(full["d_topk_w"][zero].any()) and torch.equal(some["d_topk_w"], full["d_topk_w"])
    for value in (NAN, float("inf")):
        gone = call(gate_up.masked_fill(of_row[:, None], value), w.masked_fill(zero, 0.0))
        assert not gone["d_topk_w"][zero].any() and torch.equal(gone["d_topk_w"][~zero], full["d_topk_w"][~zero])
        for n in ("d_gate_up", "act_w"):
            assert not gone[n][of_row].any() and not some[n][of_row].any()
            assert torch.equal(gone[n][~of_row], full[n][~of_row]) and torch.equal(some[n][~of_row], full[n][~of_row])
    # a gate that counts shows what its row holds
    assert bool(call(gate_up.masked_fill(of_row[:, None], NAN), w)["d_topk_w"][zero].isnan().all())
