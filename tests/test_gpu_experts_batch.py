"""The experts' products for whole batches on the GPU -- grouped products and their gradients, SwiGLU forward and backward,
the combination of a token's experts -- against 64-bit torch.

Tolerances.  Operands are bf16, so products of two are exact in fp32.  A product of K terms is accumulated in fp32 in
steps of 16 terms; a step adds with an error of at most one unit in the last place (2^-23: truncation rather than rounding is
allowed for) of a running sum that is bounded by A = sum |a b|, and so does the sum of its own 16 terms:
|error| <= (2 K / 16 + 2) 2^-23 A, and the root mean square over elements, whose running sums are no larger than the final ones
in the mean, at most (2 K / 16 + 2) 2^-23 times that of the results.  A bf16 output is rounded once more, by at most half a step:
2^-8 of its value."""
import pytest
import torch

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
NAN, INF = float("nan"), float("inf")
STEP = 2.0 ** -23
BAD_OFFSETS, BAD_ROW = 6, 7


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


def offsets_of(counts, first=0):
    at = [first]
    for c in counts:
        at.append(at[-1] + c)
    return torch.tensor(at, dtype=torch.int32, device="cuda")


def check(got, want, size, K, where=None):
    """``size``: the sums of absolute values behind ``want``."""
    out = 2.0 ** -8 if got.dtype is BF16 else 0.0
    acc = (2 * K / 16 + 2) * STEP
    err = (got.double() - want).abs()
    tol = acc * size + out * want.abs() + 1e-37
    if where is not None:
        err, tol, want = err[where], tol[where], want[where]
    assert bool((err <= tol).all()), float((err / tol).max())
    if want.numel() > 1000:
        rms = lambda x: float(x.pow(2).mean().sqrt())  # noqa: E731
        assert rms(err) <= (acc + out) * rms(want) + 1e-37


def wide(t, pad, shift=0):
    """The matrix with ``pad`` columns of NaN behind each row, ``shift`` rows of NaN in front and behind."""
    buf = torch.full((t.shape[0] + 2 * shift, t.shape[1] + pad), NAN, dtype=t.dtype, device=t.device)
    view = buf[shift:shift + t.shape[0], :t.shape[1]]
    view.copy_(t)
    return view


def groups(counts, first=0):
    at = first
    for e, c in enumerate(counts):
        if c:
            yield e, slice(at, at + c)
        at += c


# group sizes: none at all, single rows, runs of empty groups, sizes around a tile's columns (64 / 256) and a block's rows (64)
COUNTS = [[0], [1], [3, 0, 1, 0, 0, 17, 2], [15, 16, 17, 31, 32, 33], [64, 65, 63, 0, 129, 128, 127],
          [255, 0, 256, 257, 1], [700], [0, 0, 1111, 0, 300, 513]]


@pytest.mark.parametrize("counts", COUNTS)
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("n,k", [(8, 8), (264, 136), (136, 264), (1000, 520)])
def test_grouped_products(dx, counts, transposed, n, k):
    """Every form of rows: in place and gathered, written in order and scattered, bf16 and fp32, pitches wider than the rows,
    rows in front of the first group and behind the last (which hold NaN and are left as they were)."""
    binding, ctx = dx
    g = rng(n + k + sum(counts))
    E, first, live = len(counts), 5, sum(counts)
    P = first + live + 7
    off = offsets_of(counts, first)
    n_in, n_out = (n, k) if transposed else (k, n)
    w = torch.full((E, n, k + 16), NAN, dtype=BF16, device="cuda")[:, :, :k]
    w.copy_(draw(g, E, n, k, scale=0.2))
    for gathered, scatter, dtype in ((False, False, BF16), (True, False, F32), (False, True, F32), (True, True, BF16)):
        rows = draw(g, P, n_in)
        rows[:first] = NAN
        rows[first + live:] = NAN
        x, index, div = wide(rows, 8, 3), None, 1
        if gathered:      # rows anywhere in a larger matrix, the same one for several
            div = 3
            source = draw(g, 50, n_in)
            index = torch.randint(0, 150, (P,), generator=g, device="cuda", dtype=torch.int32)
            rows, x = source[(index // 3).long()], wide(source, 24)
        to = torch.randperm(P, generator=g, device="cuda").to(torch.int32) if scatter else None
        y = torch.full((P, n_out + 8), 77.0, dtype=dtype, device="cuda")[:, :n_out]
        got = binding.moe_grouped_mm(ctx, x, w, off, transposed=transposed, gather=index, gather_div=div, scatter=to, out=y)
        assert got is y
        want, size = torch.zeros((P, n_out), dtype=torch.float64, device="cuda"), torch.zeros((P, n_out), dtype=torch.float64, device="cuda")
        inside = torch.zeros(P, dtype=torch.bool, device="cuda")
        for e, here in groups(counts, first):
            m = w[e].double() if transposed else w[e].double().t()
            want[here], size[here] = rows[here].double() @ m, rows[here].double().abs() @ m.abs()
            inside[here] = True
        sorted_got = y[to.long()] if scatter else y
        check(sorted_got, want, size, n_in, inside)
        assert bool((sorted_got[~inside] == 77.0).all())
        assert bool((y.as_strided((P, 8), (n_out + 8, 1), n_out) == 77.0).all())      # (the columns behind the rows)
        again = binding.moe_grouped_mm(ctx, x, w, off, transposed=transposed, gather=index, gather_div=div, scatter=to,
                                       out_dtype=dtype)
        if scatter:
            again = again[to.long()]
        assert torch.equal(again[inside], sorted_got[inside])


@pytest.mark.parametrize("counts", COUNTS)
@pytest.mark.parametrize("n,k", [(8, 8), (264, 136), (1000, 520)])
def test_gradient_of_the_groups_matrices(dx, counts, n, k):
    """Rows in place and gathered, either operand; groups whose rows end inside a block of 64; rows outside the groups hold NaN
    and infinities; empty groups get zeros; columns behind the matrices' rows stay."""
    binding, ctx = dx
    g = rng(n + 2 * k + sum(counts))
    E, first, live = len(counts), 3, sum(counts)
    P = first + live + 70
    off = offsets_of(counts, first)
    for gather_dy, gather_x, dtype in ((False, False, F32), (True, False, BF16), (False, True, F32), (True, True, BF16)):
        mats, args = [], {}
        for name, cols, gathered in (("dy", n, gather_dy), ("x", k, gather_x)):
            rows = draw(g, P, cols)
            rows[:first] = NAN
            rows[first + live:] = INF
            if gathered:
                source = draw(g, 41, cols)
                index = torch.randint(0, 82, (P,), generator=g, device="cuda", dtype=torch.int32)
                args["gather_" + name], args[name + "_div"] = index, 2
                mats.append((source[(index // 2).long()], wide(source, 8)))
            else:
                mats.append((rows, wide(rows, 16, 2)))
        dw = torch.full((E, n, k + 8), 55.0, dtype=dtype, device="cuda")[:, :, :k]
        got = binding.moe_grouped_mm_dw(ctx, mats[0][1], mats[1][1], off, out=dw, **args)
        want = torch.zeros((E, n, k), dtype=torch.float64, device="cuda")
        size = torch.zeros_like(want)
        for e, here in groups(counts, first):
            a, b = mats[0][0][here].double(), mats[1][0][here].double()
            want[e], size[e] = a.t() @ b, a.abs().t() @ b.abs()
        check(got, want, size, max(counts + [16]))
        assert bool((dw.as_strided((E * n, 8), (k + 8, 1), k) == 55.0).all())
        again = binding.moe_grouped_mm_dw(ctx, mats[0][1], mats[1][1], off, out_dtype=dtype, **args)
        assert torch.equal(again, got)


def routed(g, N, k, E):
    ids = torch.randn((N, E), generator=g, device="cuda").topk(k, dim=1).indices.reshape(-1)
    perm = torch.sort(ids, stable=True).indices.to(torch.int32)
    counts = torch.bincount(ids, minlength=E).tolist()
    return perm, counts


@pytest.mark.parametrize("N,k,E,H,I", [(1, 2, 5, 64, 8), (7, 3, 9, 136, 40), (40, 8, 8, 264, 136), (333, 2, 3, 520, 200),
                                       (1000, 6, 64, 256, 352), (1500, 4, 64, 64, 600), (1000, 6, 64, 64, 1416),
                                       (300, 8, 100, 64, 328)])     # (the last three: tiles of no lanes between others)
def test_swiglu_forward_and_backward(dx, N, k, E, H, I):
    """act and gate_up from the same fp32 products; the gradients from what was kept.  sigmoid is good to 2^-20 relative: 1 +
    ex2 and rcp 2^-22 each, the argument's rounding 2^-24 |x| with |x| below 8."""
    binding, ctx = dx
    g = rng(N + H)
    P = N * k
    perm, counts = routed(g, N, k, E)
    off, pairs = offsets_of(counts), perm.long()
    w, x = draw(g, E, 2 * I, H, scale=1.5 * H ** -0.5), draw(g, N, H)
    gu, size = torch.zeros((P, 2 * I), dtype=torch.float64, device="cuda"), torch.zeros((P, 2 * I), dtype=torch.float64, device="cuda")
    rows = x[pairs // k].double()
    for e, here in groups(counts):
        gu[here], size[here] = rows[here] @ w[e].double().t(), rows[here].abs() @ w[e].double().abs().t()
    got = binding.moe_grouped_swiglu(ctx, wide(x, 8, 1), w, off, gather=perm, gather_div=k, save=True)
    alone = binding.moe_grouped_swiglu(ctx, x, w, off, gather=perm, gather_div=k)
    assert set(alone) == {"act"} and torch.equal(alone["act"], got["act"])
    in_place = binding.moe_grouped_swiglu(ctx, x[pairs // k].contiguous(), w, off, save=True)
    assert torch.equal(in_place["act"], got["act"]) and torch.equal(in_place["gate_up"], got["gate_up"])
    check(got["gate_up"], gu, size, H)
    gate, up = gu[:, :I], gu[:, I:]
    s = torch.sigmoid(gate)
    act = gate * s * up
    acc = (2 * H / 16 + 2) * STEP
    # |d act| <= |up| |silu'| |d gate| + |silu| |d up| + ..., |silu'| <= 1.1
    tol = acc * (1.1 * up.abs() * size[:, :I] + (gate * s).abs() * size[:, I:]) + (2.0 ** -8 + 2.0 ** -18) * act.abs() + 1e-37
    assert bool(((got["act"].double() - act).abs() <= tol).all())

    # backward: through a down matrix, from a gradient of the tokens' sums
    wd, dy = draw(g, E, H, I, scale=H ** -0.5), draw(g, N, H)
    topk_w = torch.rand((N, k), generator=g, device="cuda") + 0.1
    topk_w.view(-1)[::5] = 0.0
    gate_up = got["gate_up"].clone()
    dead = topk_w.reshape(-1)[pairs] == 0
    gate_up[dead] = NAN                                    # a pair of weight 0 is taken out, whatever its row holds
    back = binding.moe_grouped_swiglu_backward(ctx, dy, wd, wide(gate_up, 8, 2), topk_w, off, gather=perm, gather_div=k)
    a, a_size = torch.zeros((P, I), dtype=torch.float64, device="cuda"), torch.zeros((P, I), dtype=torch.float64, device="cuda")
    rows = dy[pairs // k].double()
    for e, here in groups(counts):
        a[here], a_size[here] = rows[here] @ wd[e].double(), rows[here].abs() @ wd[e].double().abs()
    gate, up = got["gate_up"].double()[:, :I], got["gate_up"].double()[:, I:]
    s = torch.sigmoid(gate)
    wt = topk_w.double().reshape(-1)[pairs][:, None]
    slope = s * (1 + gate * (1 - s))
    near = 2.0 ** -8 + 2.0 ** -18
    want = torch.cat([wt * a * up * slope, wt * a * gate * s], 1)
    # (1 - s loses what s is off by, 2^-20, times |gate|)
    loose = torch.cat([wt * a.abs() * up.abs() * (gate.abs() + 1) * 2.0 ** -19, torch.zeros_like(a)], 1)
    tol = near * want.abs() + loose + acc * torch.cat([wt * a_size * (up * slope).abs(), wt * a_size * (gate * s).abs()], 1) + 1e-37
    assert bool(((back["d_gate_up"].double() - want).abs() <= tol).all())
    act = gate * s * up
    assert bool(((back["act_w"].double() - wt * act).abs() <= near * (wt * act).abs() + 1e-37).all())
    d_w = torch.zeros(P, dtype=torch.float64, device="cuda").index_copy_(0, pairs, torch.where(dead, 0.0, (a * act).sum(1)))
    bound = torch.zeros(P, dtype=torch.float64, device="cuda").index_copy_(
        0, pairs, ((acc * a_size + (2.0 ** -18 + I * STEP) * a.abs()) * act.abs()).sum(1))
    assert bool(((back["d_topk_w"].double().reshape(-1) - d_w).abs() <= bound + 1e-37).all())
    assert not back["d_gate_up"][dead].any() and not back["act_w"][dead].any()
    # without weights: all 1, and no gradient of them
    ones = binding.moe_grouped_swiglu_backward(ctx, dy, wd, got["gate_up"], torch.ones_like(topk_w), off, gather=perm, gather_div=k)
    none = binding.moe_grouped_swiglu_backward(ctx, dy, wd, got["gate_up"], None, off, gather=perm, gather_div=k)
    assert set(none) == {"d_gate_up", "act_w"} and torch.equal(none["d_gate_up"], ones["d_gate_up"])
    assert torch.equal(none["act_w"], ones["act_w"])


def test_swiglu_gradient_against_differences(dx):
    """The gradient of L = sum dy . (sum_j w_j W_d act_j) with respect to gate and up, by central differences in 64 bits."""
    binding, ctx = dx
    g = rng(5)
    N, k, E, H, I = 6, 2, 3, 64, 24
    perm, counts = routed(g, N, k, E)
    off, pairs = offsets_of(counts), perm.long()
    wd, dy, gu = draw(g, E, H, I, scale=0.2), draw(g, N, H), draw(g, N * k, 2 * I, scale=2.0)
    topk_w = torch.rand((N, k), generator=g, device="cuda") + 0.2
    back = binding.moe_grouped_swiglu_backward(ctx, dy, wd, gu, topk_w, off, gather=perm, gather_div=k)
    of_row = torch.repeat_interleave(torch.arange(E, device="cuda"), torch.tensor(counts, device="cuda"))

    def per_pair(gate_up):
        gate, up = gate_up.chunk(2, dim=1)
        z = torch.einsum("rhi,ri->rh", wd.double()[of_row], gate / (1 + torch.exp(-gate)) * up)
        return (z * dy.double()[pairs // k]).sum(1)

    weight = topk_w.double().reshape(-1)[pairs]
    h = 1e-5
    for col in range(2 * I):
        step = torch.zeros_like(gu, dtype=torch.float64)
        step[:, col] = h
        slope = weight * (per_pair(gu.double() + step) - per_pair(gu.double() - step)) / (2 * h)
        # bf16 output; differences good to h^2 and 1e-16 / h, relative to gradients of order 1
        assert bool(((back["d_gate_up"][:, col].double() - slope).abs() <= 2.0 ** -8 * slope.abs() + 1e-4).all())
    d_w = torch.zeros(N * k, dtype=torch.float64, device="cuda").index_copy_(0, pairs, per_pair(gu.double()))
    assert bool(((back["d_topk_w"].double().reshape(-1) - d_w).abs() <= 1e-4 * d_w.abs().max()).all())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N,k,H", [(1, 1, 8), (3, 8, 64), (130, 6, 520), (2100, 3, 264), (50, 5, 4104)])
def test_combination_and_its_gradient(dx, dtype, N, k, H):
    """Sums of k products in fp32, each a rounding (2^-24) off, rounded once; rows of weight 0 hold NaN."""
    binding, ctx = dx
    g = rng(N + H)
    z = torch.randn((N * k, H), generator=g, device="cuda").to(dtype)
    w = torch.rand((N, k), generator=g, device="cuda") + 0.1
    w.view(-1)[1::4] = 0.0
    zz = z.double().view(N, k, H).masked_fill(w[:, :, None] == 0, 0.0)
    z = z.masked_fill(w.reshape(-1, 1) == 0, NAN)
    half = {BF16: 2.0 ** -8, F32: 2.0 ** -24}
    want, size = (zz * w.double()[:, :, None]).sum(1), (zz.abs() * w.double()[:, :, None]).sum(1)
    for out in (BF16, F32):
        y = binding.moe_combine_tokens(ctx, wide(z, 8), w, out_dtype=out)
        assert y.dtype is out
        assert bool(((y.double() - want).abs() <= half[out] * want.abs() + (k + 1) * 2.0 ** -24 * size).all())
    clean = torch.randn((N * k, H), generator=g, device="cuda").to(dtype)
    plain = binding.moe_combine_tokens(ctx, clean, None, top_k=k)
    total = clean.double().view(N, k, H).sum(1)
    assert bool(((plain.double() - total).abs() <= half[dtype] * total.abs() +
                 k * 2.0 ** -24 * clean.double().view(N, k, H).abs().sum(1)).all())
    dy = torch.randn((N, H), generator=g, device="cuda").to(dtype)
    back = binding.moe_combine_tokens_backward(ctx, wide(dy, 8), wide(z, 16), w)
    want = (dy.double()[:, None] * w.double()[:, :, None]).reshape(-1, H)
    assert bool(((back["dz"].double() - want).abs() <= (half[dtype] + 2.0 ** -24) * want.abs()).all())
    want, size = (zz * dy.double()[:, None]).sum(2), (zz * dy.double()[:, None]).abs().sum(2)
    assert bool(((back["d_topk_w"].double() - want).abs() <= (H / 8 + 16) * 2.0 ** -24 * size).all())
    assert not back["d_topk_w"][w == 0].any() and not back["dz"][w.reshape(-1) == 0].any()
    only = binding.moe_combine_tokens_backward(ctx, dy, None, w, out={"dz": torch.empty_like(z)})["dz"]
    assert torch.equal(only, back["dz"])
    only = binding.moe_combine_tokens_backward(ctx, dy, z, w, out={"d_topk_w": torch.empty_like(w)})["d_topk_w"]
    assert torch.equal(only, back["d_topk_w"])


def test_bad_rows_and_offsets_are_reported_and_harmless(dx):
    """Indexes outside their matrix read zeros and write nothing; offsets are cut to the rows there are."""
    binding, ctx = dx
    g = rng(9)
    w, x = draw(g, 3, 72, 64, scale=0.2), draw(g, 10, 64)
    off = offsets_of([4, 0, 6])
    index = torch.tensor([0, 3, -1, 9, 10, 2 ** 31 - 1, -2 ** 31, 5, 6, 7], dtype=torch.int32, device="cuda")
    bad = [2, 4, 5, 6]
    good = [i for i in range(10) if i not in bad]
    y = binding.moe_grouped_mm(ctx, x, w, off, gather=index, out_dtype=F32)
    assert ctx.device_status() == BAD_ROW and ctx.device_status() == 0
    assert not y[bad].any() and bool(y[good].any(dim=1).all())
    y = torch.full((10, 72), 9.0, device="cuda")
    binding.moe_grouped_mm(ctx, x, w, off, scatter=index, out=y)
    assert ctx.device_status() == BAD_ROW and ctx.device_status() == 0
    assert bool((y[[1, 2, 4, 8]] == 9.0).all()) and not bool((y[[0, 3, 9, 5, 6, 7]] == 9.0).any())
    dw = binding.moe_grouped_mm_dw(ctx, draw(g, 10, 72), x, off, gather_x=index, out_dtype=F32)
    assert ctx.device_status() == BAD_ROW and ctx.device_status() == 0
    assert bool(torch.isfinite(dw).all()) and not dw[1].any()
    gu, dy = draw(g, 10, 48), draw(g, 10, 72)
    wd = draw(g, 3, 72, 24)
    back = binding.moe_grouped_swiglu_backward(ctx, dy, wd, gu, torch.ones(10, device="cuda"), off, gather=index)
    assert ctx.device_status() == BAD_ROW and ctx.device_status() == 0
    assert not back["act_w"][bad].any() and bool(torch.isfinite(back["d_gate_up"]).all())
    # offsets that descend, are negative or go past the rows
    for values in ([0, 8, 4, 10], [-5, 3, 6, 10], [0, 4, 4, 2 ** 31 - 1], [-2 ** 31, -1, 50, 7]):
        y = binding.moe_grouped_mm(ctx, x, w, torch.tensor(values, dtype=torch.int32, device="cuda"), out_dtype=F32)
        assert ctx.device_status() == BAD_OFFSETS and ctx.device_status() == 0
        dw = binding.moe_grouped_mm_dw(ctx, dy, x, torch.tensor(values, dtype=torch.int32, device="cuda"), out_dtype=F32)
        assert ctx.device_status() == BAD_OFFSETS and ctx.device_status() == 0
        assert bool(torch.isfinite(dw).all())


def test_rows_past_two_to_the_31_elements(dx):
    """Outputs and inputs whose elements pass 32-bit positions: the last rows are right."""
    binding, ctx = dx
    g = rng(11)
    P, n, k = 540000, 4000, 64
    assert P * n > 2 ** 31
    w, x = draw(g, 2, n, k), draw(g, 1000, k)
    off = torch.tensor([0, P - 300, P], dtype=torch.int32, device="cuda")
    index = (torch.arange(P, device="cuda") % 1000).to(torch.int32)
    y = binding.moe_grouped_mm(ctx, x, w, off, gather=index)
    rows = torch.tensor([0, 1, P // 2, P - 301, P - 300, P - 1], device="cuda")
    for r in rows.tolist():
        want = w[int(r >= P - 300)].double() @ x[r % 1000].double()
        assert bool(((y[r].double() - want).abs() <= 2.0 ** -8 * want.abs() + 1e-4).all())
    # back through them: [n, k] from rows at the far end of y, and y as the operand of another product
    dw = binding.moe_grouped_mm_dw(ctx, y, x, torch.tensor([P - 100, P], dtype=torch.int32, device="cuda"), gather_x=index,
                                   out_dtype=F32)
    want = y[P - 100:].double().t() @ x[index[P - 100:].long()].double()
    assert float((dw[0].double() - want).norm() / want.norm()) <= 20 * STEP
    z = binding.moe_grouped_mm(ctx, y, w[:1], torch.tensor([P - 100, P], dtype=torch.int32, device="cuda"), transposed=True,
                               out=torch.empty((P, k), device="cuda"))
    want = y[P - 100:].double() @ w[0].double()
    assert float((z[P - 100:].double() - want).norm() / want.norm()) <= (2 * n / 16 + 2) * STEP


def test_streams_graphs_and_contexts(dx):
    """The same bits on another stream, replayed from a graph on other inputs, from two graphs of one context at once."""
    binding, ctx = dx
    g = rng(13)
    N, k, E, H, I = 300, 4, 12, 256, 136

    def state(seed):
        g = rng(seed)
        perm, counts = routed(g, N, k, E)
        return {"x": draw(g, N, H), "w": draw(g, E, 2 * I, H, scale=0.1), "wd": draw(g, E, H, I, scale=0.1), "dy": draw(g, N, H),
                "perm": perm, "off": offsets_of(counts), "tw": torch.rand((N, k), generator=g, device="cuda")}

    def step(s):
        f = binding.moe_grouped_swiglu(ctx, s["x"], s["w"], s["off"], gather=s["perm"], gather_div=k, save=True)
        z = binding.moe_grouped_mm(ctx, f["act"], s["wd"], s["off"], scatter=s["perm"])
        y = binding.moe_combine_tokens(ctx, z, s["tw"])
        b = binding.moe_grouped_swiglu_backward(ctx, s["dy"], s["wd"], f["gate_up"], s["tw"], s["off"], gather=s["perm"],
                                                gather_div=k)
        dw = binding.moe_grouped_mm_dw(ctx, b["d_gate_up"], s["x"], s["off"], gather_x=s["perm"], x_div=k)
        dwd = binding.moe_grouped_mm_dw(ctx, s["dy"], b["act_w"], s["off"], gather_dy=s["perm"], dy_div=k, out_dtype=F32)
        dz = binding.moe_grouped_mm(ctx, b["d_gate_up"], s["w"], s["off"], transposed=True, scatter=s["perm"])
        return [f["act"], y, b["d_topk_w"], dw, dwd, binding.moe_combine_tokens(ctx, dz, None, top_k=k)]

    a, b = state(1), state(2)
    want = {id(a): [t.clone() for t in step(a)], id(b): [t.clone() for t in step(b)]}
    same = lambda got, s: all(torch.equal(p, q) for p, q in zip(got, want[id(s)]))  # noqa: E731
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = step(a)
    torch.cuda.synchronize()
    assert same(got, a)
    held = [{k_: v.clone() for k_, v in a.items()} for _ in range(2)]
    graphs, outs = [], []
    for s in held:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(step(s))
        graphs.append(graph)
    for first, second in ((a, b), (b, a), (a, a)):
        for s, src in zip(held, (first, second)):
            for key in s:
                s[key].copy_(src[key])
        torch.cuda.synchronize()
        for graph, stream in zip(graphs, (side, torch.cuda.Stream())):
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        assert same(outs[0], first) and same(outs[1], second)
    del graphs


def test_nothing_to_do(dx):
    binding, ctx = dx
    w = torch.zeros((3, 16, 32), dtype=BF16, device="cuda")
    off = torch.zeros(4, dtype=torch.int32, device="cuda")
    x = torch.zeros((0, 32), dtype=BF16, device="cuda")
    assert binding.moe_grouped_mm(ctx, x, w, off).shape == (0, 16)
    assert binding.moe_grouped_swiglu(ctx, x, w, off, save=True)["gate_up"].shape == (0, 16)
    dw = binding.moe_grouped_mm_dw(ctx, torch.zeros((0, 16), dtype=BF16, device="cuda"), x, off,
                                   out=torch.full((3, 16, 40), 3.0, device="cuda")[:, :, :32])
    assert not dw.any() and dw.shape == (3, 16, 32)
    assert binding.moe_combine_tokens(ctx, x, torch.zeros((0, 4), device="cuda")).shape == (0, 32)
    # groups, but no rows in them
    x = torch.full((70, 32), NAN, dtype=BF16, device="cuda")
    y = binding.moe_grouped_mm(ctx, x, w, off, out=torch.full((70, 16), 2.0, device="cuda"))
    assert bool((y == 2.0).all())
    assert not binding.moe_grouped_mm_dw(ctx, torch.full((70, 16), NAN, dtype=BF16, device="cuda"), x, off).any()


def test_refusals(dx):
    binding, ctx = dx
    w = torch.zeros((3, 16, 32), dtype=BF16, device="cuda")
    x = torch.zeros((8, 32), dtype=BF16, device="cuda")
    off = torch.zeros(4, dtype=torch.int32, device="cuda")
    idx = torch.zeros(8, dtype=torch.int32, device="cuda")
    mm = lambda **a: binding.moe_grouped_mm(ctx, **{**dict(x=x, w=w, offsets=off), **a})  # noqa: E731
    for bad in (dict(x=x.float()), dict(x=x.cpu()), dict(x=x[:, ::2]), dict(x=x[:, :24]), dict(w=w.float()), dict(w=w[0]),
                dict(w=w.transpose(1, 2)), dict(offsets=off.long()), dict(offsets=off[:3]), dict(gather=idx.long()),
                dict(scatter=idx[:5]), dict(out_dtype=torch.float16), dict(out=torch.zeros((8, 24), device="cuda"))):
        with pytest.raises(ValueError):
            mm(**bad)
    wide_x = torch.zeros((8, 36), dtype=BF16, device="cuda")
    for bad, status in ((dict(x=wide_x[:, :32]), 8), (dict(x=torch.zeros(8 * 32 + 4, dtype=BF16, device="cuda")[4:].view(8, 32)), 1),
                        (dict(gather=idx, gather_div=0), 1), (dict(out=x.new_zeros((7, 16))), 2),
                        (dict(w=w[:, :12]), 8), (dict(w=w.new_zeros((257, 8, 32)), offsets=torch.zeros(258, dtype=torch.int32, device="cuda")), 8),
                        (dict(w=w.new_zeros((3, 32, 32)), out=x), 1)):
        with pytest.raises(binding.DxError) as err:
            mm(**bad)
        assert err.value.status == status, bad
    with pytest.raises(binding.DxError) as err:
        binding.moe_grouped_swiglu(ctx, x, w[:, :8], off)            # (four gate rows)
    assert err.value.status == 8
    with pytest.raises(ValueError):
        binding.moe_grouped_mm_dw(ctx, x, x[:4], off)
    with pytest.raises(ValueError):
        binding.moe_grouped_swiglu_backward(ctx, x, w.transpose(1, 2).contiguous(), x[:4], None, off)
    with pytest.raises(ValueError):
        binding.moe_combine_tokens(ctx, x, torch.zeros((3, 2), device="cuda"))
    with pytest.raises(binding.DxError) as err:
        binding.moe_combine_tokens(ctx, x.repeat(9, 1)[:9], None, top_k=9)
    assert err.value.status == 8


@pytest.mark.parametrize("E,mean", [(256, 9), (150, 60), (70, 200)])
@pytest.mark.parametrize("transposed", [False, True])
def test_many_tiles_one_after_another(dx, E, mean, transposed):
    """Each block of the grid has several tiles, full ones and others, of groups of very different lengths, empty ones among them."""
    binding, ctx = dx
    g = rng(E + mean)
    counts = (torch.rand(E, generator=g, device="cuda") ** 2 * 3 * mean).int().tolist()
    counts[3] = counts[E - 2] = 0
    n, k, P = 328, 264, sum(counts)
    n_in, n_out = (n, k) if transposed else (k, n)
    off = offsets_of(counts)
    w, source = draw(g, E, n, k, scale=0.2), draw(g, 501, n_in)
    index = torch.randint(0, 1002, (P,), generator=g, device="cuda", dtype=torch.int32)
    to = torch.randperm(P, generator=g, device="cuda").to(torch.int32)
    rows = source[(index // 2).long()]
    want, size = (torch.zeros((P, n_out), dtype=torch.float64, device="cuda") for _ in range(2))
    for e, here in groups(counts):
        m = w[e].double() if transposed else w[e].double().t()
        want[here], size[here] = rows[here].double() @ m, rows[here].double().abs() @ m.abs()
    for dtype in (BF16, F32):
        y = binding.moe_grouped_mm(ctx, source, w, off, transposed=transposed, gather=index, gather_div=2, scatter=to, out_dtype=dtype)
        check(y[to.long()], want, size, n_in)
        z = binding.moe_grouped_mm(ctx, rows, w, off, transposed=transposed, out_dtype=dtype)
        assert torch.equal(z, y[to.long()])
    if transposed:
        return
    dy = draw(g, P, n)
    dw, dw_size = (torch.zeros((E, n, k), dtype=torch.float64, device="cuda") for _ in range(2))
    for e, here in groups(counts):
        a, b = dy[here].double(), rows[here].double()
        dw[e], dw_size[e] = a.t() @ b, a.abs().t() @ b.abs()
    got = binding.moe_grouped_mm_dw(ctx, dy, source, off, gather_x=index, x_div=2, out_dtype=F32)
    check(got, dw, dw_size, max(counts))


def test_results_do_not_depend_on_the_overlap_of_launches(dx):
    """A chain of calls, each reading what the one in front wrote, with and without launches that start early: the same bits."""
    binding, ctx = dx
    g = rng(77)
    E, H, I, N, k = 16, 264, 136, 130, 3
    perm, counts = routed(g, N, k, E)
    off, x = offsets_of(counts), draw(g, N, H)
    wg, wd = draw(g, E, 2 * I, H, scale=0.1), draw(g, E, H, I, scale=0.1)
    topk_w = torch.rand((N, k), generator=g, device="cuda")

    def chain():
        act = binding.moe_grouped_swiglu(ctx, x, wg, off, gather=perm, gather_div=k)["act"]
        y = binding.moe_grouped_mm(ctx, act, wd, off, scatter=perm)
        return act, y, binding.moe_combine_tokens(ctx, y, topk_w)

    ctx.set_launch_overlap(0)
    plain = chain()
    ctx.set_launch_overlap(3)
    for _ in range(20):
        assert all(torch.equal(a, b) for a, b in zip(chain(), plain))


def test_a_long_contraction_is_no_wait_that_ran_out(dx):
    """One group of two million rows: its only tile's products take several times as long as the context lets a kernel wait."""
    binding, ctx = dx
    ctx.set_wait_limit(1 << 15)
    g, P = rng(5), (1 << 21) + 5
    dy, x = draw(g, P, 8), draw(g, P, 16)
    got = binding.moe_grouped_mm_dw(ctx, dy, x, offsets_of([P]), out_dtype=F32)
    assert ctx.device_status() == 0
    check(got[0], dy.double().t() @ x.double(), dy.double().abs().t() @ x.double().abs(), P)
