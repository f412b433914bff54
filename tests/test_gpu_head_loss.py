"""Cross entropy of hidden rows against a vocabulary (``spec_head_loss``) on the GPU against 64-bit torch, and a training
step through router, experts, combination and loss.

Tolerances.  A logit is a product of H terms in fp32: off by at most (2 H / 16 + 2) 2^-23 sum |h w| =: Z (see the grouped
products' tests).  The loss is a difference of two such plus the logarithm of a sum of exponentials that are good to 2^-21 each
(ex2 2^-22, the argument's two roundings 2^-24 of at most 40) and added up with at most 2^-24 per addition, of which a
term sees fewer than 200: 2 Z + 2^-16.  A probability is therefore good to the same relative error, and an element of dz, rounded
to bf16, to half a step more: 2^-8 + 2 Z + 2^-16 =: D.  dh and dW sum such elements: |error| <= D sum |dz w| + 2^-8 |result| plus
their own products' error, which is smaller than what D leaves."""
import pytest
import torch

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
NAN = float("nan")
BAD_TOKEN = 5


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


def problem(seed, N, V, H, ragged=True):
    g = rng(seed)
    W = (torch.randn((V, H), generator=g, device="cuda") * H ** -0.5).to(BF16)
    t = torch.randint(0, V, (N,), generator=g, device="cuda")
    h = (torch.randn((N, H), generator=g, device="cuda") + 8 * torch.rand((N, 1), generator=g, device="cuda") * W[t].float()).to(BF16)
    t, w = t.to(torch.int32), None
    if ragged:
        t[2::5] = -1
        w = torch.rand((N,), generator=g, device="cuda") + 0.5
        w[N - N // 4:] = 0.0
    return h, W, t, w


def reference(h, W, t, w):
    """loss, dz, which rows count, and Z."""
    z = h.double() @ W.double().t()
    Z = (2 * h.shape[1] / 16 + 2) * 2.0 ** -23 * (h.double().abs() @ W.double().abs().t()).max(dim=1).values
    logp = torch.log_softmax(z, 1)
    live = t >= 0
    scale = torch.ones_like(z[:, 0]) if w is None else w.double()
    live = live & (scale != 0)
    at = t.long().clamp(min=0)[:, None]
    loss = torch.where(live, -logp.gather(1, at)[:, 0], 0.0)
    d = logp.exp()
    d.scatter_add_(1, at, torch.full_like(at, -1.0, dtype=torch.float64))
    return loss, d * torch.where(live, scale, 0.0)[:, None], live, Z


def check(h, W, t, w, out):
    loss, dz, live, Z = reference(torch.where(torch.isfinite(h), h, torch.zeros_like(h)), W, t, w)
    assert bool(((out["loss"].double() - loss).abs() <= torch.where(live, 2 * Z + 2.0 ** -16 + 2.0 ** -23 * loss, 0.0)).all())
    D = 2.0 ** -8 + 2 * Z + 2.0 ** -16
    if "dh" in out:
        want, size = dz @ W.double(), (D[:, None] * dz.abs()) @ W.double().abs()
        assert bool(((out["dh"].double() - want).abs() <= size + 2.0 ** -8 * want.abs() + 1e-37).all())
        assert not out["dh"][~live].any()
    if "dW" in out:
        hh = torch.where(live[:, None], h, torch.zeros_like(h)).double()
        want, size = dz.t() @ hh, (D[:, None] * dz.abs()).t() @ hh.abs()
        assert bool(((out["dW"].double() - want).abs() <= size + 2.0 ** -8 * want.abs() + 1e-37).all())


@pytest.mark.parametrize("N,V,H", [(1, 1, 8), (1, 1000, 64), (2, 257, 136), (16, 5003, 256), (33, 4099, 264), (100, 20011, 64),
                                   (128, 3001, 72), (129, 3001, 72), (300, 2003, 520), (777, 9001, 128), (1500, 1000, 64)])
@pytest.mark.parametrize("ragged", [False, True])
def test_loss_and_gradients(dx, N, V, H, ragged):
    """Rows that do not count hold NaN; the loss is the same with and without gradients, bit for bit where the same tiles are
    summed, and everything the same in a second call."""
    binding, ctx = dx
    h, W, t, w = problem(N + V, N, V, H, ragged)
    if ragged:
        h[(t < 0) | (w == 0)] = NAN
    both = binding.spec_head_loss(ctx, h, W, t, row_weight=w, grad_weight=True)
    check(h, W, t, w, both)
    again = binding.spec_head_loss(ctx, h, W, t, row_weight=w, grad_weight=True)
    assert all(torch.equal(both[key], again[key]) for key in both)
    alone = binding.spec_head_loss(ctx, h, W, t, row_weight=w, grad=False)
    assert set(alone) == {"loss"} and torch.equal(alone["loss"], both["loss"])
    rows = binding.spec_head_loss(ctx, h, W, t, row_weight=w)
    assert set(rows) == {"loss", "dh"} and torch.equal(rows["dh"], both["dh"])
    head = binding.spec_head_loss(ctx, h, W, t, row_weight=w, grad=False, grad_weight=True)
    assert torch.equal(head["dW"], both["dW"])


@pytest.mark.parametrize("N,V,H", [(40, 9001, 264), (500, 6007, 128)])
def test_any_workspace_between_the_least_and_the_best(dx, N, V, H):
    binding, ctx = dx
    h, W, t, w = problem(7, N, V, H)
    least, best = binding.spec_head_loss_workspace(ctx, N, V, H)
    assert 0 < least < best
    for bytes_ in (least, least + (best - least) // 3, best - 256, best, best + 4096):
        space = torch.full((bytes_ + 512,), 0xFF, dtype=torch.uint8, device="cuda")      # (as floats: NaN)
        shift = -space.data_ptr() % 256
        out = binding.spec_head_loss(ctx, h, W, t, row_weight=w, grad_weight=True, workspace=space[shift:shift + bytes_])
        check(h, W, t, w, out)
        assert bool((space[shift + bytes_:] == 0xFF).all()) and bool((space[:shift] == 0xFF).all())
    for bad in (torch.empty(least - 256, dtype=torch.uint8, device="cuda"),):
        with pytest.raises(binding.DxError) as err:
            binding.spec_head_loss(ctx, h, W, t, workspace=bad)
        assert err.value.status == 1


def test_rows_none_of_which_counts_and_bad_targets(dx):
    binding, ctx = dx
    h, W, t, _ = problem(3, 70, 900, 64, False)
    dead = torch.full_like(t, -1)
    out = binding.spec_head_loss(ctx, torch.full_like(h, NAN), W, dead, grad_weight=True)
    assert not out["loss"].any() and not out["dh"].any() and not out["dW"].any()
    t[5], t[9], t[11] = 900, -2, 2 ** 31 - 1
    out = binding.spec_head_loss(ctx, h, W, t, grad_weight=True)
    assert ctx.device_status() == BAD_TOKEN and ctx.device_status() == 0
    bad = torch.zeros(70, dtype=torch.bool, device="cuda")
    bad[[5, 9, 11]] = True
    assert bool(out["loss"][bad].isnan().all()) and not out["dh"][bad].any()
    check(h, W, torch.where(bad, -1, t), None, {**out, "loss": torch.where(bad, 0.0, out["loss"])})
    nothing = binding.spec_head_loss(ctx, h[:0], W, t[:0], grad_weight=True)
    assert nothing["loss"].shape == (0,) and not nothing["dW"].any()


def test_confident_rows_keep_their_small_loss(dx):
    """Targets whose logits stand 5 to 14 above all others: losses down to 1e-3.  The loss is (maximum - target's logit) + log(1 +
    rest); the first is exactly 0.  The rest is good to 2^-20 relative; of the fp32 additions of a row's sum, the ones that carry the
    target's term 1 are at most 8 in its sub-sum of 32 words, 2 that join the four sub-sums, and 4 more of its half of the tile
    (the tiles are joined in 64 bits): 14 half steps, 14 * 2^-24 < 2^-20 of the sum, and as much of its logarithm."""
    binding, ctx = dx
    H, V, N = 128, 2000, 64
    W = torch.zeros((V, H), device="cuda")
    W[:H] = torch.eye(H, device="cuda")
    W = W.to(BF16)
    h = torch.zeros((N, H), device="cuda")
    t = torch.arange(N, device="cuda", dtype=torch.int32)
    lift = torch.linspace(5, 14, N, device="cuda").to(BF16).float()
    h[torch.arange(N), t.long()] = lift
    out = binding.spec_head_loss(ctx, h.to(BF16), W, t, grad_weight=True)
    rest = (V - 1) * torch.exp(-lift.double())
    want = torch.log1p(rest)
    assert bool(((out["loss"].double() - want).abs() <= 2.0 ** -20 * want + 2.0 ** -20).all())
    # dW at the target: (p - 1) h, the small difference itself: expm1 of the loss (off by what the loss is off by), rounded to
    # bf16 as dz and again as dW
    grad = out["dW"][t.long(), t.long()].double()
    want_g = -rest / (1 + rest) * lift.double()
    assert bool(((grad - want_g).abs() <= 2 * 2.0 ** -8 * want_g.abs() + 2.0 ** -20 * (1 + want) * lift.double()).all())


def test_gradients_against_differences(dx):
    binding, ctx = dx
    h, W, t, w = problem(17, 5, 300, 64)
    out = binding.spec_head_loss(ctx, h, W, t, row_weight=w, grad_weight=True)

    def total(hh, WW):
        loss, _, live, _ = reference(hh, WW, t, w)
        return float((loss * torch.where(live, w.double(), 0.0)).sum())

    g, eps = rng(3), 1e-5
    for _ in range(20):
        a = torch.randn(h.shape, generator=g, device="cuda", dtype=torch.float64)
        b = torch.randn(W.shape, generator=g, device="cuda", dtype=torch.float64)
        slope = (total(h.double() + eps * a, W.double() + eps * b) - total(h.double() - eps * a, W.double() - eps * b)) / (2 * eps)
        have = float((out["dh"].double() * a).sum() + (out["dW"].double() * b).sum())
        # (bf16 elements, errors of either sign: a few 2^-8 of the direction's size)
        size = float((out["dh"].double() * a).pow(2).sum().sqrt() + (out["dW"].double() * b).pow(2).sum().sqrt())
        assert abs(have - slope) <= 6 * 2.0 ** -8 * size + 1e-5


def test_pitches_streams_and_graphs(dx):
    binding, ctx = dx
    h, W, t, w = problem(23, 90, 3001, 136)
    want = {k: v.clone() for k, v in binding.spec_head_loss(ctx, h, W, t, row_weight=w, grad_weight=True).items()}
    hw = torch.full((90, 200), NAN, dtype=BF16, device="cuda")[:, 8:144]
    Ww = torch.full((3001, 144), NAN, dtype=BF16, device="cuda")[:, :136]
    hw.copy_(h)
    Ww.copy_(W)
    out = {"loss": torch.empty(90, device="cuda"), "dh": torch.full((90, 144), 4.0, dtype=BF16, device="cuda")[:, :136],
           "dW": torch.full((3001, 160), 4.0, dtype=BF16, device="cuda")[:, :136]}
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        binding.spec_head_loss(ctx, hw, Ww, t, row_weight=w, grad_weight=True, out=out)
    torch.cuda.synchronize()
    assert all(torch.equal(out[k], want[k]) for k in want)
    assert bool((out["dW"].as_strided((3001, 24), (160, 1), 136) == 4.0).all())
    # two graphs of one context at once, on other inputs than they were captured with
    held = [(h.clone(), t.clone(), w.clone()) for _ in range(2)]
    graphs, outs = [], []
    for hh, tt, ww in held:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(binding.spec_head_loss(ctx, hh, W, tt, row_weight=ww, grad_weight=True))
        graphs.append(graph)
    h2, _, t2, w2 = problem(29, 90, 3001, 136)
    want2 = {k: v.clone() for k, v in binding.spec_head_loss(ctx, h2, W, t2, row_weight=w2, grad_weight=True).items()}
    held[1][0].copy_(h2), held[1][1].copy_(t2), held[1][2].copy_(w2)
    torch.cuda.synchronize()
    for graph, stream in zip(graphs, (side, torch.cuda.Stream())):
        with torch.cuda.stream(stream):
            graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(outs[0][k], want[k]) and torch.equal(outs[1][k], want2[k]) for k in want)
    del graphs


def test_training_step_of_a_routed_layer(dx):
    """Router, experts, combination and loss forward and backward as a training step runs them, against autograd through the
    same model in 64 bits with the same selection.  Activations and gradients between the operators are bf16: every one of
    the half dozen on the way adds at most 2^-8 relative per element, of either sign: 2 % of each gradient's norm."""
    binding, ctx = dx
    g = rng(31)
    N, H, I, E, k, V = 200, 128, 72, 8, 2, 1000
    draw = lambda *s, scale=1.0: (torch.randn(s, generator=g, device="cuda") * scale).to(BF16)  # noqa: E731
    x, W_r = draw(N, H), draw(E, H, scale=0.2)
    W_gu, W_d, W_lm = draw(E, 2 * I, H, scale=0.15), draw(E, H, I, scale=0.15), draw(V, H, scale=0.1)
    targets = torch.randint(0, V, (N,), generator=g, device="cuda").to(torch.int32)
    targets[-9:] = -1
    weight = torch.full((N,), 1.0 / N, device="cuda")
    # forward
    logits = binding.moe_grouped_mm(ctx, x, W_r[None], torch.tensor([0, N], dtype=torch.int32, device="cuda"), out_dtype=F32)
    route = binding.moe_route_tokens(ctx, logits, k, score_fn=1, routed_scale=1.5)
    off, perm, tw = route["offsets"], route["perm"], route["topk_w"]
    f = binding.moe_grouped_swiglu(ctx, x, W_gu, off, gather=perm, gather_div=k, save=True)
    z = binding.moe_grouped_mm(ctx, f["act"], W_d, off, scatter=perm)
    y = binding.moe_combine_tokens(ctx, z, tw)
    head = binding.spec_head_loss(ctx, y, W_lm, targets, row_weight=weight, grad_weight=True)
    # backward
    b = binding.moe_grouped_swiglu_backward(ctx, head["dh"], W_d, f["gate_up"], tw, off, gather=perm, gather_div=k)
    dW_d = binding.moe_grouped_mm_dw(ctx, head["dh"], b["act_w"], off, gather_dy=perm, dy_div=k, out_dtype=F32)
    dW_gu = binding.moe_grouped_mm_dw(ctx, b["d_gate_up"], x, off, gather_x=perm, x_div=k, out_dtype=F32)
    dx_pairs = binding.moe_grouped_mm(ctx, b["d_gate_up"], W_gu, off, transposed=True, scatter=perm)
    d_x = binding.moe_combine_tokens(ctx, dx_pairs, None, top_k=k, out_dtype=F32)
    d_logits = binding.moe_route_tokens_backward(ctx, logits, route["topk_ids"], b["d_topk_w"], score_fn=1, routed_scale=1.5)
    dW_r = d_logits.t() @ x.float()
    d_x = d_x + d_logits @ W_r.float()
    # 64 bits
    P = [t.double().requires_grad_(True) for t in (x, W_r, W_gu, W_d, W_lm)]
    ids = route["topk_ids"].long()
    r = torch.sigmoid(P[0] @ P[1].t()).gather(1, ids)
    w = 1.5 * r / r.sum(1, keepdim=True)
    gu = torch.einsum("nkih,nh->nki", P[2][ids], P[0])
    act = torch.nn.functional.silu(gu[..., :I]) * gu[..., I:]
    yy = torch.einsum("nk,nkhi,nki->nh", w, P[3][ids], act)
    logp = torch.log_softmax(yy @ P[4].t(), 1)
    live = targets >= 0
    loss = -logp.gather(1, targets.long().clamp(min=0)[:, None])[:, 0] * live
    want = torch.autograd.grad((loss * weight.double()).sum(), P)
    assert float((head["loss"].double() - loss.detach()).abs().max()) <= 0.02 * float(loss.detach().max())
    for name, have, ref in zip(("x", "router", "gate/up", "down", "head"), (d_x, dW_r, dW_gu, dW_d, head["dW"]), want):
        assert float((have.double() - ref).norm()) <= 0.02 * float(ref.norm()), name


def test_a_short_last_piece_leaves_no_block_without_an_end(dx):
    """Many rows, a short hidden row: dz is made in pieces of the vocabulary, the last one shorter, and a piece's words are dealt
    out to many blocks; a block of the last piece that got no words at all would wait for products that nobody issues."""
    binding, ctx = dx
    h, W, t, _ = problem(11, 8192, 34816, 64, False)
    out = binding.spec_head_loss(ctx, h, W, t)
    assert ctx.device_status() == 0
    rows = slice(0, 8192, 97)
    check(h[rows], W, t[rows], None, {key: value[rows] for key, value in out.items()})


@pytest.mark.parametrize("N", [255, 256, 257])
def test_rows_listed_by_their_own_blocks_or_by_one(dx, N):
    binding, ctx = dx
    h, W, t, w = problem(N, N, 1200, 72)
    h[(t < 0) | (w == 0)] = NAN
    check(h, W, t, w, binding.spec_head_loss(ctx, h, W, t, row_weight=w, grad_weight=True))


@pytest.mark.parametrize("N,V", [(400, 50003), (2800, 50003)])
def test_kept_and_recomputed_logits_give_the_same_bits(dx, N, V):
    """Long hidden rows and enough workspace: the logits are kept, in one piece of dz or several; without their bytes the products
    are computed twice."""
    binding, ctx = dx
    H = 1288
    h, W, t, w = problem(N, N, V, H)
    h[(t < 0) | (w == 0)] = NAN
    kept = binding.spec_head_loss(ctx, h, W, t, row_weight=w, grad_weight=True)
    check(h, W, t, w, kept)
    _, best = binding.spec_head_loss_workspace(ctx, N, V, H)
    less = torch.full((best - N * 50176 * 4,), 0xFF, dtype=torch.uint8, device="cuda")
    twice = binding.spec_head_loss(ctx, h, W, t, row_weight=w, grad_weight=True, workspace=less)
    assert all(torch.equal(kept[key], twice[key]) for key in kept)
    check(h, W, t, w, binding.spec_head_loss(ctx, h, W, t, row_weight=w, grad_weight=True, workspace=less[:-4096]))


@pytest.mark.parametrize("N,V,H", [(70, 40009, 1032), (64, 9001, 2048), (600, 12007, 2048)])
def test_larger_heads(dx, N, V, H):
    binding, ctx = dx
    h, W, t, w = problem(N, N, V, H)
    h[(t < 0) | (w == 0)] = NAN
    check(h, W, t, w, binding.spec_head_loss(ctx, h, W, t, row_weight=w, grad_weight=True))
