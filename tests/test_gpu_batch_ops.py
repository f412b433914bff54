"""The batch operators on the GPU against the fp64 checker: token log probabilities with entropy and alternatives,
distillation from a teacher's top log probabilities with its gradient, batch routing and its gradient.

Tolerances, from the arithmetic (u = 2^-24, half a step of fp32):
  * sums of exponentials: ex2.approx is good to 2^-22; its argument carries two roundings, |z - max| / T * log2(e) * 2u
    in the exponent, at most 1.5e-5 relative for terms that fp32 can hold (exponent above -126); a thread adds at most
    about 200 terms per accumulator, 200 u = 1.2e-5.  Together below 3e-5 relative: S_ERR.  Log S is that far off in
    absolute terms, a log probability in addition by the two roundings of (z - max) / T, 2^-23 relative.
  * entropy = log S - (sum u e^u) / S, both terms non-negative and each good to S_ERR relative (the second twice).
  * a gradient is a difference of magnitudes the checker returns; each is good to S_ERR (unlisted part: its own sum of
    exponentials) plus a handful of roundings; a bf16 gradient is rounded once more, 2^-8 relative.  exp results below
    2^-126 are flushed to zero.
  * gates: expf is good to 2^-22, its argument's rounding adds |x| u <= 30 u, a quotient and a product 2u: 5e-6.
Integers (alternatives, selected experts, permutation) are exact."""
import numpy as np
import pytest
import torch

from oracle import batch_oracle as B

pytestmark = pytest.mark.gpu

S_ERR = 3e-5
GATE = 5e-6
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


def rows(values, dtype, pad=0, shift=0, fill=123.0):
    """The matrix on the GPU with ``pad`` extra columns per row, ``shift`` elements into its allocation."""
    N, V = values.shape
    buf = torch.full((N * (V + pad) + shift + 16,), fill, dtype=dtype, device="cuda")
    view = buf[shift:shift + N * (V + pad)].view(N, V + pad)[:, :V]
    view.copy_(values.to(dtype))
    return view


def np64(t):
    return t.detach().to(torch.float64).cpu().numpy()


def draw_logits(seed, N, V, scale=2.0):
    g = torch.Generator().manual_seed(seed)
    z = torch.randn((N, V), generator=g) * scale
    hot = torch.randint(0, V, (N, 5), generator=g)
    return z.scatter_add_(1, hot, torch.rand((N, 5), generator=g) * 12)


# ---- token log probabilities ------------------------------------------------------------------------------------------
def check_logprobs(dx, view, tokens, n_top, T):
    binding, ctx = dx
    tok = None if tokens is None else torch.tensor(tokens, dtype=torch.int32, device="cuda")
    out = binding.spec_token_logprobs(ctx, view, tok, top_n=n_top, temperature=T)
    ref = B.token_logprobs(np64(view), [-1] * view.shape[0] if tokens is None else tokens, n_top, T)
    with np.errstate(over="ignore"):
        for name in ("logprob", "top_logprobs"):           # (what fp32 cannot hold rounds to -inf)
            ref[name] = np.where(np.isinf(ref[name].astype(np.float32)), -np.inf, ref[name])
    if tokens is not None:
        lp, want = np64(out["logprob"]), ref["logprob"]
        same = (lp == want) | (np.isnan(lp) & np.isnan(want))
        with np.errstate(invalid="ignore"):
            assert np.all(same | (np.abs(lp - want) <= S_ERR + 2.0 ** -22 * np.abs(want)))
    ent, want = np64(out["entropy"]), ref["entropy"]
    with np.errstate(invalid="ignore"):
        assert np.all((np.isnan(ent) & np.isnan(want)) | (np.abs(ent - want) <= 2 * S_ERR * (1 + np.abs(want))))
    if n_top:
        assert np.array_equal(out["top_ids"].cpu().numpy(), ref["top_ids"])
        lp, want = np64(out["top_logprobs"]), ref["top_logprobs"]
        same = (lp == want) | (np.isnan(lp) & np.isnan(want))
        with np.errstate(invalid="ignore"):
            assert np.all(same | (np.abs(lp - want) <= S_ERR + 2.0 ** -22 * np.abs(want)))
    return out


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("N,V,pad,shift,n_top,T", [
    (1, 1, 0, 0, 1, 1.0), (3, 2, 0, 1, 2, 1.0), (2, 7, 1, 3, 5, 0.5), (5, 8, 0, 0, 8, 1.0), (4, 9, 0, 1, 9, 1.0),
    (3, 31, 2, 5, 31, 2.0), (2, 64, 0, 2, 32, 1.0), (7, 255, 0, 0, 20, 1.0), (2, 257, 3, 7, 32, 1.3),
    (33, 1000, 0, 0, 8, 1.0), (64, 1024, 8, 0, 20, 1.0), (1, 2048, 0, 1, 5, 1.0), (16, 4099, 0, 3, 20, 0.7),
    (700, 3001, 1, 1, 3, 1.0), (5, 32003, 0, 0, 32, 1.0), (1, 102400, 0, 0, 8, 1.0), (2, 102400, 8, 4, 20, 0.8),
    (1, 163840, 0, 0, 32, 1.0), (3, 163839, 0, 2, 0, 1.0), (1, 400001, 1, 1, 20, 1.0)])
def test_logprobs_small_and_ragged(dx, dtype, N, V, pad, shift, n_top, T):
    view = rows(draw_logits(N + V, N, V), dtype, pad, shift)
    g = torch.Generator().manual_seed(5)
    tokens = torch.randint(-1, V, (N,), generator=g).tolist()
    check_logprobs(dx, view, tokens, n_top, T)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("N,V", [(2, 100), (1, 40000), (320, 40003)])
def test_logprobs_ties_and_crowded_threads(dx, dtype, N, V):
    """Equal rows, rows of two values, and rows whose largest elements all belong to a few threads (more of them than
    the candidate list holds: with 320 rows a row is one CTA's, 16-byte vectors 256 apart are one thread's)."""
    z = torch.zeros((N, V))
    per = 4 if dtype == torch.float32 else 8
    g = torch.Generator().manual_seed(9)
    for t in range(N):
        kind = t % 5 if N > 2 else t
        if kind == 0:
            z[t] = 1.5
        elif kind == 1:
            z[t] = (torch.rand((V,), generator=g) < 0.3).float()
        elif kind == 2:
            z[t, :] = torch.randn((V,), generator=g)
            vec = torch.arange(V) // per
            z[t, (vec % 256) < 8] += 100.0
        elif kind == 3:
            z[t] = torch.arange(V).float() / 64
        else:
            z[t, V - 1] = 0.0
            z[t, : V - 1] = -0.0
    # (with odd V the rows start at other offsets from a vector's border: all the threads of a pattern shift together)
    view = rows(z, dtype)
    if N > 2:
        view = view[:12]
        big = rows(z, dtype)
        from_big = dx[0].spec_token_logprobs(dx[1], big, None, top_n=20)
        ref = B.token_logprobs(np64(view), [-1] * 12, 20, 1.0)
        assert np.array_equal(from_big["top_ids"][:12].cpu().numpy(), ref["top_ids"])
    check_logprobs(dx, view, [0] * view.shape[0], 20, 1.0)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", [40, 5000, 70001])
def test_logprobs_masks_infinities_nan(dx, dtype, V):
    low = torch.finfo(dtype).min
    z = draw_logits(3, 10, V)
    z[0, ::2] = -INF
    z[1, :] = -INF
    z[2, :] = low
    z[3, 1:] = low                   # one word left
    z[4, 1:] = -INF
    z[5, V // 2] = NAN
    z[6, :] = NAN
    z[7, 3] = INF
    z[8, : V // 2] = low
    z[8, V // 2:] = -INF
    z[9, 5] = 3e38                   # far above everything, masks far below
    z[9, 6:] = low
    tokens = [1, 2, V - 1, 0, 0, 1, 1, 1, 0, 5]
    out = check_logprobs(dx, rows(z, dtype, 1, 1), tokens, 8, 1.0)
    assert out["logprob"][1] == -INF and out["entropy"][1] == 0
    assert abs(float(out["logprob"][2]) + np.log(V)) < 1e-4
    assert float(out["logprob"][3]) == 0.0 == float(out["logprob"][4])
    assert torch.isnan(out["logprob"][5:8]).all() and torch.isnan(out["entropy"][5:8]).all()


def test_logprobs_bad_tokens_optional_outputs_and_columns_behind_the_row(dx):
    binding, ctx = dx
    view = rows(draw_logits(4, 4, 300), torch.bfloat16, 20, 0, fill=1e4)      # (columns behind a row hold huge values)
    check_logprobs(dx, view, [299, 0, -1, 5], 4, 1.0)
    check_logprobs(dx, view, None, 4, 1.0)
    out = binding.spec_token_logprobs(ctx, view, torch.tensor([300, -2, 5, -1], dtype=torch.int32, device="cuda"))
    assert torch.isnan(out["logprob"][:2]).all() and not torch.isnan(out["logprob"][2:]).any()
    assert ctx.device_status() == 5 and ctx.device_status() == 0
    empty = binding.spec_token_logprobs(ctx, view[:0], torch.empty((0,), dtype=torch.int32, device="cuda"), top_n=3)
    assert empty["logprob"].shape == (0,)


def test_logprobs_offsets_past_32_bits(dx):
    """Rows that start beyond 2^32 bytes and 2^31 elements of their buffer."""
    binding, ctx = dx
    ld = (1 << 30) + 24
    buf = torch.empty((2 * ld + 5000,), dtype=torch.bfloat16, device="cuda")
    view = buf.as_strided((3, 5000), (ld, 1))
    view.copy_(draw_logits(6, 3, 5000).to(torch.bfloat16))
    check_logprobs(dx, view, [1, 2, 4999], 8, 1.0)
    grad = torch.empty((2 * ld + 5000,), dtype=torch.bfloat16, device="cuda").as_strided((3, 5000), (ld, 1))
    ids = torch.tensor([[1, 7], [2, 3], [4999, 0]], dtype=torch.int32, device="cuda")
    lp = torch.log(torch.full((3, 2), 0.4, device="cuda"))
    a = binding.spec_distill_topk(ctx, view, ids, lp, out={"loss": torch.empty(3, device="cuda"), "dlogits": grad})
    b = binding.spec_distill_topk(ctx, view.contiguous(), ids, lp)
    assert torch.equal(a["loss"], b["loss"]) and torch.equal(grad.contiguous(), b["dlogits"])


# ---- distillation --------------------------------------------------------------------------------------------------------
def teacher_lists(seed, z, k, ragged, T=1.0):
    g = torch.Generator().manual_seed(seed)
    N, V = z.shape
    k_eff = min(k, V)
    t = torch.log_softmax(z.float() / T + torch.randn((N, V), generator=g), dim=1)
    lp, ids = t.topk(k_eff, dim=1)
    ids = ids.to(torch.int32)
    if k_eff < k:
        ids = torch.cat([ids, torch.full((N, k - k_eff), -1, dtype=torch.int32)], 1)
        lp = torch.cat([lp, torch.zeros((N, k - k_eff))], 1)
    perm = torch.stack([torch.randperm(k, generator=g) for _ in range(N)])
    ids, lp = ids.gather(1, perm), lp.gather(1, perm)
    if ragged:
        ids[torch.rand((N, k), generator=g) < 0.4] = -1
        ids[N // 2] = -1
    return ids.contiguous(), lp.contiguous()


def check_distill(dx, view, ids, lp, tail, T, weight=None, in_place=False, out_rows=None):
    binding, ctx = dx
    z = np64(view)
    dev = [x if x is None else x.cuda() for x in (ids, lp, weight)]
    only = binding.spec_distill_topk(ctx, view, dev[0], dev[1], tail=tail, temperature=T, row_weight=dev[2], grad=False)
    out = None
    if in_place:
        out = {"loss": torch.empty(view.shape[0], device="cuda"), "dlogits": view}
    elif out_rows is not None:
        out = {"loss": torch.empty(view.shape[0], device="cuda"), "dlogits": out_rows}
    got = binding.spec_distill_topk(ctx, view, dev[0], dev[1], tail=tail, temperature=T, row_weight=dev[2], out=out)
    assert torch.equal(torch.nan_to_num(only["loss"], nan=-7.0), torch.nan_to_num(got["loss"], nan=-7.0))
    loss, grad, size = B.distill_topk(z, ids.numpy(), lp.numpy().astype(np.float64), tail, T,
                                      None if weight is None else weight.numpy().astype(np.float64))
    have = np64(got["loss"])
    with np.errstate(invalid="ignore"):
        # (log S and log R, each off by S_ERR, weighted with masses that sum to one)
        assert np.all((have == loss) | (np.isnan(have) & np.isnan(loss)) |
                      (np.abs(have - loss) <= 2 * S_ERR + 2.0 ** -22 * np.abs(loss)))
        d = np64(got["dlogits"])
        tol = 2 * S_ERR * size + HALF[view.dtype] * np.abs(grad) + 1e-36
        assert np.all((np.isnan(d) & np.isnan(grad)) | (np.abs(d - grad) <= tol)), np.nanmax(np.abs(d - grad) - tol)
    return got


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("N,V,pad,shift,k,T", [
    (1, 1, 0, 0, 1, 1.0), (2, 3, 0, 1, 3, 1.0), (3, 7, 1, 3, 2, 0.5), (2, 8, 0, 0, 8, 1.0), (4, 17, 0, 1, 5, 2.0),
    (3, 64, 2, 5, 33, 1.0), (5, 300, 0, 7, 64, 1.0), (2, 200, 0, 0, 128, 1.0), (33, 1024, 0, 0, 8, 1.0),
    (9, 4099, 0, 3, 20, 1.0), (650, 3001, 1, 1, 4, 1.0), (3, 32003, 0, 0, 65, 2.0), (2, 102400, 8, 0, 8, 1.0),
    (1, 163840, 0, 0, 20, 1.0), (2, 163839, 0, 1, 100, 1.0)])
def test_distill_small_and_ragged(dx, dtype, tail, N, V, pad, shift, k, T):
    z = draw_logits(N * 3 + V, N, V)
    ids, lp = teacher_lists(N + V, z, k, ragged=N > 1, T=T)
    view = rows(z, dtype, pad, shift)
    out_rows = rows(torch.zeros((N, V)), dtype, pad + 1, (shift + 2) % 8, fill=77.0)    # another pitch and alignment
    check_distill(dx, view, ids, lp, tail, T, out_rows=out_rows)
    full = out_rows.as_strided((N, V + pad + 1), (V + pad + 1, 1))
    assert torch.all(full[:, V:] == 77.0)                                               # columns behind the rows
    w = torch.linspace(-1, 2, N)
    w[0] = 0.0
    check_distill(dx, view, ids, lp, tail, T, weight=w)
    keep = view.as_strided((N, V + pad), (V + pad, 1))[:, V:].clone()
    check_distill(dx, view, ids, lp, tail, T, weight=w, in_place=True)
    assert torch.equal(view.as_strided((N, V + pad), (V + pad, 1))[:, V:], keep)


@pytest.mark.parametrize("dtype", DTYPES)
def test_distill_many_rows(dx, dtype):
    """As many rows as take the form for large batches, at a row length of four CTAs; every row against the checker."""
    N, V = 300, 70001 if dtype == torch.bfloat16 else 35001
    z = draw_logits(11, N, V)
    ids, lp = teacher_lists(12, z, 16, ragged=True)
    check_distill(dx, rows(z, dtype), ids, lp, True, 1.0)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("V", [50, 9001, 140003])
def test_distill_masks_infinities_nan_and_odd_lists(dx, dtype, tail, V):
    low = torch.finfo(dtype).min
    N = 14
    z = draw_logits(13, N, V)
    ids = torch.full((N, 6), -1, dtype=torch.int32)
    lp = torch.log(torch.tensor([0.5, 0.2, 0.1, 0.05, 0.02, 0.01])).repeat(N, 1)
    for t in range(N):
        ids[t, :4] = torch.tensor([3, V - 1, 7, 20], dtype=torch.int32)
    w = torch.ones(N)
    z[0, 10:15] = -INF                                  # masked words that are not listed
    z[1, 3] = -INF                                      # a listed word without mass: loss +inf, finite gradient
    z[2, :] = -INF                                      # no distribution
    z[3, :] = low
    z[4, 30:] = low
    ids[5, 1] = 3                                       # the same word twice
    ids[5, 3] = 3
    lp[6, :] = -INF                                     # a teacher without mass on its list
    lp[7, 0] = 0.0                                      # ... with all of it on one word
    lp[7, 1:] = -INF
    lp[8, :] = torch.log(torch.tensor(0.3))             # masses that add up to more than one
    z[9, :] = NAN                                       # weight 0: not looked at
    w[9] = 0.0
    ids[10, :] = -1                                     # nothing listed
    z[10, 4] = NAN
    z[11, 5] = NAN
    z[12, [3, 7, 20, V - 1]] += 60.0                    # the student's mass on unlisted words is far below 2^-24
    z[13, [3, 7, 20, V - 1]] = -INF                     # every listed word masked
    view = rows(z, dtype, 3, 1)
    got = check_distill(dx, view, ids, lp, tail, 1.0, weight=w)
    assert float(got["loss"][1]) == INF and float(got["loss"][13]) == INF and torch.isfinite(got["dlogits"][1]).all()
    assert not got["dlogits"][2].any() and not got["dlogits"][9].any() and not got["dlogits"][10].any()
    assert torch.isnan(got["dlogits"][11]).all() and torch.isnan(got["loss"][11])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T", [1e-4, 0.03, 0.7, 0.9, 1.1, 1.3, 1.7, 3.0, 5.0, 7.7, 100.0, 1e4])
def test_temperatures(dx, dtype, T):
    """Over the whole range, with masked words: log2(e) / T rounds up for some temperatures and down for others."""
    z = draw_logits(31, 6, 3000)
    z[1, 100:200] = -INF
    z[2, 1:] = -INF
    z[3, 5:] = torch.finfo(dtype).min
    ids, lp = teacher_lists(32, z.clamp(min=-50), 9, ragged=False)
    ids[2, 0], ids[2, 1] = 0, -1
    view = rows(z, dtype, 1)
    check_logprobs(dx, view, [1, 2, 0, 3, 2999, -1], 12, T)
    check_distill(dx, view, ids, lp, True, T)
    check_distill(dx, view, ids, lp, False, T)


def test_distill_whole_vocabulary_listed(dx):
    z = draw_logits(14, 3, 100)
    ids, lp = teacher_lists(15, z, 100, ragged=False)
    check_distill(dx, rows(z, torch.float32), ids, lp, False, 1.0)
    lp2 = (lp.double() - 1e-3).float()                  # mass left over, and no word to compare it with
    got = check_distill(dx, rows(z, torch.float32), ids, lp2, True, 1.0)
    assert torch.isinf(got["loss"]).all() and torch.isfinite(got["dlogits"]).all()


def test_distill_gradient_between_the_logits_rows(dx):
    binding, ctx = dx
    N, V = 20, 3001
    z = draw_logits(33, N, V)
    ids, lp = teacher_lists(34, z, 8, ragged=False)
    buf = torch.zeros((N, 2 * V + 3), device="cuda")
    buf[:, :V] = z.cuda()
    got = binding.spec_distill_topk(ctx, buf[:, :V], ids.cuda(), lp.cuda(),
                                    out={"loss": torch.empty(N, device="cuda"), "dlogits": buf[:, V:2 * V]})
    want = binding.spec_distill_topk(ctx, z.cuda(), ids.cuda(), lp.cuda())
    assert torch.equal(buf[:, :V].cpu(), z) and not buf[:, 2 * V:].any()
    # (rows at other offsets from a vector's border add up in another order)
    assert bool(((got["dlogits"].double() - want["dlogits"].double()).abs() <= 4 * S_ERR).all())


def test_distill_bad_ids_and_sizes(dx):
    binding, ctx = dx
    z = draw_logits(16, 2, 50)
    ids = torch.tensor([[1, 50, 2], [-5, 3, 4]], dtype=torch.int32)
    lp = torch.log(torch.full((2, 3), 0.25))
    check_distill(dx, rows(z, torch.float32), ids, lp, True, 1.0)
    assert ctx.device_status() == 5 and ctx.device_status() == 0
    empty = binding.spec_distill_topk(ctx, rows(z, torch.float32)[:0], ids[:0].cuda(), lp[:0].cuda())
    assert empty["dlogits"].shape == (0, 50)
    big = torch.zeros((1, 2_000_000), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(binding.DxError) as err:
        binding.spec_distill_topk(ctx, big, ids[:1].cuda(), lp[:1].cuda())
    assert err.value.status == 8


@pytest.mark.parametrize("dtype,V", [(torch.bfloat16, 1_700_001), (torch.float32, 900_000)])
def test_distill_longest_rows(dx, dtype, V):
    z = draw_logits(17, 2, V)
    ids, lp = teacher_lists(18, z, 32, ragged=False)
    check_distill(dx, rows(z, dtype), ids, lp, True, 1.0)


def test_distill_gradient_against_differences(dx):
    """The gradient the kernel returns predicts how the loss it returns changes: a fp32 loss is good to about 1e-6 here
    (2 S_ERR at worst, see above, in practice a few steps of log S), a step of 0.05 changes it by 1e-3 and more; the
    second-order term of a central difference is below 0.05^2 / 24 of the third derivative, which is at most 1."""
    binding, ctx = dx
    z = draw_logits(19, 1, 600, scale=1.0)
    ids, lp = teacher_lists(20, z, 10, ragged=False)
    dev = z.cuda()
    h = 0.05
    base = binding.spec_distill_topk(ctx, dev, ids.cuda(), lp.cuda(), tail=True)
    for v in [int(ids[0, 0]), int(ids[0, 5]), int(z[0].argmax()), 17]:
        e = torch.zeros_like(dev)
        e[0, v] = h
        up = binding.spec_distill_topk(ctx, dev + e, ids.cuda(), lp.cuda(), tail=True, grad=False)["loss"]
        down = binding.spec_distill_topk(ctx, dev - e, ids.cuda(), lp.cuda(), tail=True, grad=False)["loss"]
        diff = float(up.double() - down.double()) / (2 * h)
        assert abs(diff - float(base["dlogits"][0, v])) <= 2 * S_ERR / h + h * h / 24 + 1e-6


# ---- routing ----------------------------------------------------------------------------------------------------------
def check_route(dx, view, k, sigmoid, norm, scale, bias=None, groups=1, keep=1, top2=False):
    binding, ctx = dx
    out = binding.moe_route_tokens(ctx, view, k, score_fn=int(sigmoid), norm_topk=int(norm), routed_scale=scale,
                                   select_bias=None if bias is None else bias.cuda(), n_groups=groups, topk_groups=keep,
                                   group_score=int(top2))
    ids, w, offsets, perm = B.route(np64(view), k, sigmoid, norm, float(np.float32(scale)),
                                    None if bias is None else bias.numpy().astype(np.float64), groups, keep, top2)
    got = out["topk_ids"].cpu().numpy()
    assert np.array_equal(got, ids), np.nonzero((got != ids).any(axis=1))[0][:5]
    assert np.all(np.abs(np64(out["topk_w"]) - w) <= GATE * np.abs(w) + 1e-37)
    assert np.array_equal(out["offsets"].cpu().numpy(), offsets) and np.array_equal(out["perm"].cpu().numpy(), perm)
    return out


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("N,E,k,groups,keep,top2,biased,norm,pad", [
    (1, 1, 1, 1, 1, False, False, True, 0), (3, 2, 2, 1, 1, False, True, True, 0), (5, 8, 2, 1, 1, False, False, True, 0),
    (4, 9, 8, 1, 1, False, True, False, 1), (7, 32, 8, 4, 2, True, True, True, 0), (6, 30, 5, 3, 2, True, False, True, 3),
    (9, 60, 8, 1, 1, False, True, True, 0), (4, 64, 6, 1, 1, False, False, True, 0), (64, 64, 6, 8, 3, True, True, True, 8),
    (65, 64, 6, 8, 4, False, True, False, 0), (100, 72, 7, 9, 3, True, True, True, 0), (33, 128, 8, 16, 4, True, True, True, 0),
    (40, 130, 8, 13, 2, True, False, True, 1), (31, 160, 6, 8, 3, False, True, True, 0), (50, 256, 8, 8, 4, True, True, True, 0),
    (50, 256, 8, 32, 5, True, True, False, 4), (70, 255, 8, 1, 1, False, True, True, 0), (20, 254, 3, 2, 1, True, False, False, 2),
    (17, 96, 8, 32, 3, False, True, True, 0), (1000, 64, 6, 1, 1, False, True, True, 0), (513, 24, 4, 4, 3, True, True, True, 0)])
def test_route_small_and_ragged(dx, dtype, sigmoid, N, E, k, groups, keep, top2, biased, norm, pad):
    z = draw_logits(N + E, N, E, scale=1.5).clamp(-12, 12)
    bias = torch.randn((E,), generator=torch.Generator().manual_seed(E)) * 0.05 if biased else None
    check_route(dx, rows(z, dtype, pad, pad), k, sigmoid, norm, 2.446 if sigmoid else 1.0, bias, groups, keep, top2)


@pytest.mark.parametrize("N", [4000, 20011])
def test_route_large_batches(dx, N):
    """Enough tokens for both launches and every CTA; selection in fp64 torch (the row-by-row checker is too slow)."""
    binding, ctx = dx
    E, k = 96, 6
    g = torch.Generator().manual_seed(N)
    z = torch.randn((N, E), generator=g)
    bias = torch.randn((E,), generator=g) * 0.1
    out = binding.moe_route_tokens(ctx, z.cuda(), k, score_fn=1, select_bias=bias.cuda())
    v = torch.sigmoid(z.double()) + bias.double()
    ids = torch.sort(v, dim=1, descending=True, stable=True).indices[:, :k]
    assert torch.equal(out["topk_ids"].cpu().long(), ids)
    flat = ids.reshape(-1)
    assert torch.equal(out["perm"].cpu().long(), torch.sort(flat, stable=True).indices)
    assert out["offsets"].cpu().tolist() == [0] + torch.cumsum(torch.bincount(flat, minlength=E), 0).tolist()
    again = binding.moe_route_tokens(ctx, z.cuda(), k, score_fn=1, select_bias=bias.cuda())
    assert all(torch.equal(out[name], again[name]) for name in out)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("E", [20, 64, 200, 256])
def test_route_ties_and_values_32_bits_cannot_tell_apart(dx, dtype, E):
    g = torch.Generator().manual_seed(E)
    z = torch.randn((24, E), generator=g)
    z[0] = 0.0
    z[1] = torch.randint(0, 3, (E,), generator=g).float()
    z[2] = 1.0
    z[2, E // 2] = float(np.nextafter(np.float32(1.0), np.float32(2.0)))
    z[3, ::2] = -0.0
    z[3, 1::2] = 0.0
    z = z.to(dtype).float()
    for sigmoid in (False, True):
        check_route(dx, rows(z, dtype), 6, sigmoid, True, 1.0)
        check_route(dx, rows(z, dtype), 6, sigmoid, True, 1.0, bias=torch.zeros(E))
        # a bias that brings every selection value of row 4 to the same place, up to its own rounding to fp32
        r = B.scores(z[4].double().numpy(), sigmoid)
        bias = torch.from_numpy((1.0 - r).astype(np.float32))
        check_route(dx, rows(z, dtype), 6, sigmoid, True, 1.0, bias=bias)
        if E % 4 == 0:
            check_route(dx, rows(z, dtype), 5, sigmoid, True, 1.0, bias=bias, groups=4, keep=2, top2=True)
            check_route(dx, rows(z, dtype), 5, sigmoid, True, 1.0, groups=4, keep=2, top2=True)
            check_route(dx, rows(z, dtype), 5, sigmoid, True, 1.0, groups=4, keep=2, top2=False)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("biased", [False, True])
def test_route_masked_experts(dx, dtype, sigmoid, norm, biased):
    low = torch.finfo(dtype).min
    E = 64
    z = torch.randn((8, E), generator=torch.Generator().manual_seed(3))
    z[0, ::2] = -INF
    z[1, 3:] = -INF                     # fewer experts than are selected
    z[2, :] = -INF
    z[3, 2:] = low
    z[4, 8:16] = -INF                   # a whole group
    z[5, :] = -100.0                    # scores that underflow: the gates' ratios do not
    z[5, 7] = -99.0
    z[6, 1:] = -30.0
    bias = torch.randn((E,), generator=torch.Generator().manual_seed(4)) if biased else None
    view = rows(z, dtype)
    check_route(dx, view, 6, sigmoid, norm, 2.0, bias)
    check_route(dx, view, 6, sigmoid, norm, 2.0, bias, groups=8, keep=3, top2=True)
    check_route(dx, view, 6, sigmoid, norm, 2.0, bias, groups=8, keep=3, top2=False)


def test_route_nan_and_infinite_logits_keep_the_ids_valid(dx):
    binding, ctx = dx
    z = torch.randn((6, 40), generator=torch.Generator().manual_seed(7))
    z[0, 5] = NAN
    z[1, :] = NAN
    z[2, 5] = INF
    z[3, :] = INF
    z[4, 2] = 1e30
    for sigmoid in (0, 1):
        for bias in (None, torch.randn(40).cuda(), torch.full((40,), NAN).cuda()):
            for groups, keep in ((1, 1), (5, 2), (10, 4)):
                out = binding.moe_route_tokens(ctx, z.cuda(), 6, score_fn=sigmoid, select_bias=bias, n_groups=groups,
                                               topk_groups=keep, group_score=1)
                ids = out["topk_ids"].cpu()
                assert ids.min() >= 0 and ids.max() < 40 and all(len(set(r)) == 6 for r in ids.tolist())
                flat = ids.reshape(-1).long()
                assert torch.equal(out["perm"].cpu().long(), torch.sort(flat, stable=True).indices)
    ids = binding.moe_route_tokens(ctx, z[:1].cuda(), 8, score_fn=1)["topk_ids"][0].tolist()
    assert 5 not in ids                                   # NaN behind everything else


@pytest.mark.parametrize("dtype", DTYPES)
def test_route_biases_far_from_the_scores(dx, dtype):
    """Biases whose common part leaves a 32-bit sum nothing of the scores: the selection is still exact."""
    z = draw_logits(35, 70, 64, scale=1.2).clamp(-9, 9)
    small = torch.randn((64,), generator=torch.Generator().manual_seed(36)) * 0.01
    for bias in (small + 50.0, small - 3000.0, small * 1e6, torch.full((64,), 1e30), small.clone().fill_(-INF)):
        for sigmoid in (False, True):
            ref_bias = bias
            if not torch.isfinite(bias).all():
                out = dx[0].moe_route_tokens(dx[1], rows(z, dtype), 6, score_fn=int(sigmoid), select_bias=bias.cuda())
                assert torch.equal(out["topk_ids"].cpu(), torch.arange(6, dtype=torch.int32).expand(70, 6))
                continue
            check_route(dx, rows(z, dtype), 6, sigmoid, True, 1.0, ref_bias)
            check_route(dx, rows(z, dtype), 6, sigmoid, True, 1.0, ref_bias, groups=8, keep=3, top2=True)


@pytest.mark.parametrize("top2", [False, True])
@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("E,groups,keep", [(64, 8, 3), (64, 4, 2), (256, 8, 4), (256, 32, 3), (128, 2, 1), (60, 6, 2), (96, 4, 1)])
def test_route_groups_of_nearly_equal_scores(dx, E, groups, keep, top2, sigmoid):
    """Groups that hold the same values in another order, apart by less than fp32 sums tell, or not at all."""
    N, per = 97, E // groups
    g = torch.Generator().manual_seed(40 + E + groups)
    one = torch.randn((N, 1, per), generator=g).expand(N, groups, per)
    bias_one = torch.randn((1, 1, per), generator=g) * 0.05
    order = torch.rand((1, groups, per), generator=g).argsort(dim=2)
    bias = bias_one.expand(1, groups, per).gather(2, order).reshape(E).contiguous()
    for step in (0.0, 2.0 ** -24, 2.0 ** -21, 2.0 ** -16):
        z = one.gather(2, order.expand(N, groups, per))
        z = (z + z.abs() * step * torch.randint(-3, 4, z.shape, generator=g)).reshape(N, E)
        z[5, : E // 2] = -INF
        check_route(dx, rows(z, torch.float32), 4, sigmoid, True, 1.0, bias, groups, keep, top2)
        check_route(dx, rows(z, torch.float32), 4, sigmoid, True, 1.0, None, groups, keep, False)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("N,E,k,off,groups,keep", [
    (1, 8, 7, 3, 1, 1),                                   # all experts but one are selected, three of them without a bias
    (9, 8, 8, 8, 1, 1), (70, 8, 7, 4, 2, 2), (300, 64, 6, 40, 1, 1), (300, 64, 6, 40, 8, 3), (33, 130, 8, 126, 1, 1),
    (130, 256, 8, 100, 8, 4), (20, 30, 5, 12, 5, 2),
])
def test_route_experts_put_aside_by_their_bias(dx, dtype, sigmoid, N, E, k, off, groups, keep):
    """Biases of -inf and NaN beside finite ones: such experts are selected last, in the order of their ids."""
    z = draw_logits(37 + E, N, E, scale=1.2).clamp(-9, 9)
    bias = torch.randn((E,), generator=torch.Generator().manual_seed(38)) * 0.05
    aside = torch.randperm(E, generator=torch.Generator().manual_seed(39))[:off]
    for values in ((NAN,), (-INF,), (-INF, NAN)):
        bias[aside] = torch.tensor(values).repeat(off)[:off]
        plain = torch.where(torch.isnan(bias), torch.full_like(bias, -INF), bias)
        for top2 in (False, True):
            out = dx[0].moe_route_tokens(dx[1], rows(z, dtype), k, score_fn=int(sigmoid), select_bias=bias.cuda(),
                                         n_groups=groups, topk_groups=keep, group_score=int(top2))
            want = check_route(dx, rows(z, dtype), k, sigmoid, True, 1.0, plain, groups, keep, top2)
            assert all(torch.equal(out[name], want[name]) for name in want)


def test_route_no_tokens_and_optional_outputs(dx):
    binding, ctx = dx
    empty = binding.moe_route_tokens(ctx, torch.empty((0, 16), device="cuda"), 4)
    assert empty["topk_ids"].shape == (0, 4) and not empty["offsets"].any()
    z = torch.randn((200, 16), device="cuda")
    out = {"topk_ids": torch.empty((200, 4), dtype=torch.int32, device="cuda"), "topk_w": torch.empty((200, 4), device="cuda")}
    binding.moe_route_tokens(ctx, z, 4, out=out)
    full = binding.moe_route_tokens(ctx, z, 4)
    assert torch.equal(out["topk_ids"], full["topk_ids"]) and torch.equal(out["topk_w"], full["topk_w"])


# ---- gradient of the gates ------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("N,E,k,pad", [(1, 1, 1, 0), (3, 8, 2, 0), (5, 9, 8, 1), (33, 31, 5, 2), (40, 64, 6, 0),
                                       (17, 100, 8, 3), (300, 130, 7, 0), (50, 256, 8, 0), (9, 255, 1, 5)])
def test_route_grad(dx, dtype, sigmoid, norm, N, E, k, pad):
    binding, ctx = dx
    z = torch.randn((N, E), generator=torch.Generator().manual_seed(N + E)) * 1.5
    if N > 4 and E > 8:
        z[1, 3:6] = -INF
        z[2] = -INF
    view = rows(z, dtype, pad, pad)
    ids = binding.moe_route_tokens(ctx, view, k, score_fn=int(sigmoid))["topk_ids"]
    dw = torch.randn((N, k), generator=torch.Generator().manual_seed(1))
    if N > 4 and E > 8 and k > 1:
        ids[3, 1] = ids[3, 0]                              # the same expert twice
    out = rows(torch.zeros((N, E)), dtype, pad + 2, 0, fill=55.0)
    got = binding.moe_route_tokens_backward(ctx, view, ids, dw.cuda(), score_fn=int(sigmoid), norm_topk=int(norm),
                                            routed_scale=2.446, out=out)
    want, size = B.route_grad(np64(view), ids.cpu().numpy(), dw.numpy().astype(np.float64), sigmoid, norm,
                              float(np.float32(2.446)))
    d = np64(got)
    # (each of up to nine magnitudes good to GATE)
    assert np.all(np.abs(d - want) <= 2 * GATE * size + HALF[dtype] * np.abs(want) + 1e-37)
    assert torch.all(out.as_strided((N, E + pad + 2), (E + pad + 2, 1))[:, E:] == 55.0)


def test_route_grad_bad_ids_and_underflow(dx):
    binding, ctx = dx
    z = torch.randn((4, 16), generator=torch.Generator().manual_seed(2))
    z[3] = -100.0
    z[3, 2] = -99.5
    ids = torch.tensor([[0, 16], [-1, 3], [5, 6], [2, 4]], dtype=torch.int32, device="cuda")
    dw = torch.tensor([[1.0, 2.0], [3.0, -1.0], [0.5, 0.25], [1.0, -1.0]])
    got = binding.moe_route_tokens_backward(ctx, z.cuda(), ids, dw.cuda(), score_fn=1, norm_topk=1)
    want, size = B.route_grad(z.double().numpy(), ids.cpu().numpy(), dw.double().numpy(), True, True, 1.0)
    assert np.all(np.abs(np64(got) - want) <= 2 * GATE * size + 1e-37)
    assert ctx.device_status() == 1 and ctx.device_status() == 0
    empty = binding.moe_route_tokens_backward(ctx, z[:0].cuda(), ids[:0], dw[:0].cuda())
    assert empty.shape == (0, 16)


# ---- streams, graphs, devices, refusals ------------------------------------------------------------------------------------
def _all_calls(binding, ctx, s):
    lp = binding.spec_token_logprobs(ctx, s["teacher"], s["tokens"], top_n=16)
    ds = binding.spec_distill_topk(ctx, s["logits"], lp["top_ids"], lp["top_logprobs"], tail=True)
    rt = binding.moe_route_tokens(ctx, s["router"], 6, score_fn=1, select_bias=s["bias"], n_groups=4, topk_groups=2,
                                  group_score=1)
    gr = binding.moe_route_tokens_backward(ctx, s["router"], rt["topk_ids"], rt["topk_w"], score_fn=1)
    return [lp[k] for k in sorted(lp)] + [ds["loss"], ds["dlogits"]] + [rt[k] for k in sorted(rt)] + [gr]


def _state(N, V, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    draw = lambda *shape: torch.randn(shape, generator=g, device="cuda")  # noqa: E731
    return {"teacher": (draw(N, V) * 3).bfloat16(), "logits": (draw(N, V) * 2).bfloat16(), "router": draw(N, 64),
            "bias": draw(64) * 0.1, "tokens": torch.arange(N, dtype=torch.int32, device="cuda") % V}


@pytest.mark.parametrize("N,V", [(3, 20001), (200, 5000)])
def test_graph_replay_other_streams_and_two_contexts(dx, N, V):
    binding, ctx = dx
    a, b = _state(N, V, 1), _state(N, V, 2)
    want_a = [t.clone() for t in _all_calls(binding, ctx, a)]
    want_b = [t.clone() for t in _all_calls(binding, ctx, b)]
    torch.cuda.synchronize()
    # captured once, replayed on other inputs in the same buffers
    s = {k: v.clone() for k, v in a.items()}
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = _all_calls(binding, ctx, s)
    for state, want in ((a, want_a), (b, want_b), (a, want_a)):
        for k in s:
            s[k].copy_(state[k])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(outs, want))
    # two contexts at once on two streams
    other = binding.Context(0)
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(5):
        with torch.cuda.stream(s1):
            got_a = _all_calls(binding, ctx, a)
        with torch.cuda.stream(s2):
            got_b = _all_calls(binding, other, b)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got_a, want_a))
        assert all(torch.equal(x, y) for x, y in zip(got_b, want_b))
    assert other.device_status() == 0
    other.close()


def test_binding_refusals(dx):
    binding, ctx = dx
    z = torch.zeros((4, 32), device="cuda")
    tok = torch.zeros((4,), dtype=torch.int32, device="cuda")
    ids = torch.zeros((4, 2), dtype=torch.int32, device="cuda")
    lp = torch.zeros((4, 2), device="cuda")
    for bad in (z.half(), z.t(), z[0], z.cpu(), z[:, ::2]):
        with pytest.raises(ValueError):
            binding.spec_token_logprobs(ctx, bad, None, top_n=1)
    for call in (lambda: binding.spec_token_logprobs(ctx, z, tok.long()),
                 lambda: binding.spec_token_logprobs(ctx, z, tok[:3]),
                 lambda: binding.spec_distill_topk(ctx, z, ids.long(), lp),
                 lambda: binding.spec_distill_topk(ctx, z, ids, lp.double()),
                 lambda: binding.spec_distill_topk(ctx, z, ids, lp, row_weight=torch.ones(3, device="cuda")),
                 lambda: binding.spec_distill_topk(ctx, z, ids, lp, out={"dlogits": z.bfloat16()}),
                 lambda: binding.moe_route_tokens(ctx, z, 4, select_bias=torch.zeros(31, device="cuda")),
                 lambda: binding.moe_route_tokens_backward(ctx, z, ids, lp[:, :1])):
        with pytest.raises(ValueError):
            call()
    for call, status in ((lambda: binding.spec_token_logprobs(ctx, z, tok, top_n=33), 2),
                         (lambda: binding.spec_token_logprobs(ctx, z.expand(4, 32)[:, :32], tok, temperature=0.0), 1),
                         (lambda: binding.spec_token_logprobs(ctx, z[:1].expand(4, 32), tok), 2),
                         (lambda: binding.spec_distill_topk(ctx, z[:3], ids[:3], lp[:3], out={"dlogits": z[1:]}), 1),
                         (lambda: binding.moe_route_tokens(ctx, z, 9), 8),
                         (lambda: binding.moe_route_tokens(ctx, z, 4, n_groups=5), 2),
                         (lambda: binding.moe_route_tokens_backward(ctx, z, ids, lp, out=z), 1)):
        with pytest.raises(binding.DxError) as err:
            call()
        assert err.value.status == status


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("N,V,k", [(400, 9001, 100), (310, 61003, 9), (40, 410001, 70)])
def test_distill_rows_that_follow_one_another(dx, dtype, tail, N, V, k):
    """More rows than run at a time, of an odd length (their alignment changes from row to row), rows of weight zero, of
    no list and of NaN among them: what a CTA keeps from one row to the next must not show.  Rows
    equal themselves in calls of their own, in a second call and in place."""
    binding, ctx = dx
    g = torch.Generator(device="cuda").manual_seed(N)
    z = torch.randn((N, V), generator=g, device="cuda") * 2
    z[5] = NAN
    view = rows(z, dtype)
    lp, ids = torch.log_softmax(torch.randn((N, V), generator=g, device="cuda") * 2, 1).topk(k, dim=1)
    ids = ids.to(torch.int32).contiguous()
    lp = lp.contiguous()
    w = torch.rand((N,), generator=g, device="cuda") + 0.5
    w[::3] = 0.0
    ids[1::7] = -1
    whole = binding.spec_distill_topk(ctx, view, ids, lp, tail=tail, row_weight=w)
    again = binding.spec_distill_topk(ctx, view, ids, lp, tail=tail, row_weight=w)
    bits = lambda t: t.view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32)  # noqa: E731
    assert torch.equal(bits(whole["dlogits"]), bits(again["dlogits"])) and torch.equal(bits(whole["loss"]), bits(again["loss"]))
    for r in range(0, N, 97):
        one = binding.spec_distill_topk(ctx, view[r:r + 1], ids[r:r + 1], lp[r:r + 1], tail=tail, row_weight=w[r:r + 1].contiguous())
        live = bool(w[r] != 0) and bool((ids[r] >= 0).any())
        if not live:
            assert float(whole["loss"][r]) == 0 and not whole["dlogits"][r].any() and not one["dlogits"].any()
        elif r != 5:
            # (a lone row is split over more CTAs: other partial sums)
            assert abs(float(one["loss"][0]) - float(whole["loss"][r])) <= 4 * S_ERR
            diff = (one["dlogits"][0].double() - whole["dlogits"][r].double()).abs()
            assert bool((diff <= 4 * S_ERR * float(w[r]) + 2 * HALF[dtype] * whole["dlogits"][r].double().abs()).all())
    assert torch.isnan(whole["dlogits"][5]).all() == bool(w[5] != 0 and (ids[5] >= 0).any())
    mine = rows(z, dtype)
    binding.spec_distill_topk(ctx, mine, ids, lp, tail=tail, row_weight=w,
                              out={"loss": torch.empty(N, device="cuda"), "dlogits": mine})
    assert torch.equal(bits(mine.contiguous()), bits(whole["dlogits"]))


@pytest.mark.parametrize("N,E,k,groups,keep,biased,dtype", [
    (40000, 256, 8, 8, 4, True, torch.bfloat16), (40000, 256, 8, 1, 1, False, torch.bfloat16),
    (120001, 32, 8, 1, 1, True, torch.float32), (33333, 64, 6, 4, 2, False, torch.float32),
    (20000, 100, 7, 10, 3, True, torch.bfloat16), (30000, 64, 8, 1, 1, False, torch.bfloat16)])
@pytest.mark.parametrize("sigmoid", [False, True])
def test_route_large_batches_of_every_form(dx, N, E, k, groups, keep, biased, dtype, sigmoid):
    """Selection in fp64 torch: thousands of tokens whose selection 32 bits cannot settle are among these."""
    binding, ctx = dx
    g = torch.Generator(device="cuda").manual_seed(N + E)
    z = (torch.randn((N, E), generator=g, device="cuda") * 1.3).to(dtype)
    bias = torch.randn((E,), generator=g, device="cuda") * 0.05 if biased else None
    out = binding.moe_route_tokens(ctx, z, k, score_fn=int(sigmoid), select_bias=bias, n_groups=groups, topk_groups=keep,
                                   group_score=1 if groups > 1 else 0, routed_scale=1.5)
    x = z.double()
    r = torch.sigmoid(x) if sigmoid else torch.softmax(x, 1)
    v = x if bias is None else r + bias.double()
    if groups > 1:
        by = (r if bias is None else v).view(N, groups, -1).topk(2, dim=2).values.sum(2)
        kept = torch.sort(by, dim=1, descending=True, stable=True).indices[:, :keep]
        on = torch.zeros((N, groups), dtype=torch.bool, device="cuda").scatter_(1, kept, True)
        v = v.masked_fill(~on.repeat_interleave(E // groups, 1), -INF)
    ids = torch.sort(v, dim=1, descending=True, stable=True).indices[:, :k]
    assert torch.equal(out["topk_ids"].long(), ids)
    w = r.gather(1, ids)
    w = 1.5 * w / w.sum(1, keepdim=True)
    assert bool(((out["topk_w"].double() - w).abs() <= GATE * w).all())
    flat = ids.reshape(-1)
    assert torch.equal(out["perm"].long(), torch.sort(flat, stable=True).indices)
    assert out["offsets"].tolist() == [0] + torch.cumsum(torch.bincount(flat, minlength=E), 0).tolist()


def test_results_do_not_depend_on_the_launch_overlap(dx):
    binding, ctx = dx
    z = torch.randn((5000, 64), device="cuda")
    want = binding.moe_route_tokens(ctx, z, 6, score_fn=1)
    for mask in (0, 1, 7):
        ctx.set_launch_overlap(mask)
        for _ in range(20):
            got = binding.moe_route_tokens(ctx, z, 6, score_fn=1)
            assert all(torch.equal(got[n], want[n]) for n in want)
    ctx.set_launch_overlap(3)


def test_first_call_of_a_context_inside_a_capture(dx):
    binding, ctx = dx
    s = _state(6, 30001, 5)
    want = [t.clone() for t in _all_calls(binding, ctx, s)]
    fresh = binding.Context(0)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = _all_calls(binding, fresh, s)
    for _ in range(50):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(outs, want))
    assert fresh.device_status() == 0
    del graph
    fresh.close()


# ---- the operators together: one training step of a small drafter --------------------------------------------------------
def test_training_step_of_a_small_drafter(dx):
    """The target's logits are scored and cut to a top list; the drafter (a routed layer of linear experts and an LM
    head) is distilled against it; the gradients of its router, experts and head, put together from the operators'
    gradients and matrix products, equal autograd's through the same model in fp64 with the same selection."""
    binding, ctx = dx
    N, H, E, k, V = 48, 32, 16, 4, 500
    g = torch.Generator(device="cuda").manual_seed(21)
    draw = lambda *shape: torch.randn(shape, generator=g, device="cuda")  # noqa: E731
    h, W_r, W_e, W_lm = draw(N, H), draw(E, H) * 0.3, draw(E, H, H) * 0.2, draw(V, H) * 0.3
    target_logits = draw(N, V) * 2
    target = binding.spec_token_logprobs(ctx, target_logits, target_logits.argmax(1).to(torch.int32), top_n=12)
    assert torch.equal(target["logprob"], target["top_logprobs"][:, 0])
    weight = torch.full((N,), 1.0 / N, device="cuda")
    weight[-5:] = 0.0
    # forward
    z = h @ W_r.t()
    route = binding.moe_route_tokens(ctx, z, k, score_fn=1, norm_topk=1, routed_scale=2.446, select_bias=draw(E) * 0.1)
    offsets, perm = route["offsets"].tolist(), route["perm"].long()
    parts = torch.empty((N * k, H), device="cuda")
    for e in range(E):
        mine = perm[offsets[e]:offsets[e + 1]]
        parts[mine] = h[mine // k] @ W_e[e].t()
    gate = route["topk_w"].reshape(-1, 1)
    y = (gate * parts).view(N, k, H).sum(1)
    step = binding.spec_distill_topk(ctx, y @ W_lm.t(), target["top_ids"], target["top_logprobs"], tail=True,
                                     row_weight=weight)
    # backward
    d_lm = step["dlogits"].t() @ y
    dy = step["dlogits"] @ W_lm
    d_gate = (parts.view(N, k, H) * dy[:, None]).sum(2)
    d_parts = gate * dy.repeat_interleave(k, 0)
    d_e = torch.zeros_like(W_e)
    for e in range(E):
        mine = perm[offsets[e]:offsets[e + 1]]
        d_e[e] = d_parts[mine].t() @ h[mine // k]
    d_z = binding.moe_route_tokens_backward(ctx, z, route["topk_ids"], d_gate.contiguous(), score_fn=1, norm_topk=1,
                                            routed_scale=2.446)
    d_r = d_z.t() @ h
    # fp64
    P = [t.double().requires_grad_(True) for t in (W_r, W_e, W_lm)]
    r = torch.sigmoid(h.double() @ P[0].t()).gather(1, route["topk_ids"].long())
    w = 2.446 * r / r.sum(1, keepdim=True)
    yy = torch.einsum("nk,nkh->nh", w, torch.einsum("nkoh,nh->nko", P[1][route["topk_ids"].long()], h.double()))
    logq = torch.log_softmax(yy @ P[2].t(), dim=1)
    tz = torch.log_softmax(target_logits.double(), dim=1)
    tl, ti = tz.topk(12, dim=1)
    assert torch.equal(ti.to(torch.int32), target["top_ids"])
    p, rest = tl.exp(), 1 - tl.exp().sum(1)
    other = torch.ones((N, V), dtype=torch.bool, device="cuda").scatter_(1, ti, False)
    log_r = torch.logsumexp(logq.masked_fill(~other, -INF), dim=1)
    loss = (p * (tl - logq.gather(1, ti))).sum(1) + rest * (rest.log() - log_r)
    want = torch.autograd.grad((loss * weight.double()).sum(), P)
    live = weight != 0
    assert torch.allclose(step["loss"][live].double(), loss[live], rtol=1e-4, atol=1e-4) and not step["loss"][~live].any()
    for have, ref in zip((d_r, d_e, d_lm), want):
        # (fp32 matrix products of a few hundred terms on top of the operators' own error)
        assert float((have.double() - ref).abs().max()) <= 1e-4 * float(ref.abs().max())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("N,V,k", [(9000, 1001, 7), (9001, 1000, 40), (2600, 60003, 9), (1000, 400001, 33)])
def test_distill_many_rows_per_cta(dx, dtype, tail, N, V, k):
    """Rows by the dozen on every CTA, with and without a gradient, rows of weight zero and of no list among them: all
    losses against 64 bits, the same with and without gradient, and the gradients' sums (zero up to roundings)."""
    binding, ctx = dx
    if dtype is torch.float32 and V > 100000:
        N //= 2
    g = torch.Generator(device="cuda").manual_seed(N + V)
    z = torch.empty((N, V), dtype=dtype, device="cuda")
    ids = torch.empty((N, k), dtype=torch.int32, device="cuda")
    lp = torch.empty((N, k), device="cuda")
    w = torch.rand((N,), generator=g, device="cuda") + 0.5
    w[2::5] = 0.0
    loss = torch.empty((N,), dtype=torch.float64, device="cuda")
    for a in range(0, N, 100):
        b = min(a + 100, N)
        x = torch.randn((b - a, V), generator=g, device="cuda") * 2
        z[a:b] = x.to(dtype)
        t = torch.log_softmax(x + torch.randn((b - a, V), generator=g, device="cuda"), 1)
        l, i = t.topk(k, dim=1)
        ids[a:b], lp[a:b] = i.int(), l
        logq = torch.log_softmax(z[a:b].double(), 1).gather(1, i)
        p = l.double().exp()
        if tail:
            r = 1 - p.sum(1)
            loss[a:b] = (p * (l.double() - logq)).sum(1) + r * (r.log() - torch.log1p(-logq.exp().sum(1)))
        else:
            p = p / p.sum(1, keepdim=True)
            loss[a:b] = (p * (p.log() - logq)).sum(1)
    ids[4::11] = -1
    loss[4::11] = 0
    loss[2::5] = 0
    only = binding.spec_distill_topk(ctx, z, ids, lp, tail=tail, row_weight=w, grad=False)["loss"]
    got = binding.spec_distill_topk(ctx, z, ids, lp, tail=tail, row_weight=w)
    assert torch.equal(only, got["loss"])
    assert bool(((only.double() - loss).abs() <= 2 * S_ERR + 2.0 ** -22 * loss.abs()).all())
    # a row's gradient is w / T (beta q - p): its sum is that of the errors, S_ERR and a rounding of each part
    for a in range(0, N, 500):
        d = got["dlogits"][a:a + 500].double()
        assert bool((d.sum(1).abs() <= 4 * S_ERR * w[a:a + 500] + HALF[dtype] * d.abs().sum(1)).all())
        dead = (w[a:a + 500] == 0) | (ids[a:a + 500] < 0).all(1)
        assert not d[dead].any() and bool((d[~dead].abs().sum(1) > 0).all())
