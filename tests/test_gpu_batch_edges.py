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


def near_teacher(N, V, k, eps, T, dtype, seed):
    """Logits, and the lists of a teacher whose logits differ from them by `eps` at random."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    z = torch.randn((N, V), generator=g, device="cuda") * 2
    lift = torch.rand((N, 30), generator=g, device="cuda") * 9 + 3
    z.scatter_add_(1, torch.randint(0, V, (N, 30), generator=g, device="cuda"), lift)
    z = z.to(dtype)
    noise = torch.randn((N, V), generator=g, device="cuda", dtype=torch.float64)
    lp, ids = torch.log_softmax(z.double() / T + eps * noise, 1).topk(k, dim=1)
    return z, ids.to(torch.int32), lp.float()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("N,V,k,T", [(512, 2000, 20, 1.0), (128, 32003, 20, 1.0), (128, 32003, 70, 1.0), (64, 102400, 20, 1.0),
                                     (400, 9000, 5, 2.0), (40, 163840, 100, 0.7)])
@pytest.mark.parametrize("eps", [1e-3, 1e-5])
def test_distill_gradient_of_a_student_close_to_its_teacher(dx, dtype, tail, N, V, k, T, eps):
    """The gradient is then a small difference.  With R the student's mass on the unlisted words, r the teacher's, P = 1 - R,
    the only inexact sum is R's: its exponentials are good to 2^-22 and to 2^-24 on average, their arguments and the sums add
    errors of either sign that average out over the words, so R is good to 2^-23 (rms over rows).  An unlisted word's
    factor beta - r / R is off by P times that (r close to R), a listed word's beta q - p by p R times that; either is rounded to
    the output's type."""
    binding, ctx = dx
    T = float(np.float32(T))                            # (what the entry point gets)
    z, ids, lp = near_teacher(N, V, k, eps, T, dtype, seed=N + V)
    d = binding.spec_distill_topk(ctx, z, ids, lp, tail=tail, temperature=T)["dlogits"].double() * T
    q = torch.softmax(z.double() / T, 1)
    at = ids.long()
    p = lp.double().exp()
    other = q.scatter(1, at, 0.0)
    R = other.sum(1)
    if not tail:
        p = p / p.sum(1, keepdim=True)
    rest = (1 - p.sum(1)) if tail else torch.zeros_like(R)
    beta = p.sum(1) + rest
    want = beta[:, None] * q.gather(1, at) - p
    tol = 2.0 ** -23 * p * R[:, None] + HALF[dtype] * want.abs()
    err = (d.gather(1, at) - want) / tol
    assert float(err.pow(2).mean().sqrt()) <= 1, float(err.pow(2).mean().sqrt())
    factor = beta - rest / R
    # (the factor as the row's unlisted words show it together: each of them is factor times an exponential, whose argument of
    # at most 20 powers of two is rounded twice, 2 * 20 * 2^-24 * ln 2, and which is good to 2^-22 itself; the factor's last
    # quotient and products add 2^-21: below 2^-18 together; words of equal logits, which bf16 has many of, are rounded alike,
    # so the roundings of the output add up to half a step of the sum)
    have = d.scatter(1, at, 0.0).sum(1) / R
    tol = 2.0 ** -23 * (1 - R) + (HALF[dtype] + 2.0 ** -18) * factor.abs()
    err = (have - factor) / tol
    assert float(err.pow(2).mean().sqrt()) <= 1, float(err.pow(2).mean().sqrt())
    if tail and eps == 1e-3:
        assert bool((have.sign() == factor.sign())[factor.abs() > 2.0 ** -20].all())


def microseconds(call, repeats=9):
    times = []
    for _ in range(repeats):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        call()
        b.record()
        torch.cuda.synchronize()
        times.append(a.elapsed_time(b) * 1e3)
    return sorted(times)[repeats // 2]


@pytest.mark.parametrize("grad", [False, True])
def test_distill_rows_without_weight_or_list_are_not_fetched(dx, grad):
    """The logits of such rows are not read (but for the few that a CTA begins with): a batch of 840 MB of them takes a
    fraction of the time of one whose rows all count -- with a gradient half of it, the zeros being written, else next
    to nothing -- and so does a batch whose second half is padding."""
    binding, ctx = dx
    N, V, k = 4096, 102400, 8
    z = torch.zeros((N, V), dtype=torch.bfloat16, device="cuda")
    ids = torch.randint(0, V, (N, k), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(torch.int32)
    lp = torch.full((N, k), -3.0, device="cuda")
    one, half = torch.ones(N, device="cuda"), torch.arange(N, device="cuda") < N // 2
    out = {"loss": torch.empty(N, device="cuda")}
    if grad:
        out["dlogits"] = torch.empty_like(z)

    def time(weight, lists):
        call = lambda: binding.spec_distill_topk(ctx, z, lists, lp, row_weight=weight, grad=grad, out=out)  # noqa: E731
        call()
        return microseconds(call)

    none = torch.full_like(ids, -1)
    whole = time(one, ids)
    assert time(0 * one, ids) <= 0.65 * whole and time(one, none) <= 0.65 * whole
    assert time(half.float(), ids) <= 0.85 * whole and time(one, torch.where(half[:, None], ids, none)) <= 0.85 * whole


def test_route_calls_that_share_a_context_unordered_stay_inside_their_outputs(dx):
    """Two captured graphs of one context share its scratch.  Replayed one after the other they give their own results;
    replayed at once, which the header rules out, the permutations are undefined but nothing beside them is written."""
    binding, ctx = dx
    N, E, k, pad = 40000, 64, 6, 1 << 20
    graphs, outs, buffers, wants = [], [], [], []
    for i in range(2):
        z = torch.randn((N, E), generator=torch.Generator(device="cuda").manual_seed(i), device="cuda")
        z[:, (0 if i else E // 2):(E // 2 if i else E)] += 4.0          # (the two select other experts)
        want = binding.moe_route_tokens(ctx, z, k, score_fn=1)
        buf = torch.full((N * k + 2 * pad,), -7, dtype=torch.int32, device="cuda")
        out = {name: torch.empty_like(want[name]) for name in ("topk_ids", "topk_w", "offsets")}
        out["perm"] = buf[pad:pad + N * k]
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            binding.moe_route_tokens(ctx, z, k, score_fn=1, out=out)
        graphs.append(graph), outs.append(out), buffers.append((buf, z)), wants.append(want)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(200):
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
    torch.cuda.synchronize()
    for (buf, _), out, want in zip(buffers, outs, wants):
        assert (buf[:pad] == -7).all() and (buf[pad + N * k:] == -7).all()
        assert torch.equal(out["topk_ids"], want["topk_ids"]) and torch.equal(out["topk_w"], want["topk_w"])
    ctx.device_status()
    for graph in graphs:
        graph.replay()
    torch.cuda.synchronize()
    for out, want in zip(outs, wants):
        assert all(torch.equal(out[name], want[name]) for name in want)


@pytest.mark.parametrize("up", [False, True])
def test_logprobs_are_corrected_for_the_rounding_of_their_factor(dx, up):
    """log2(e) / T is rounded to fp32, by up to 2^-24 of it, which would shift the log probabilities of a row by that times its
    mean |u|: at the temperature with the largest rounding, and rows whose mass lies seven below their largest logit, by 3e-7
    and more, in one direction.  What is left has either sign from row to row -- the mean over 2000 rows loses it -- but for
    the mean error of ex2, at most 2^-24: together less than 2^-23."""
    binding, ctx = dx
    grid = np.arange(1.2, 1.44, 1e-4).astype(np.float32)
    c = 1.4426950408889634 / grid.astype(np.float64)
    rounding = (c - c.astype(np.float32).astype(np.float64)) / c
    i = int(rounding.argmin() if up else rounding.argmax())
    T, rounding = float(grid[i]), float(rounding[i])
    assert abs(rounding) > 2.0 ** -24.5
    N, V = 2000, 20000
    z = torch.randn((N, V), generator=torch.Generator(device="cuda").manual_seed(60), device="cuda")
    z[:, 100] = 12.0
    tokens = torch.arange(N, dtype=torch.int32, device="cuda") % 100
    got = binding.spec_token_logprobs(ctx, z, tokens, temperature=T)
    logq = torch.log_softmax(z.double() / T, 1)
    want = logq.gather(1, tokens.long()[:, None])[:, 0]
    q = logq.exp()
    u = (z.double() - 12.0) / T
    mean_u = (q * u).sum(1)
    shift = float(mean_u.mean()) * rounding                                      # ... of an uncorrected log probability
    assert abs(shift) > 2.0 ** -22
    assert abs(float((got["logprob"].double() - want).mean())) <= 2.0 ** -23
    entropy = -(q * logq).sum(1)
    # The correction makes log S that of T and leaves the mean u with the weights of the rounded factor: together the entropy
    # at log2(e) / c instead of T, which the derivative, the variance of u, tells from the one at T.  (log S as above; the
    # quotient of two sums with the same errors up to 7 times 2^-24 off on average.)
    variance = float((q * u * u).sum(1).mean() - (mean_u ** 2).mean())
    assert abs(float((got["entropy"].double() - entropy).mean())) <= 2.0 ** -23 + 7 * 2.0 ** -24 + abs(rounding) * variance


@pytest.mark.parametrize("dtype", DTYPES)
def test_logprobs_are_probabilities_where_one_word_has_nearly_all(dx, dtype):
    """log p <= 0 and entropy >= 0, wherever in the row the likely word lies and however far it stands above the rest."""
    binding, ctx = dx
    N, V = 300, 30011
    z = torch.randn((N, V), generator=torch.Generator(device="cuda").manual_seed(61), device="cuda")
    at = torch.randint(0, V, (N,), generator=torch.Generator(device="cuda").manual_seed(62), device="cuda")
    z[torch.arange(N), at] = torch.linspace(4.0, 60.0, N, device="cuda")
    z = z.to(dtype)
    for T in (1.0, 0.3, 1.3):
        got = binding.spec_token_logprobs(ctx, z, at.to(torch.int32), top_n=4, temperature=T)
        assert (got["logprob"] <= 0).all() and (got["top_logprobs"] <= 0).all() and (got["entropy"] >= 0).all()
        logq = torch.log_softmax(z.double() / float(np.float32(T)), 1)
        want = logq.gather(1, at[:, None])[:, 0]
        # (5.5 in 32 bits, a few steps; the sums' own error, an exponential's 2^-22 and its argument's rounding, relative to S)
        assert float((got["logprob"].double() - want).abs().max()) <= 5.5 * 2.0 ** -22 + 2.0 ** -20 + 2.0 ** -22 * float(want.abs().max())


@pytest.mark.parametrize("N,V,T", [(2000, 20000, 1.0), (300, 102400, 2.0), (1500, 3001, 0.7)])
def test_rounding_errors_of_log_probabilities_and_losses(dx, N, V, T):
    """Root mean squares over the rows.  A log probability is (z - m) / T - log S: the difference and its quotient, the logarithm
    and the result are each rounded to fp32, by 2^-24 of a magnitude below M, uniformly (rms: 3^-1/2 of that), and S, a sum
    over many words, is good to 2^-23: twice M 2^-24 + 2^-23.  A loss is put together in 64 bits from that S, whatever its
    size, and rounded once."""
    binding, ctx = dx
    T = float(np.float32(T))
    g = torch.Generator(device="cuda").manual_seed(N)
    z = torch.randn((N, V), generator=g, device="cuda") * 2
    tokens = torch.randint(0, V, (N,), generator=g, device="cuda").to(torch.int32)
    got = binding.spec_token_logprobs(ctx, z, tokens, top_n=16, temperature=T)
    logq = torch.log_softmax(z.double() / T, 1)
    rms = lambda x: float(x.double().pow(2).mean().sqrt())  # noqa: E731
    for have, at in ((got["logprob"][:, None], tokens[:, None]), (got["top_logprobs"], got["top_ids"])):
        want = logq.gather(1, at.long())
        assert rms(have.double() - want) <= 2 * (float(want.abs().max()) * 2.0 ** -24 + 2.0 ** -23)
    lists = torch.log_softmax(z + torch.randn((N, V), generator=g, device="cuda"), 1).topk(16, dim=1)
    ids, lp = lists.indices.to(torch.int32), lists.values
    p = lp.double().exp()
    listed = logq.gather(1, ids.long())
    rest = 1 - p.sum(1)
    log_r = torch.log1p(-listed.exp().sum(1))
    tail = (p * (lp.double() - listed)).sum(1) + rest * (rest.log() - log_r)
    p = p / p.sum(1, keepdim=True)
    plain = (p * (p.log() - listed)).sum(1)
    for want, with_tail in ((tail, True), (plain, False)):
        have = binding.spec_distill_topk(ctx, z, ids, lp, tail=with_tail, temperature=T, grad=False)["loss"]
        assert rms(have.double() - want) <= 2.0 ** -23 + float(want.abs().max()) * 2.0 ** -24


@pytest.mark.parametrize("dtype", DTYPES)
def test_route_scores_that_64_bits_cannot_tell_apart_are_ties(dx, dtype):
    """Selection values are compared as they are in 64 bits: sigmoids of logits beyond 37 are all 1, scores far below their
    biases' last place add nothing to them.  Without a bias the logits themselves are compared."""
    binding, ctx = dx
    z = torch.full((4, 16), -2.0, device="cuda")
    z[0, 3:9] = torch.arange(40.0, 46.0, device="cuda")
    z[1, 3:9] = torch.arange(-60.0, -54.0, device="cuda")
    z[1, 9:], z[1, :3] = -80.0, -80.0
    z[2, 3:9] = torch.arange(1.0, 7.0, device="cuda")
    z = z.to(dtype)
    bias = torch.zeros(16, device="cuda")
    bias[3:9] = 0.25
    ids = binding.moe_route_tokens(ctx, z, 4, score_fn=1, select_bias=bias)["topk_ids"].tolist()
    assert ids[0] == [3, 4, 5, 6] and ids[1] == [3, 4, 5, 6] and ids[2] == [8, 7, 6, 5] and ids[3] == [3, 4, 5, 6]
    ids = binding.moe_route_tokens(ctx, z, 4, score_fn=1)["topk_ids"].tolist()
    assert ids[0] == ids[1] == ids[2] == [8, 7, 6, 5] and ids[3] == [0, 1, 2, 3]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("sigmoid", [False, True])
def test_route_grad_of_one_renormalised_gate_is_zero(dx, dtype, sigmoid):
    """The gate of the only selected expert is routed_scale whatever its logit: no gradient, not even a rounding of one."""
    binding, ctx = dx
    z = (torch.randn((500, 24), generator=torch.Generator(device="cuda").manual_seed(70), device="cuda") * 3).to(dtype)
    ids = binding.moe_route_tokens(ctx, z, 1, score_fn=int(sigmoid))["topk_ids"]
    dw = torch.randn((500, 1), generator=torch.Generator(device="cuda").manual_seed(71), device="cuda")
    got = binding.moe_route_tokens_backward(ctx, z, ids, dw, score_fn=int(sigmoid), norm_topk=1, routed_scale=2.446)
    assert not got.any()
