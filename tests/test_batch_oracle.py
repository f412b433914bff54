"""Pins of the checker of the batch operators (no GPU): torch's fp64 autograd, finite differences, closed forms; and the
refusals of the library's entry points, which come before anything touches a device."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import batch_oracle as B


@pytest.mark.parametrize("T", [1.0, 0.7, 2.0])
def test_token_logprobs_against_torch(T):
    rng = np.random.default_rng(1)
    z = rng.normal(0, 3, (4, 37))
    tok = np.array([3, 36, -1, 0])
    out = B.token_logprobs(z, tok, 5, T)
    lp = torch.log_softmax(torch.from_numpy(z) / T, dim=1)
    for t in range(4):
        assert abs(out["logprob"][t] - (0.0 if tok[t] < 0 else float(lp[t, tok[t]]))) < 1e-12
    ent = torch.distributions.Categorical(logits=lp).entropy()
    assert np.abs(out["entropy"] - ent.numpy()).max() < 1e-12
    assert np.array_equal(out["top_ids"], torch.topk(lp, 5, dim=1).indices.numpy())


def test_token_logprobs_of_a_uniform_row():
    out = B.token_logprobs(np.full((1, 64), -3.0), np.array([7]), 4, 1.0)
    assert abs(out["logprob"][0] + np.log(64)) < 1e-12 and abs(out["entropy"][0] - np.log(64)) < 1e-12
    assert out["top_ids"][0].tolist() == [0, 1, 2, 3]
    z = np.array([2.0, np.nan, 5.0, -np.inf, 5.0])
    assert B.order(z).tolist() == [2, 4, 0, 3, 1] == np.argsort(-z, kind="stable").tolist()


def _distill_torch(z, ids, lp, tail, T):
    """The loss built from torch operations, for autograd."""
    zt = torch.from_numpy(z).requires_grad_(True)
    logq = torch.log_softmax(zt / T, dim=1)
    loss = 0.0
    for t in range(z.shape[0]):
        use = ids[t] >= 0
        p = torch.from_numpy(np.exp(lp[t][use]))
        if not tail:
            p = p / p.sum()
        e = torch.from_numpy(ids[t][use])
        loss = loss + (p * (p.log() - logq[t, e])).sum()
        if tail:
            rest = 1.0 - p.sum()
            other = torch.ones(z.shape[1], dtype=torch.bool)
            other[e] = False
            loss = loss + rest * (rest.log() - torch.logsumexp(logq[t, other], 0))
    return float(loss.detach()), torch.autograd.grad(loss, zt)[0].numpy()


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("T", [1.0, 2.5])
def test_distill_against_autograd_and_differences(tail, T):
    rng = np.random.default_rng(2)
    z = rng.normal(0, 2, (3, 23))
    teacher = torch.log_softmax(torch.from_numpy(rng.normal(0, 2, (3, 23))), dim=1)
    lp, ids = teacher.topk(6, dim=1)
    lp, ids = lp.numpy(), ids.numpy().copy()
    ids[1, 4:] = -1
    loss, grad, _ = B.distill_topk(z, ids, lp, tail, T)
    total, g = _distill_torch(z, ids, lp, tail, T)
    assert abs(loss.sum() - total) < 1e-11 and np.abs(grad - g).max() < 1e-12
    for t, v in ((0, int(ids[0, 0])), (1, 5), (2, 22)):
        up, down = z.copy(), z.copy()
        up[t, v] += 1e-5
        down[t, v] -= 1e-5
        diff = (B.distill_topk(up, ids, lp, tail, T)[0][t] - B.distill_topk(down, ids, lp, tail, T)[0][t]) / 2e-5
        assert abs(diff - grad[t, v]) < 1e-8


def test_distill_weights_duplicates_and_empty_rows():
    rng = np.random.default_rng(3)
    z = rng.normal(0, 2, (3, 9))
    ids = np.array([[1, 2, 1], [-1, -1, -1], [4, 3, -1]])
    lp = np.log(np.array([[0.5, 0.3, 0.9], [0.1, 0.1, 0.1], [0.6, 0.2, 0.7]]))
    loss, grad, _ = B.distill_topk(z, ids, lp, True, 1.0, np.array([2.0, 1.0, 0.0]))
    once, g, _ = B.distill_topk(z[:1], ids[:1, :2], lp[:1, :2], True, 1.0)
    assert abs(loss[0] - once[0]) < 1e-15 and np.abs(grad[0] - 2 * g[0]).max() < 1e-15
    assert loss[1] == 0 and loss[2] == 0 and not grad[1:].any()


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("norm", [False, True])
def test_route_grad_against_autograd(sigmoid, norm):
    rng = np.random.default_rng(4)
    z = rng.normal(0, 1.5, (5, 12))
    ids, w, offsets, perm = B.route(z, 4, sigmoid, norm, 2.446)
    zt = torch.from_numpy(z).requires_grad_(True)
    r = torch.sigmoid(zt) if sigmoid else torch.softmax(zt, 1)
    wt = r.gather(1, torch.from_numpy(ids))
    wt = 2.446 * (wt / wt.sum(1, keepdim=True) if norm else wt)
    assert np.abs(w - wt.detach().numpy()).max() < 1e-12
    dw = rng.normal(0, 1, w.shape)
    want = torch.autograd.grad(wt, zt, torch.from_numpy(dw))[0].numpy()
    assert np.abs(B.route_grad(z, ids, dw, sigmoid, norm, 2.446)[0] - want).max() < 1e-12
    assert np.array_equal(ids, torch.topk(zt, 4, dim=1).indices.numpy())
    for e in range(12):
        assert [p // 4 for p in perm[offsets[e]:offsets[e + 1]]] == [t for t in range(5) if e in ids[t]]


def test_route_groups_by_enumeration():
    z = np.array([[0.0, 3.0, 2.9, 2.8, 1.0, 1.1, -np.inf, 4.0]])
    # pairs: (0, 3) (2.9, 2.8) (1, 1.1) (-inf, 4): by their largest value groups 3 and 1, by two sigmoid scores 1 and 2
    assert B.route(z, 2, True, True, 1.0, groups=4, keep=2)[0].tolist() == [[7, 1]]
    assert B.route(z, 3, True, True, 1.0, groups=4, keep=2, top2=True)[0].tolist() == [[2, 3, 5]]
    bias = np.array([5.0, 0, 0, 0, 0, 0, 9.0, 0])
    ids, w, _, _ = B.route(z, 2, True, True, 1.0, bias=bias)
    assert ids.tolist() == [[0, 7]]                       # the bias selects, the masked expert 6 stays out
    r = B.scores(z[0], True)
    assert np.abs(w[0] - r[[0, 7]] / r[[0, 7]].sum()).max() < 1e-12
    ids, w, _, _ = B.route(np.full((1, 4), -np.inf), 3, False, True, 1.0)
    assert ids.tolist() == [[0, 1, 2]] and not w.any()


# ---- refusals: they come before the context is used, so a blank stand-in for one will do -----------------------------
@pytest.fixture()
def lib():
    if torch.cuda.is_available():
        pytest.skip("host-only: with a device a call that is not refused would run on made-up addresses")
    from paper_2607_24434_b200 import binding
    blank = ctypes.create_string_buffer(4096)
    return binding, binding.load(), ctypes.addressof(blank), blank


def test_logprobs_refusals(lib):
    _, L, ctx, _ = lib

    def call(ctx=ctx, logits=4096, dtype=1, N=2, V=100, ld=100, tokens=4096, T=1.0, n=0, lp=4096, ent=4096, ids=None,
             tops=None):
        return L.spec_token_logprobs(ctx, logits, dtype, N, V, ld, tokens, T, n, lp, ent, ids, tops, None)

    assert call(ctx=None) == 1 and call(logits=None) == 1 and call(logits=4097) == 1 and call(dtype=2) == 1
    assert call(logits=4098, dtype=0) == 1
    assert call(N=-1) == 2 and call(V=0) == 2 and call(ld=99) == 2
    assert call(T=0.0) == 1 and call(T=-1.0) == 1 and call(T=float("nan")) == 1 and call(T=float("inf")) == 1
    assert call(n=-1) == 2 and call(n=101) == 2 and call(n=33) == 8 and call(n=4) == 1
    assert call(tokens=None) == 1 and call(lp=None) == 1 and call(tokens=None, lp=None, ent=None) == 1
    assert call(N=0, logits=None, tokens=None, lp=None, ent=None) == 0


def test_distill_refusals(lib):
    _, L, ctx, _ = lib

    def call(ctx=ctx, logits=4096, dtype=1, N=2, V=100, ld=100, ids=4096, lp=4096, k=4, tail=0, T=1.0, w=None, loss=4096,
             d=1 << 20, ld_d=100):
        return L.spec_distill_topk(ctx, logits, dtype, N, V, ld, ids, lp, k, tail, T, w, loss, d, ld_d, None)

    assert call(ctx=None) == 1 and call(logits=None) == 1 and call(dtype=3) == 1 and call(logits=4099) == 1
    assert call(N=-1) == 2 and call(V=0) == 2 and call(ld=50) == 2 and call(ld_d=99) == 2
    assert call(k=0) == 2 and call(k=129) == 8 and call(tail=2) == 1 and call(T=1e5) == 1
    assert call(ids=None) == 1 and call(lp=None) == 1 and call(loss=None, d=None) == 1
    assert call(d=4096, ld_d=101) == 1                     # the logits buffer at another pitch
    assert call(d=4096 + 200) == 1 and call(d=4096 + 398) == 1 and call(d=4096 - 2) == 1
    # between rows of a larger pitch: one element short of the room is refused (room enough goes on to the device)
    assert call(ld=199, ld_d=199, d=4096 + 200) == 1 and call(ld=200, ld_d=200, d=4096 + 198) == 1
    assert call(ld=200, ld_d=200, d=4096 + 200) == 3 and call(ld=200, ld_d=200, d=4096 - 200) == 3
    assert call(ld=200, ld_d=201, d=4096 + 200) == 1
    assert call(N=0x7ff00001) == 8
    assert call(d=4097) == 1
    assert call(N=0, logits=None, ids=None, lp=None, loss=None, d=None) == 0


def test_route_refusals(lib):
    binding, L, ctx, _ = lib

    def desc(E=64, k=6, score=0, norm=1, groups=1, keep=1, by=0):
        return ctypes.byref(binding.RouteDesc(E, k, score, norm, groups, keep, by, 1.0))

    def call(d, ctx=ctx, logits=4096, dtype=1, N=2, ld=64, bias=None, ids=4096, w=4096, off=4096, perm=4096):
        return L.moe_route_tokens(ctx, d, logits, dtype, N, ld, bias, ids, w, off, perm, None)

    assert call(desc(), ctx=None) == 1 and call(None) == 1 and call(desc(score=2)) == 1 and call(desc(by=2)) == 1
    assert call(desc(E=0)) == 2 and call(desc(k=0)) == 2 and call(desc(E=4, k=5)) == 2
    assert call(desc(E=257)) == 8 and call(desc(k=9)) == 8
    assert call(desc(groups=7)) == 2 and call(desc(groups=8, keep=9)) == 2 and call(desc(groups=8, keep=0)) == 2
    assert call(desc(groups=16, keep=1)) == 2               # four experts stay, six are asked for
    assert call(desc(groups=64, keep=8)) == 8
    assert call(desc(), ld=63) == 2 and call(desc(), N=-1) == 2 and call(desc(), dtype=2) == 1
    assert call(desc(), logits=None) == 1
    assert call(desc(), N=1 << 30) == 8                     # more pairs than 32-bit positions
    assert call(desc(), off=None) == 1 and call(desc(), perm=None) == 1 and call(desc(), ids=None) == 1 and call(desc(), w=None) == 1

    def back(d, ctx=ctx, logits=4096, N=2, ld=64, ids=4096, dw=4096, out=1 << 20, ld_d=64):
        return L.moe_route_tokens_backward(ctx, d, logits, 1, N, ld, ids, dw, out, ld_d, None)

    assert back(desc(), ctx=None) == 1 and back(None) == 1 and back(desc(score=-1)) == 1 and back(desc(E=300)) == 8
    assert back(desc(), logits=None) == 1 and back(desc(), ids=None) == 1 and back(desc(), dw=None) == 1
    assert back(desc(), out=None) == 1 and back(desc(), ld_d=10) == 2
    assert back(desc(), out=4096) == 1 and back(desc(), out=4096 + 128) == 1    # over the logits
    assert back(desc(), N=0, logits=None, ids=None, dw=None, out=None) == 0


def test_binding_checks_what_a_pointer_cannot_show():
    from paper_2607_24434_b200 import binding

    class Ctx:
        device = 0

    with pytest.raises(ValueError):
        binding.spec_token_logprobs(Ctx(), torch.zeros(2, 8), torch.zeros(2, dtype=torch.int32))      # not on the GPU
    with pytest.raises(ValueError):
        binding.moe_route_tokens(Ctx(), torch.zeros(2, 8), 2)
    assert ctypes.sizeof(binding.RouteDesc) == 8 * 4


def test_distill_lists_outside_the_range_of_exp():
    rng = np.random.default_rng(7)
    z = rng.normal(0, 2, (3, 30))
    ids = np.tile(np.arange(5), (3, 1))
    base = -rng.integers(0, 160, 5) / 16.0
    lp = np.stack([base, base - 1024.0, base + 1024.0])
    loss, grad, _ = B.distill_topk(np.tile(z[:1], (3, 1)), ids, lp, False, 1.0)
    assert np.isfinite(loss).all() and loss[0] > 0 and (loss == loss[0]).all() and (grad == grad[0]).all()
