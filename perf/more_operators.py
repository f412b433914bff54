"""Measured cases of the operators that take a batch of tokens through routed experts and into the loss, and back.

  experts      products of rows, sorted by expert, with their experts' matrices (or the transposed ones)
  dw           the gradient of those matrices
  swiglu       gate and up products of an expert with the activation, and the gradient through the down product
  combine      the weighted sum of a token's experts, and its gradient
  head         cross entropy of hidden rows against a vocabulary, with the gradients of the rows and of the head

Rows are (token, choice) pairs: pair p = t * k + j; ``perm`` lists the pairs by expert, ``offsets`` where each expert
begins.  ``run`` computes an operator in elementary torch operations (``own`` false) or through the library (``own`` true).
"""
import math

import torch

own = False

_DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
_SIZE = {"fp32": 4, "bf16": 2}


# ---- cases ---------------------------------------------------------------------------------------------------------
def listed():
    return [
        # down product of one decoded token: six matrices of 64, latency and weight bytes
        dict(name="experts-token", op="experts", N=1, k=6, E=64, n=2048, m=1408, transposed=False, gather=False,
             scatter=True, out="bf16"),
        # training batch: gradient of the experts' input through both halves of the gate/up matrix
        dict(name="experts-batch", op="experts", N=16384, k=6, E=64, n=2816, m=2048, transposed=True, gather=False,
             scatter=True, out="bf16"),
        # training batch: gate/up weight gradients, in fp32 as an optimiser's master gradients are
        dict(name="dw-batch", op="dw", N=8192, k=6, E=64, n=2816, m=2048, gather_dy=False, gather_x=True, out="fp32"),
        # fine-grained experts, few tokens: most groups have a handful of rows, some none
        dict(name="dw-ragged", op="dw", N=203, k=3, E=130, n=1000, m=520, gather_dy=True, gather_x=False, out="bf16"),
        # one decoded token through six experts' gate and up matrices
        dict(name="swiglu-token", op="swiglu", N=1, k=6, E=64, H=2048, I=1408, save=False),
        # training batch, gate and up kept for the backward pass
        dict(name="swiglu-batch", op="swiglu", N=16384, k=6, E=64, H=2048, I=1408, save=True),
        # a drafter updated on one prompt: every expert's weights are read for some sixty rows
        dict(name="swiglu-grad-prompt", op="swiglu_grad", N=700, k=6, E=64, H=2048, I=1408),
        # training batch, backward
        dict(name="swiglu-grad-batch", op="swiglu_grad", N=8192, k=6, E=64, H=2048, I=1408),
        # training batch: a token's six experts are added
        dict(name="combine-batch", op="combine", N=16384, k=6, H=2048, weighted=True, grad=False, dtype="bf16"),
        # a smaller one backwards, fp32 rows
        dict(name="combine-grad", op="combine", N=4999, k=4, H=1000, weighted=True, grad=True, dtype="fp32"),
        # the block that was just verified, head frozen: the head is read, sixteen rows of gradient come back
        dict(name="head-block", op="head", N=16, V=102400, H=2048, ragged=False, dh=True, dw=False),
        # training batch with a padded end, gradients of rows and head
        dict(name="head-batch", op="head", N=4096, V=102400, H=2048, ragged=True, dh=True, dw=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _log_8(rng, lo, hi):
    return 8 * _log_int(rng, lo // 8, hi // 8)


def draw(rng):
    op = rng.choice(["experts", "dw", "swiglu", "swiglu_grad", "combine", "head"])
    if op == "head":
        H = _log_8(rng, 64, 2048)
        V = _log_int(rng, 1000, 163840)
        if rng.random() < 0.5:
            V += (V % 2 == 0)
        dh = rng.random() < 0.7
        most = min(8192, int(4096 * 102400 * 2048 / (V * H)))
        return dict(op=op, N=_log_int(rng, 1, max(2, most)), V=V, H=H, ragged=rng.random() < 0.5, dh=dh,
                    dw=dh and rng.random() < 0.5)
    k = rng.randint(1, 8)
    if op == "combine":
        return dict(op=op, N=_log_int(rng, 1, 98304 // k), k=k, H=_log_8(rng, 64, 2048), weighted=rng.random() < 0.8,
                    grad=rng.random() < 0.4, dtype=rng.choice(["fp32", "bf16"]))
    E = max(k, _log_int(rng, 1, 130))
    a, b = _log_8(rng, 64, 2816), _log_8(rng, 64, 2048)
    while E * a * b > 64 * 2816 * 2048:
        E = max(k, E // 2)
    N = _log_int(rng, 1, 98304 // k)
    out = rng.choice(["bf16", "bf16", "fp32"])
    if op == "experts":
        return dict(op=op, N=N, k=k, E=E, n=a, m=b, transposed=rng.random() < 0.5, gather=rng.random() < 0.5,
                    scatter=rng.random() < 0.5, out=out)
    if op == "dw":
        return dict(op=op, N=N, k=k, E=E, n=a, m=b, gather_dy=rng.random() < 0.5, gather_x=rng.random() < 0.5, out=out)
    H, I = b, max(8, a // 16 * 8)
    if op == "swiglu":
        return dict(op=op, N=N, k=k, E=E, H=H, I=I, save=rng.random() < 0.5)
    return dict(op=op, N=N, k=k, E=E, H=H, I=I)


def _live_experts(c):
    """Experts that some row selects, about: k of E distinct ones per token."""
    return min(c["E"], round(c["E"] * (1.0 - (1.0 - c["k"] / c["E"]) ** c["N"])))


def work(case):
    c, N = case, case["N"]
    op = c["op"]
    if op == "head":
        grads = int(c["dh"]) + int(c["dw"])
        byt = c["V"] * c["H"] * 2 * (1 + int(c["dw"])) + N * c["H"] * 2 * (1 + int(c["dh"])) + N * 12
        live = N - (N // 8 if c["ragged"] else 0) - N // 9            # rows with a token and a weight
        return {"bytes": byt, "flops": 2 * max(1, live) * c["V"] * c["H"] * (1 + grads)}
    P = N * c["k"]
    if op == "combine":
        es, H = _SIZE[c["dtype"]], c["H"]
        if c["grad"]:
            return {"bytes": es * H * (N + 2 * P) + P * 8, "flops": 3 * P * H}
        return {"bytes": es * H * (N + P) + P * 4, "flops": 2 * P * H}
    if op == "dw":
        rows = (N if c["gather_dy"] else P) * c["n"] + (N if c["gather_x"] else P) * c["m"]
        return {"bytes": 2 * rows + c["E"] * c["n"] * c["m"] * _SIZE[c["out"]], "flops": 2 * P * c["n"] * c["m"]}
    live = _live_experts(c)
    if op == "experts":
        n_in, n_out = (c["n"], c["m"]) if c["transposed"] else (c["m"], c["n"])
        return {"bytes": 2 * live * c["n"] * c["m"] + 2 * (N if c["gather"] else P) * n_in + P * n_out * _SIZE[c["out"]],
                "flops": 2 * P * c["n"] * c["m"]}
    H, I = c["H"], c["I"]
    if op == "swiglu":
        return {"bytes": 4 * live * I * H + 2 * N * H + 2 * P * I * (3 if c["save"] else 1), "flops": 4 * P * I * H}
    # the down matrices, the tokens' gradients, gate and up in; their gradients and the weighted products out
    return {"bytes": 2 * live * I * H + 2 * N * H + 2 * P * I * 5 + P * 8, "flops": 2 * P * I * H}


# ---- inputs --------------------------------------------------------------------------------------------------------
_context = []


def _own():
    from paper_2607_24434_b200 import binding
    if not _context:
        _context.append(binding.Context(torch.cuda.current_device()))
    return binding, _context[0]


def _randn(g, *shape, scale=1.0):
    return torch.randn(shape, generator=g, device="cuda").mul_(scale).to(torch.bfloat16)


def _routing(g, s, N, k, E):
    """k distinct experts per token, some experts liked more than others; pairs sorted by expert."""
    score = torch.randn((N, E), generator=g, device="cuda") + 0.3 * torch.randn((E,), generator=g, device="cuda")
    ids = score.topk(k, dim=1).indices.reshape(-1)
    s["perm"] = torch.sort(ids, stable=True).indices.to(torch.int32)
    counts = torch.bincount(ids, minlength=E)
    s["offsets"] = torch.cat([counts.new_zeros(1), counts.cumsum(0)]).to(torch.int32)
    s["most"] = int(counts.max())                                       # rows of the largest group
    w = torch.rand((N, k), generator=g, device="cuda") + 0.1
    s["topk_w"] = w / w.sum(dim=1, keepdim=True)


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device="cuda").manual_seed(int(seed) * 6151 + 29)
    s = {"case": c}
    N, op = c["N"], c["op"]
    if op == "head":
        V, H = c["V"], c["H"]
        s["W"] = _randn(g, V, H, scale=0.02)
        t = torch.randint(0, V, (N,), generator=g, device="cuda")
        # the model likes the right word more or less: its logit stands up to some twelve above the others
        lift = torch.rand((N, 1), generator=g, device="cuda") * (12.0 / (4e-4 * H))
        s["h"] = (torch.randn((N, H), generator=g, device="cuda") + lift * s["W"][t].float()).to(torch.bfloat16)
        t = t.to(torch.int32)
        t[8::9] = -1                                                   # rows without a next token
        s["targets"] = t
        s["weight"] = None
        if c["ragged"]:
            w = torch.rand((N,), generator=g, device="cuda") + 0.5
            w[N - N // 8:] = 0.0                                       # the padded end of the batch
            s["weight"] = w
    elif op == "combine":
        P, H, dt = N * c["k"], c["H"], _DTYPES[c["dtype"]]
        s["z"] = torch.randn((P, H), generator=g, device="cuda").to(dt)
        s["topk_w"] = None
        if c["weighted"]:
            w = torch.rand((N, c["k"]), generator=g, device="cuda") + 0.05
            s["topk_w"] = w / w.sum(dim=1, keepdim=True)
        if c["grad"]:
            s["dy"] = torch.randn((N, H), generator=g, device="cuda").to(dt)
    else:
        k, E = c["k"], c["E"]
        P = N * k
        _routing(g, s, N, k, E)
        if op == "experts":
            s["w"] = _randn(g, E, c["n"], c["m"], scale=0.02)
            s["x"] = _randn(g, N if c["gather"] else P, c["n"] if c["transposed"] else c["m"])
        elif op == "dw":
            s["dy"] = _randn(g, N if c["gather_dy"] else P, c["n"], scale=0.01)
            s["x"] = _randn(g, N if c["gather_x"] else P, c["m"])
        elif op == "swiglu":
            s["x"] = _randn(g, N, c["H"])
            s["w"] = _randn(g, E, 2 * c["I"], c["H"], scale=0.02)      # gate rows, then up rows
        else:
            s["dy"] = _randn(g, N, c["H"], scale=0.01)
            s["w"] = _randn(g, E, c["H"], c["I"], scale=0.02)
            s["gate_up"] = _randn(g, P, 2 * c["I"])
    if own:
        _own()
    return s


# ---- plain forms ---------------------------------------------------------------------------------------------------
def _expert_of_row(s, P):
    return torch.searchsorted(s["offsets"][1:], torch.arange(P, device="cuda", dtype=torch.int32), right=True)


def _padded(s, rows):
    """[E, most, width]: every expert's rows, zeros behind them."""
    at = s["offsets"][:-1, None].long() + torch.arange(s["most"], device="cuda")
    inside = at < s["offsets"][1:, None]
    return rows[at.clamp(max=rows.shape[0] - 1)] * inside[:, :, None]


def _product(s, rows, w):
    """w[e of the row] times the row, for rows in sorted order."""
    P, E = rows.shape[0], w.shape[0]
    e = _expert_of_row(s, P)
    if P < E:                                                          # few rows: each with its own matrix
        return torch.matmul(w[e].float(), rows[:, :, None])[:, :, 0]
    y = torch.bmm(_padded(s, rows), w.float().transpose(1, 2))
    place = e * s["most"] + torch.arange(P, device="cuda") - s["offsets"][e]
    return y.view(-1, y.shape[2])[place]


def _plain_experts(s):
    c = s["case"]
    pair = s["perm"].long()
    rows = s["x"][pair // c["k"]] if c["gather"] else s["x"]
    w = s["w"].transpose(1, 2) if c["transposed"] else s["w"]
    y = _product(s, rows.float(), w).to(_DTYPES[c["out"]])
    return torch.empty_like(y).index_copy_(0, pair, y) if c["scatter"] else y


def _plain_dw(s):
    c = s["case"]
    pair = s["perm"].long()
    dy = s["dy"][pair // c["k"]] if c["gather_dy"] else s["dy"]
    x = s["x"][pair // c["k"]] if c["gather_x"] else s["x"]
    return torch.bmm(_padded(s, dy.float()).transpose(1, 2), _padded(s, x.float())).to(_DTYPES[c["out"]])


def _plain_swiglu(s):
    c = s["case"]
    rows = s["x"][s["perm"].long() // c["k"]].float()
    gu = _product(s, rows, s["w"])
    gate, up = gu[:, :c["I"]], gu[:, c["I"]:]
    out = {"act": (gate / (1.0 + torch.exp(-gate)) * up).to(torch.bfloat16)}
    if c["save"]:
        out["gate_up"] = gu.to(torch.bfloat16)
    return out


def _plain_swiglu_grad(s):
    c = s["case"]
    pair = s["perm"].long()
    a = _product(s, s["dy"][pair // c["k"]].float(), s["w"].transpose(1, 2))
    gate, up = s["gate_up"][:, :c["I"]].float(), s["gate_up"][:, c["I"]:].float()
    sig = 1.0 / (1.0 + torch.exp(-gate))
    act = gate * sig * up
    w = s["topk_w"].reshape(-1)
    d_w = torch.empty_like(w).index_copy_(0, pair, (a * act).sum(dim=1))
    row_w = w[pair][:, None]
    d = a * row_w
    d_gate = d * up * sig * (1.0 + gate * (1.0 - sig))
    d_up = d * gate * sig
    return {"d_gate_up": torch.cat([d_gate, d_up], dim=1).to(torch.bfloat16), "act_w": (row_w * act).to(torch.bfloat16),
            "d_topk_w": d_w.view(c["N"], c["k"])}


def _plain_combine(s):
    c = s["case"]
    z = s["z"].float().view(c["N"], c["k"], c["H"])
    w = s["topk_w"]
    if c["grad"]:
        dy = s["dy"].float()[:, None, :]
        dz = (dy * w[:, :, None] if w is not None else dy.expand(-1, c["k"], -1)).reshape(-1, c["H"])
        out = {"dz": dz.to(s["z"].dtype)}
        if w is not None:
            out["d_topk_w"] = (z * dy).sum(dim=2)
        return out
    return (z if w is None else z * w[:, :, None]).sum(dim=1).to(s["z"].dtype)


def _plain_head(s):
    c = s["case"]
    h, W = s["h"].float(), s["W"].float()
    z = h @ W.t()
    top = z.max(dim=1, keepdim=True).values
    e = torch.exp(z - top)
    total = e.sum(dim=1, keepdim=True, dtype=torch.float64)
    t = s["targets"].long()
    live = t >= 0
    if s["weight"] is not None:
        live = live & (s["weight"] != 0)
    at = t.clamp(min=0)[:, None]
    loss = torch.log(total) - (z.gather(1, at).double() - top.double())
    out = {"loss": torch.where(live, loss[:, 0], torch.zeros_like(loss[:, 0])).float()}
    if c["dh"]:
        d = e.div_(total.float())
        d.scatter_add_(1, at, torch.full_like(at, -1.0, dtype=torch.float32))
        scale = live.float() if s["weight"] is None else torch.where(live, s["weight"], torch.zeros_like(s["weight"]))
        d *= scale[:, None]
        out["dh"] = (d @ W).to(torch.bfloat16)
        if c["dw"]:
            out["dW"] = (d.t() @ h).to(torch.bfloat16)
    return out


_PLAIN = {"experts": _plain_experts, "dw": _plain_dw, "swiglu": _plain_swiglu, "swiglu_grad": _plain_swiglu_grad,
          "combine": _plain_combine, "head": _plain_head}


# ---- one pass ------------------------------------------------------------------------------------------------------
def run(state):
    s, c = state, state["case"]
    op = c["op"]
    if not own:
        return _PLAIN[op](s)
    binding, ctx = _own()
    if op == "experts":
        return binding.moe_grouped_mm(ctx, s["x"], s["w"], s["offsets"], transposed=c["transposed"],
                                      gather=s["perm"] if c["gather"] else None, gather_div=c["k"] if c["gather"] else 1,
                                      scatter=s["perm"] if c["scatter"] else None, out_dtype=_DTYPES[c["out"]])
    if op == "dw":
        return binding.moe_grouped_mm_dw(ctx, s["dy"], s["x"], s["offsets"],
                                         gather_dy=s["perm"] if c["gather_dy"] else None, dy_div=c["k"],
                                         gather_x=s["perm"] if c["gather_x"] else None, x_div=c["k"],
                                         out_dtype=_DTYPES[c["out"]])
    if op == "swiglu":
        return binding.moe_grouped_swiglu(ctx, s["x"], s["w"], s["offsets"], gather=s["perm"], gather_div=c["k"],
                                          save=c["save"])
    if op == "swiglu_grad":
        return binding.moe_grouped_swiglu_backward(ctx, s["dy"], s["w"], s["gate_up"], s["topk_w"], s["offsets"],
                                                   gather=s["perm"], gather_div=c["k"])
    if op == "combine":
        if c["grad"]:
            return binding.moe_combine_tokens_backward(ctx, s["dy"], s["z"], s["topk_w"], top_k=c["k"])
        return binding.moe_combine_tokens(ctx, s["z"], s["topk_w"], top_k=c["k"])
    return binding.spec_head_loss(ctx, s["h"], s["W"], s["targets"], row_weight=s["weight"], grad=c["dh"],
                                  grad_weight=c["dw"])


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------
def _groups(s):
    """(expert, its pairs, where they stand in the sorted order)"""
    ends = s["offsets"].tolist()
    return [(e, s["perm"][a:b].long(), slice(a, b)) for e, (a, b) in enumerate(zip(ends, ends[1:])) if b > a]


def _exact_rows(s, c):
    P = c["N"] * c["k"]
    new = {"dtype": torch.float64, "device": "cuda"}
    if c["op"] == "experts":
        y = torch.zeros((P, c["m"] if c["transposed"] else c["n"]), **new)
        for e, pairs, here in _groups(s):
            src = s["x"][torch.div(pairs, c["k"], rounding_mode="floor")] if c["gather"] else s["x"][here]
            m = s["w"][e].double()
            y[pairs if c["scatter"] else here] = torch.einsum("rn,nm->rm" if c["transposed"] else "rm,nm->rn", src.double(), m)
        return y
    if c["op"] == "dw":
        out = torch.zeros((c["E"], c["n"], c["m"]), **new)
        for e, pairs, here in _groups(s):
            tokens = torch.div(pairs, c["k"], rounding_mode="floor")
            a, b = s["dy"][tokens if c["gather_dy"] else here], s["x"][tokens if c["gather_x"] else here]
            out[e] = torch.einsum("rn,rm->nm", a.double(), b.double())
        return out
    I = c["I"]
    if c["op"] == "swiglu":
        out = {"act": torch.zeros((P, I), **new)}
        if c["save"]:
            out["gate_up"] = torch.zeros((P, 2 * I), **new)
        for e, pairs, here in _groups(s):
            gu = s["x"][torch.div(pairs, c["k"], rounding_mode="floor")].double() @ s["w"][e].double().t()
            out["act"][here] = torch.nn.functional.silu(gu[:, :I]) * gu[:, I:]
            if c["save"]:
                out["gate_up"][here] = gu
        return out
    out = {"d_gate_up": torch.zeros((P, 2 * I), **new), "act_w": torch.zeros((P, I), **new),
           "d_topk_w": torch.zeros((c["N"] * c["k"],), **new)}
    flat_w = s["topk_w"].reshape(-1).double()
    for e, pairs, here in _groups(s):
        a = s["dy"][torch.div(pairs, c["k"], rounding_mode="floor")].double() @ s["w"][e].double()
        gate, up = s["gate_up"][here].double().chunk(2, dim=1)
        sg = torch.sigmoid(gate)
        w = flat_w[pairs, None]
        out["act_w"][here] = w * gate * sg * up
        out["d_topk_w"][pairs] = torch.einsum("ri,ri->r", a, gate * sg * up)
        out["d_gate_up"][here, :I] = w * a * up * (sg + gate * sg * (1 - sg))
        out["d_gate_up"][here, I:] = w * a * gate * sg
    out["d_topk_w"] = out["d_topk_w"].view(c["N"], c["k"])
    return out


def _exact_combine(s, c):
    N, k = c["N"], c["k"]
    w = torch.ones((N, k), device="cuda", dtype=torch.float64) if s["topk_w"] is None else s["topk_w"].double()
    if not c["grad"]:
        y = torch.zeros((N, c["H"]), device="cuda", dtype=torch.float64)
        for j in range(k):
            y += w[:, j:j + 1] * s["z"][j::k].double()
        return y
    out = {"dz": torch.repeat_interleave(s["dy"].double(), k, dim=0) * w.reshape(-1, 1)}
    if s["topk_w"] is not None:
        out["d_topk_w"] = torch.stack([torch.einsum("th,th->t", s["z"][j::k].double(), s["dy"].double())
                                       for j in range(k)], dim=1)
    return out


def _exact_head(s, c):
    N, V = c["N"], c["V"]
    W = s["W"].double()
    scale = torch.ones((N,), device="cuda", dtype=torch.float64) if s["weight"] is None else s["weight"].double()
    scale = torch.where(s["targets"] < 0, torch.zeros_like(scale), scale)
    losses, dh = [], []
    dW = torch.zeros((V, c["H"]), device="cuda", dtype=torch.float64) if c["dw"] else None
    step = max(1, (1 << 27) // V)
    for a in range(0, N, step):
        rows = slice(a, min(N, a + step))
        h = s["h"][rows].double()
        logp = torch.log_softmax(h @ W.t(), dim=1)
        t = s["targets"][rows].long()
        losses.append(torch.where(scale[rows] != 0, -logp.gather(1, t.clamp_min(0)[:, None])[:, 0], torch.zeros_like(scale[rows])))
        if c["dh"]:
            d = logp.exp_()
            on = torch.nonzero(t >= 0)[:, 0]
            d[on, t[on]] -= 1.0
            d *= scale[rows, None]
            dh.append(d @ W)
            if c["dw"]:
                dW.addmm_(d.t(), h)
    out = {"loss": torch.cat(losses)}
    if c["dh"]:
        out["dh"] = torch.cat(dh)
    if c["dw"]:
        out["dW"] = dW
    return out


def exact(case, seed):
    s = prepare(case, seed)
    c = s["case"]
    if c["op"] == "head":
        return _exact_head(s, c)
    return _exact_combine(s, c) if c["op"] == "combine" else _exact_rows(s, c)
