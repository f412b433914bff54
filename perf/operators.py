"""Measured cases of the operators that score, distil and route whole batches of tokens.

  logprobs    log probabilities of given tokens, entropy and the most likely alternatives, from rows of logits
  distill     distillation from a teacher's top log probabilities: loss per row and the gradient of the logits
  route       expert selection for a batch of tokens: scores, balance bias, groups, top-k, gate weights, permutation
  route_grad  the gradient of the gate weights with respect to the router logits

``run`` computes an operator in elementary torch operations (``own`` false) or through the library (``own`` true).
"""
import math

import torch

own = False

NEG_INF = float("-inf")
_DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
_SIZE = {"fp32": 4, "bf16": 2}


# ---- cases ---------------------------------------------------------------------------------------------------------
def listed():
    return [
        # the token a decode step has just emitted, with eight alternatives: latency counts
        dict(name="logprobs-token", op="logprobs", N=1, V=102400, pad=0, dtype="bf16", top=8, T=1.0, banned=False),
        # a full verification block (16 rows) of the larger vocabulary, sampled at a temperature, some words banned
        dict(name="logprobs-block", op="logprobs", N=16, V=163840, pad=0, dtype="fp32", top=20, T=0.8, banned=True),
        # a prompt scored token by token (evaluation of a draft, recording of teacher signal)
        dict(name="logprobs-prompt", op="logprobs", N=2048, V=102400, pad=0, dtype="bf16", top=20, T=1.0, banned=False),
        # drafter updated on the block that was just verified: a handful of rows
        dict(name="distill-block", op="distill", N=8, V=102400, pad=0, dtype="bf16", k=8, T=1.0, tail=False,
             ragged=False, grad=True),
        # training batch of the drafter, recorded top 64, renormalised over the list
        dict(name="distill-batch", op="distill", N=2048, V=102400, pad=0, dtype="bf16", k=64, T=1.0, tail=False,
             ragged=False, grad=True),
        # fp32 logits, larger vocabulary, short ragged lists with the rest of the mass in one bucket, padded rows
        dict(name="distill-tail", op="distill", N=1024, V=163840, pad=0, dtype="fp32", k=20, T=2.0, tail=True,
             ragged=True, grad=True),
        # evaluation of a drafter: loss alone, odd vocabulary in rows of an odd pitch
        dict(name="distill-eval", op="distill", N=777, V=32003, pad=2, dtype="bf16", k=33, T=1.0, tail=True,
             ragged=True, grad=False),
        # one verification block of the 64-expert layer
        dict(name="route-block", op="route", N=4, E=64, k=6, score="softmax", norm=True, scale=1.0, bias=False,
             groups=1, keep=1, top2=False, dtype="fp32"),
        # a prompt / training batch through the sigmoid router with routed scale 2.446 and a balance bias
        dict(name="route-batch", op="route", N=16384, E=64, k=6, score="sigmoid", norm=True, scale=2.446, bias=True,
             groups=1, keep=1, top2=False, dtype="fp32"),
        # the widest router the library takes, limited to four of eight expert groups
        dict(name="route-groups", op="route", N=32768, E=256, k=8, score="sigmoid", norm=True, scale=2.446, bias=True,
             groups=8, keep=4, top2=True, dtype="bf16"),
        # training direction, softmax gates that are not renormalised: every expert's logit gets a gradient
        dict(name="route-grad-batch", op="route_grad", N=16384, E=64, k=6, score="softmax", norm=False, scale=1.0,
             dtype="fp32"),
        # training direction of the widest router
        dict(name="route-grad-wide", op="route_grad", N=65536, E=256, k=8, score="sigmoid", norm=True, scale=2.446,
             dtype="bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["logprobs", "distill", "route", "route_grad"])
    dtype = rng.choice(["fp32", "bf16"])
    if op in ("logprobs", "distill"):
        V = _log_int(rng, 1000, 163840)
        if rng.random() < 0.5:
            V += (V % 2 == 0)
        limit = (2048 * 102400 if dtype == "bf16" else 1024 * 102400) // V
        N = _log_int(rng, 1, min(4096, max(1, limit)))
        pad = rng.choice([0, 0, 1, 8, 13])
        T = rng.choice([1.0, 1.0, 0.7, 2.0])
        if op == "logprobs":
            return dict(op=op, N=N, V=V, pad=pad, dtype=dtype, top=rng.choice([0, 1, 5, 8, 20, 32]), T=T,
                        banned=rng.random() < 0.5)
        return dict(op=op, N=N, V=V, pad=pad, dtype=dtype, k=rng.randint(1, 64), T=T, tail=rng.random() < 0.5,
                    ragged=rng.random() < 0.5, grad=rng.random() < 0.75)
    score = rng.choice(["softmax", "sigmoid"])
    if op == "route":
        groups = rng.choice([1, 1, 2, 4, 8])
        E = groups * rng.randint(max(2, 16 // groups), 256 // groups)
        keep = rng.randint((groups + 1) // 2, groups)
        k = rng.randint(1, min(8, keep * (E // groups)))
        return dict(op=op, N=_log_int(rng, 1, 32768), E=E, k=k, score=score, norm=rng.random() < 0.7,
                    scale=rng.choice([1.0, 2.446]), bias=rng.random() < 0.6, groups=groups, keep=keep,
                    top2=groups > 1 and rng.random() < 0.5, dtype=dtype)
    E = rng.randint(8, 256)
    return dict(op=op, N=_log_int(rng, 1, 32768), E=E, k=rng.randint(1, 8), score=score, norm=rng.random() < 0.5,
                scale=rng.choice([1.0, 2.446]), dtype=dtype)


def work(case):
    c, N = case, case["N"]
    if c["op"] == "logprobs":
        # every logit read once; per logit a difference, an exponential and two accumulations
        return {"bytes": N * c["V"] * _SIZE[c["dtype"]] + N * (4 + 8 + 8 * c["top"]), "flops": 5 * N * c["V"]}
    if c["op"] == "distill":
        live = N - (N // 8 if c["ragged"] else 0)             # rows of weight zero are not read
        es = _SIZE[c["dtype"]]
        out = N * c["V"] * es if c["grad"] else 0             # ... but their gradient is written (zeros)
        return {"bytes": live * c["V"] * es + out + N * (8 * c["k"] + 8),
                "flops": live * c["V"] * (6 if c["grad"] else 3)}
    es = _SIZE[c["dtype"]]
    if c["op"] == "route":
        return {"bytes": N * c["E"] * es + 4 * c["E"] * (2 if c["bias"] else 1) + N * c["k"] * 12,
                "flops": N * c["E"] * (4 + c["k"])}
    return {"bytes": 2 * N * c["E"] * es + N * c["k"] * 8, "flops": N * c["E"] * 8}


# ---- inputs --------------------------------------------------------------------------------------------------------
def _logits(g, N, V, pad, dtype):
    """Rows that look like a language model's: a broad floor, a few dozen words far above it."""
    z = torch.randn((N, V + pad), generator=g, device="cuda").mul_(1.7)
    hot = torch.randint(0, V, (N, 40), generator=g, device="cuda")
    lift = 14.0 - 3.0 * torch.log1p(torch.arange(40, device="cuda", dtype=torch.float32))
    z.scatter_add_(1, hot, lift.expand(N, 40).contiguous())
    return z.to(_DTYPES[dtype])


_context = []


def _own():
    from paper_2607_24434_b200 import binding
    if not _context:
        _context.append(binding.Context(torch.cuda.current_device()))
    return binding, _context[0]


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 11)
    s = {"case": c}
    N = c["N"]
    if c["op"] == "logprobs":
        z = _logits(g, N, c["V"], c["pad"], c["dtype"])
        if c["banned"]:
            ban = torch.randint(0, c["V"], (max(1, c["V"] // 500),), generator=g, device="cuda")
            z[:, ban] = NEG_INF
        z = z[:, :c["V"]]
        s["logits"] = z
        # mostly likely words, as a model's own text has them; every ninth row has no token (padding)
        likely = z.float().topk(min(4, c["V"]), dim=1).indices
        pick = torch.randint(0, likely.shape[1], (N, 1), generator=g, device="cuda")
        tok = likely.gather(1, pick).squeeze(1).to(torch.int32)
        tok[8::9] = -1
        s["tokens"] = tok
    elif c["op"] == "distill":
        z = _logits(g, N, c["V"], c["pad"], c["dtype"])
        s["logits"] = z[:, :c["V"]]
        k = min(c["k"], c["V"])
        teacher = s["logits"].float() * (0.9 / c["T"])
        teacher += torch.randn((N, c["V"]), generator=g, device="cuda")
        lp, ids = torch.log_softmax(teacher, dim=1).topk(k, dim=1)
        ids = ids.to(torch.int32)
        s["weight"] = None
        if c["ragged"]:
            length = torch.randint(0, k + 1, (N, 1), generator=g, device="cuda")
            length[0] = k
            ids = torch.where(torch.arange(k, device="cuda") < length, ids, torch.full_like(ids, -1))
            w = torch.rand((N,), generator=g, device="cuda") + 0.5
            w[N - N // 8:] = 0.0                               # the padded end of the batch
            s["weight"] = w
        s["teacher_ids"], s["teacher_logprobs"] = ids.contiguous(), lp.contiguous()
    elif c["op"] == "route":
        s["logits"] = torch.randn((N, c["E"]), generator=g, device="cuda").mul_(1.3).to(_DTYPES[c["dtype"]])
        s["bias"] = torch.randn((c["E"],), generator=g, device="cuda").mul_(0.05) if c["bias"] else None
    else:
        s["logits"] = torch.randn((N, c["E"]), generator=g, device="cuda").mul_(1.3).to(_DTYPES[c["dtype"]])
        s["topk_ids"] = s["logits"].float().topk(c["k"], dim=1).indices.to(torch.int32).contiguous()
        s["d_topk_w"] = torch.randn((N, c["k"]), generator=g, device="cuda")
    if own:
        _own()
    return s


# ---- plain forms ---------------------------------------------------------------------------------------------------
def _top_keys(z, n):
    """The n largest entries of each row, ties to the lower index: sorted on (value, reversed index) in one integer."""
    bits = (z + 0.0).view(torch.int32).to(torch.int64)
    bits = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits)      # a float's bits in the order of its value
    last = z.shape[1] - 1
    key = bits * (1 << 31) + (last - torch.arange(z.shape[1], device=z.device))
    return last - (key.topk(n, dim=1).values & ((1 << 31) - 1))


def _plain_logprobs(s):
    c = s["case"]
    z = s["logits"].float()
    x = z / c["T"]
    m = x.max(dim=1, keepdim=True).values
    u = x - m
    e = torch.exp(u)
    total = e.sum(dim=1, keepdim=True)
    log_total = torch.log(total)
    entropy = log_total - torch.where(e > 0, u * e, torch.zeros_like(e)).sum(dim=1, keepdim=True) / total
    tok = s["tokens"].long()
    lp = torch.where(tok >= 0, (u.gather(1, tok.clamp(min=0)[:, None]) - log_total).squeeze(1), torch.zeros_like(m[:, 0]))
    out = {"logprob": lp, "entropy": entropy.squeeze(1)}
    if c["top"]:
        ids = _top_keys(z, c["top"])
        out["top_ids"] = ids.to(torch.int32)
        out["top_logprobs"] = u.gather(1, ids) - log_total
    return out


def _plain_distill(s):
    c = s["case"]
    N, V = s["logits"].shape
    ids = s["teacher_ids"].long()
    used = ids >= 0
    at = ids.clamp(min=0)
    z = s["logits"].float()
    top = z.max(dim=1, keepdim=True).values
    e = torch.exp((z - top) / c["T"])
    # the loss is a difference of logarithms that nearly cancel: the few terms it is made of stay in 64 bits
    total = e.sum(dim=1, keepdim=True, dtype=torch.float64)
    p = torch.where(used, torch.exp(s["teacher_logprobs"].double()), torch.zeros((), dtype=torch.float64, device="cuda"))
    if not c["tail"]:
        mass = p.sum(dim=1, keepdim=True)
        p = torch.where(mass > 0, p / mass, p)
    logq = (z.gather(1, at).double() - top.double()) / c["T"] - torch.log(total)
    loss = torch.where(p > 0, p * (torch.log(p) - logq), torch.zeros_like(p)).sum(dim=1)
    beta = p.sum(dim=1, keepdim=True)
    alpha = beta
    if c["tail"]:
        rest_mass = (1.0 - beta).clamp(min=0.0)
        live = used.any(dim=1, keepdim=True)
        rest_mass = torch.where(live, rest_mass, torch.zeros_like(rest_mass))
        listed_words = torch.zeros((N, V + 1), dtype=torch.bool, device="cuda")
        listed_words.scatter_(1, torch.where(used, at, torch.full_like(at, V)), True)
        rest = e.masked_fill(listed_words[:, :V], 0.0).sum(dim=1, keepdim=True,
                                                                                dtype=torch.float64)
        log_rest = torch.log(rest) - torch.log(total)
        loss = loss + torch.where(rest_mass > 0, rest_mass * (torch.log(rest_mass) - log_rest),
                                  torch.zeros_like(rest_mass)).squeeze(1)
        beta = beta + rest_mass
        alpha = beta - torch.where(rest > 0, rest_mass * (total / rest), torch.zeros_like(rest_mass))
        factor = torch.where(listed_words[:, :V], beta.float(), alpha.float())
    else:
        factor = beta.float()
    w = s["weight"]
    if w is not None:
        loss = torch.where(w != 0, loss, torch.zeros_like(loss))
    out = {"loss": loss.float()}
    if c["grad"]:
        d = e * (factor / total.float())
        d.scatter_add_(1, at, -p.float())                      # (unused entries carry no mass)
        d *= (1.0 / c["T"] if w is None else (w / c["T"])[:, None])
        out["dlogits"] = d.to(s["logits"].dtype)
    return out


def _plain_route(s):
    c = s["case"]
    N, E = s["logits"].shape
    z = s["logits"].double()
    if c["score"] == "softmax":
        r = torch.exp(z - z.max(dim=1, keepdim=True).values)
        r = r / r.sum(dim=1, keepdim=True)
    else:
        r = 1.0 / (1.0 + torch.exp(-z))
    sel = z if s["bias"] is None else r + s["bias"].double()
    if c["groups"] > 1:
        by = (r if s["bias"] is None else sel).view(N, c["groups"], E // c["groups"])
        by = by.topk(2 if c["top2"] else 1, dim=2).values.sum(dim=2)
        kept = torch.sort(by, dim=1, descending=True, stable=True).indices[:, :c["keep"]]
        allowed = torch.zeros((N, c["groups"]), dtype=torch.bool, device="cuda").scatter_(1, kept, True)
        sel = sel.masked_fill(~allowed.repeat_interleave(E // c["groups"], dim=1), NEG_INF)
    ids = torch.sort(sel, dim=1, descending=True, stable=True).indices[:, :c["k"]]
    w = r.gather(1, ids)
    if c["norm"]:
        w = w / w.sum(dim=1, keepdim=True)
    w = w * c["scale"]
    flat = ids.reshape(-1)
    perm = torch.sort(flat, stable=True).indices
    ends = (flat[None, :] == torch.arange(E, device="cuda")[:, None]).sum(dim=1).cumsum(0)
    offsets = torch.cat([ends.new_zeros(1), ends])
    return {"topk_ids": ids.to(torch.int32), "topk_w": w.float(), "offsets": offsets.to(torch.int32),
            "perm": perm.to(torch.int32)}


def _plain_route_grad(s):
    c = s["case"]
    z = s["logits"].float()
    ids = s["topk_ids"].long()
    g = s["d_topk_w"] * c["scale"]
    if c["score"] == "softmax":
        r = torch.exp(z - z.max(dim=1, keepdim=True).values)
        r = r / r.sum(dim=1, keepdim=True)
    else:
        r = 1.0 / (1.0 + torch.exp(-z))
    chosen = r.gather(1, ids)
    if c["norm"]:
        total = chosen.sum(dim=1, keepdim=True)
        g = (g - (g * chosen).sum(dim=1, keepdim=True) / total) / total
    d = torch.zeros_like(z).scatter_add_(1, ids, g)
    if c["score"] == "softmax":
        d = r * (d - (d * r).sum(dim=1, keepdim=True))
    else:
        d = d * r * (1.0 - r)
    return d.to(s["logits"].dtype)


# ---- one pass ------------------------------------------------------------------------------------------------------
def run(state):
    c = state["case"]
    if not own:
        return {"logprobs": _plain_logprobs, "distill": _plain_distill, "route": _plain_route,
                "route_grad": _plain_route_grad}[c["op"]](state)
    binding, ctx = _own()
    if c["op"] == "logprobs":
        return binding.spec_token_logprobs(ctx, state["logits"], state["tokens"], top_n=c["top"], temperature=c["T"])
    if c["op"] == "distill":
        return binding.spec_distill_topk(ctx, state["logits"], state["teacher_ids"], state["teacher_logprobs"],
                                         tail=c["tail"], temperature=c["T"], row_weight=state["weight"],
                                         grad=c["grad"])
    score = 1 if c["score"] == "sigmoid" else 0
    if c["op"] == "route":
        return binding.moe_route_tokens(ctx, state["logits"], c["k"], score_fn=score, norm_topk=int(c["norm"]),
                                        routed_scale=c["scale"], select_bias=state["bias"], n_groups=c["groups"],
                                        topk_groups=c["keep"], group_score=1 if c["top2"] else 0)
    return binding.moe_route_tokens_backward(ctx, state["logits"], state["topk_ids"], state["d_topk_w"],
                                             score_fn=score, norm_topk=int(c["norm"]), routed_scale=c["scale"])


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------
def _rows(N, width):
    """Row ranges small enough for a few 64-bit temporaries of ``width`` columns."""
    step = max(1, (1 << 25) // max(1, width))
    return [(a, min(N, a + step)) for a in range(0, N, step)]


def _exact_logprobs(s, c):
    parts = []
    for a, b in _rows(c["N"], c["V"]):
        z = s["logits"][a:b].to(torch.float64)
        logp = torch.log_softmax(z / c["T"], dim=1)
        prob = torch.exp(logp)
        row = {"logprob": torch.stack([logp[i, t] if t >= 0 else logp.new_zeros(()) for i, t in
                                       enumerate(s["tokens"][a:b].tolist())]),
               "entropy": -(prob * logp.masked_fill(prob == 0, 0.0)).sum(dim=1)}
        if c["top"]:
            order = torch.argsort(z, dim=1, descending=True, stable=True)[:, :c["top"]]
            row["top_ids"] = order.to(torch.int32)
            row["top_logprobs"] = torch.take_along_dim(logp, order, dim=1)
        parts.append(row)
    return {key: torch.cat([p[key] for p in parts]) for key in parts[0]}


def _exact_distill(s, c):
    losses, grads = [], []
    for a, b in _rows(c["N"], c["V"]):
        z = s["logits"][a:b].to(torch.float64)
        logq = torch.log_softmax(z / c["T"], dim=1)
        q = logq.exp()
        # the teacher as a dense vector of probabilities and a membership vector, row by row
        ids, lp = s["teacher_ids"][a:b].long(), s["teacher_logprobs"][a:b].to(torch.float64)
        p, member = torch.zeros_like(z), torch.zeros_like(z, dtype=torch.bool)
        r, j = torch.nonzero(ids >= 0, as_tuple=True)
        p[r, ids[r, j]] = lp[r, j].exp()
        member[r, ids[r, j]] = True
        some = member.any(dim=1)
        if c["tail"]:
            rest_p = torch.where(some, (1.0 - p.sum(dim=1)).clamp_min(0.0), torch.zeros_like(p[:, 0]))
            rest_q = (q * ~member).sum(dim=1)
        else:
            p = p / torch.where(some, p.sum(dim=1), torch.ones_like(p[:, 0]))[:, None]
            rest_p = rest_q = torch.zeros_like(p[:, 0])
        loss = torch.special.xlogy(p, p).sum(dim=1) - (p * logq).masked_fill(p == 0, 0.0).sum(dim=1)
        on = rest_p > 0
        loss = loss + torch.where(on, rest_p * (rest_p.clamp_min(1e-300).log() - rest_q.clamp_min(1e-300).log()),
                                  torch.zeros_like(loss))
        w = torch.ones_like(loss) if s["weight"] is None else s["weight"][a:b].to(torch.float64)
        losses.append(torch.where(w != 0, loss, torch.zeros_like(loss)))
        if c["grad"]:
            # sum over the buckets: d(-p_j log q_j) = p_j (q - 1_j); d(-rest log rest_q) = rest (q - q 1_rest / rest_q)
            d = q * p.sum(dim=1, keepdim=True) - p
            share = torch.where(on & (rest_q > 0), rest_p / rest_q.clamp_min(1e-300), torch.zeros_like(rest_p))
            d = d + rest_p[:, None] * q - share[:, None] * (q * ~member)
            grads.append(d * (w / c["T"])[:, None])
    out = {"loss": torch.cat(losses)}
    if c["grad"]:
        out["dlogits"] = torch.cat(grads)
    return out


def _exact_route(s, c):
    z = s["logits"].to(torch.float64)
    r = torch.softmax(z, dim=1) if c["score"] == "softmax" else torch.sigmoid(z)
    per = c["E"] // c["groups"]
    want = z.clone() if s["bias"] is None else r + s["bias"].to(torch.float64)
    if c["groups"] > 1:
        chosen_by = r if s["bias"] is None else want
        best = torch.stack([torch.sort(chosen_by[:, i * per:(i + 1) * per], dim=1, descending=True)
                            .values[:, :2 if c["top2"] else 1].sum(dim=1) for i in range(c["groups"])], dim=1)
        for i in range(c["groups"]):
            # a group stays if fewer than ``keep`` groups come before it (higher, or equal with a lower number)
            before = (best > best[:, i:i + 1]).sum(dim=1) + (best[:, :i] == best[:, i:i + 1]).sum(dim=1)
            want[before >= c["keep"], i * per:(i + 1) * per] = NEG_INF
    ids = []
    left = want
    for _ in range(c["k"]):
        top = left.max(dim=1, keepdim=True).values
        first = (left == top).to(torch.int8).argmax(dim=1, keepdim=True)
        ids.append(first)
        left = left.scatter(1, first, NEG_INF)
    ids = torch.cat(ids, dim=1)
    w = torch.take_along_dim(r, ids, dim=1)
    w = c["scale"] * (w / w.sum(dim=1, keepdim=True) if c["norm"] else w)
    flat = ids.reshape(-1).cpu()
    count = torch.bincount(flat, minlength=c["E"])
    offsets = torch.cat([torch.zeros(1, dtype=torch.int64), torch.cumsum(count, 0)])
    pairs = torch.argsort(flat * flat.numel() + torch.arange(flat.numel()))
    return {"topk_ids": ids.to(torch.int32), "topk_w": w, "offsets": offsets.to(torch.int32).cuda(),
            "perm": pairs.to(torch.int32).cuda()}


def _exact_route_grad(s, c):
    z = s["logits"].to(torch.float64).requires_grad_(True)
    r = torch.softmax(z, dim=1) if c["score"] == "softmax" else torch.sigmoid(z)
    w = torch.take_along_dim(r, s["topk_ids"].long(), dim=1)
    w = c["scale"] * (w / w.sum(dim=1, keepdim=True) if c["norm"] else w)
    return torch.autograd.grad(w, z, s["d_topk_w"].to(torch.float64))[0]


def exact(case, seed):
    c = dict(case)
    s = prepare(c, seed)
    return {"logprobs": _exact_logprobs, "distill": _exact_distill, "route": _exact_route,
            "route_grad": _exact_route_grad}[c["op"]](s, c)
